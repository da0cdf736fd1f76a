"""The native part of the training operators' binding refuses what it cannot take before any call of the library.  No GPU."""
import sys
import types

import pytest
import torch


@pytest.fixture(scope="module")
def native():
    from paper_2304_14463_amd import training
    return training._bound()


@pytest.mark.parametrize("version", [None, 0], ids=["missing", "of another version"])
def test_native_part_that_does_not_fit_the_binding(monkeypatch, version):
    """... is refused with the command that builds it."""
    import paper_2304_14463_amd
    from paper_2304_14463_amd import training
    other = None if version is None else types.ModuleType("paper_2304_14463_amd._training")
    if other is not None:
        other.training_version, other.__file__ = version, "elsewhere.so"
    monkeypatch.setitem(sys.modules, "paper_2304_14463_amd._training", other)
    monkeypatch.delattr(paper_2304_14463_amd, "_training", raising=False)
    if other is not None:
        monkeypatch.setattr(paper_2304_14463_amd, "_training", other, raising=False)
    monkeypatch.setattr(training, "_native", None)
    with pytest.raises(RuntimeError, match="paper_2304_14463_amd.build"):
        training._bound()


@pytest.mark.parametrize("call", ["checkpoint_write", "checkpoint_read", "norm_forward", "norm_backward", "linear_forward", "linear_backward_input", "linear_backward_weight", "bind"])
def test_wrong_numbers_of_arguments(native, call):
    with pytest.raises(TypeError):
        getattr(native, call)()
    with pytest.raises(TypeError):
        getattr(native, call)(*[None] * 20)


def test_what_is_no_tensor_is_refused(native):
    from paper_2304_14463_amd import training as tr
    for bad in (None, 3, [1.0], "x"):
        for call in (lambda: tr.moc_checkpoint_write(bad), lambda: tr.moc_checkpoint_read(bad, torch.float32), lambda: tr.moc_norm_forward(bad), lambda: tr.moc_linear_forward(bad, bad),
                     lambda: tr.moc_norm_backward(bad, bad, None, bad, bad), lambda: tr.moc_linear_backward_input(bad, bad), lambda: tr.moc_linear_backward_weight(bad, bad)):
            with pytest.raises(TypeError):
                call()
    kept = tr.empty_checkpoint(4, 64, "int8", "cpu")
    kept.codes = None
    with pytest.raises(ValueError):
        tr.moc_checkpoint_read(kept, torch.float32)
    with pytest.raises(TypeError):
        native.bind(tr.Checkpoint, None, {})
    with pytest.raises(KeyError):
        native.bind(tr.Checkpoint, len, {})
    with pytest.raises(ValueError):   # what was bound stays
        tr.moc_checkpoint_write(torch.zeros(4, 64))
