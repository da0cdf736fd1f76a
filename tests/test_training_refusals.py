"""Arguments that the training operators refuse before anything touches a device.  No GPU."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, F16, BF16, E4M3, I8 = range(5)
A = 1 << 20   # an aligned address; nothing looks at it


@pytest.fixture(scope="module")
def lib():
    from paper_2304_14463_amd import training
    return training.lib()


def mat(type_, cols=64, stride=None, data=A, scales=None, scale_stride=None, reserved=0):
    from paper_2304_14463_amd.training import Matrix
    kept = type_ in (E4M3, I8)
    return Matrix(data, (A if scales is None else scales) if kept else None, cols if stride is None else stride,
                  ((cols + 31) // 32 if scale_stride is None else scale_stride) if kept else 0, type_, reserved)


def test_header_and_binding_agree():
    from paper_2304_14463_amd import moccasin, training
    text = open(os.path.join(ROOT, "include", "moccasin_training.h")).read()
    code = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(moc_[a-z_]+)\s*\(", code))
    assert declared == set(training.EXPORTS)
    L = ctypes.CDLL(moccasin.LIB_PATH)
    for name in declared:
        assert hasattr(L, name), name
    assert L.moc_training_version() == training.MOC_TRAINING_VERSION == int(re.search(r"#define MOC_TRAINING_VERSION (\d+)", text).group(1))
    for name in ("F32", "F16", "BF16", "E4M3", "I8"):
        assert int(re.search(rf"#define MOC_{name}\s+(\d+)", text).group(1)) == getattr(training, f"MOC_{name}")
    for name, value in training.ACTS.items():
        assert int(re.search(rf"#define MOC_ACT_{name.upper()} (\d+)", text).group(1)) == value
    assert ctypes.sizeof(training.Matrix) == 40


def test_library_without_the_operators_is_refused(monkeypatch):
    from paper_2304_14463_amd import moccasin, training
    monkeypatch.setattr(training, "_lib", None)
    monkeypatch.setattr(moccasin, "lib", lambda: object())
    with pytest.raises(RuntimeError, match="paper_2304_14463_amd.build"):
        training.lib()


BAD_VALUES = [None, mat(7), mat(-1), mat(BF16, stride=63), mat(BF16, data=None), mat(BF16, data=A + 1), mat(F32, data=A + 2), mat(BF16, stride=1 << 23), mat(BF16, reserved=1), mat(E4M3)]
BAD_KEPT = [None, mat(BF16), mat(E4M3, data=None), mat(I8, scales=0), mat(I8, scale_stride=1), mat(E4M3, stride=10), mat(I8, scale_stride=1 << 23)]


def test_checkpoint_refusals(lib):
    w, r = lib.moc_checkpoint_write, lib.moc_checkpoint_read
    for x in BAD_VALUES:
        assert w(4, 64, x, mat(I8), None) == -1
        assert r(4, 64, mat(I8), 0, x, None) == -1
    for k in BAD_KEPT:
        assert w(4, 64, mat(BF16), k, None) == -1
        assert r(4, 64, k, 0, mat(BF16), None) == -1
    for rows, cols in ((-1, 64), (4, -1), (1 << 31, 64), (4, 1 << 23)):
        assert w(rows, cols, mat(BF16), mat(I8), None) == -1 and r(rows, cols, mat(I8), 0, mat(BF16), None) == -1
    for act in (-1, 4):
        assert r(4, 64, mat(I8), act, mat(BF16), None) == -1
    # nothing to do: no device is asked
    assert w(0, 64, mat(BF16, data=None), mat(I8, data=None), None) == 0
    assert r(0, 64, mat(I8, data=None), 0, mat(BF16, data=None), None) == 0


def test_norm_refusals(lib):
    f, b = lib.moc_norm_forward, lib.moc_norm_backward
    good = mat(BF16)
    for x in (BAD_VALUES[:-1]):
        assert f(4, 64, x, None, None, 0, 1e-5, good, None, A, A, None) == -1
        assert f(4, 64, good, None, None, 0, 1e-5, x, None, A, A, None) == -1
        assert b(4, 64, x, good, None, 0, A, A, None, good, None, None, None, 0, None) == -1
        assert b(4, 64, good, x, None, 0, A, A, None, good, None, None, None, 0, None) == -1
        assert b(4, 64, good, good, None, 0, A, A, None, x, None, None, None, 0, None) == -1
        if x is not None:
            assert b(4, 64, good, good, None, 0, A, A, x, good, None, None, None, 0, None) == -1
    for k in BAD_KEPT[1:]:
        assert f(4, 64, good, None, None, 0, 1e-5, good, k, A, A, None) == -1
    for bad in ((4, 0), (-1, 64)):
        assert f(*bad, good, None, None, 0, 1e-5, good, None, A, A, None) == -1
    for eps in (-1.0, float("nan")):
        assert f(4, 64, good, None, None, 0, eps, good, None, A, A, None) == -1
    for mean, rstd in ((None, A), (A, None), (A + 2, A)):
        assert f(4, 64, good, None, None, 0, 1e-5, good, None, mean, rstd, None) == -1
        assert b(4, 64, good, good, None, 0, mean, rstd, None, good, None, None, None, 0, None) == -1
    assert f(4, 64, good, A, None, 3, 1e-5, good, None, A, A, None) == -1          # gamma as a checkpoint
    assert f(4, 64, good, A + 2, None, 0, 1e-5, good, None, A, A, None) == -1      # misaligned
    assert b(4, 64, good, good, None, 0, A, A, None, good, A, None, A, 1 << 20, None) == -1   # one of the two
    assert f(0, 64, mat(BF16, data=None), None, None, 0, 1e-5, mat(BF16, data=None), None, None, None, None) == 0
    assert b(0, 64, good, good, None, 0, None, None, None, good, None, None, None, 0, None) == 0
    assert lib.moc_norm_backward_work(4, 0) == -1 and lib.moc_norm_backward_work(-4, 8) == -1


def test_linear_refusals(lib):
    f, i, w = lib.moc_linear_forward, lib.moc_linear_backward_input, lib.moc_linear_backward_weight
    good = mat(BF16)
    for x in BAD_VALUES + [mat(F32), mat(F16)]:
        assert f(4, 64, 64, x, good, None, 0, 0, None, good, None, None, 0, None) == -1
        assert f(4, 64, 64, good, x, None, 0, 0, None, good, None, None, 0, None) == -1
        assert i(4, 64, 64, x, good, 0, None, good, None, 0, None) == -1
        assert i(4, 64, 64, good, x, 0, None, good, None, 0, None) == -1
        assert w(4, 64, 64, x, good, good, None, None, 0, None) == -1
    for x in BAD_VALUES + [mat(F16)]:
        assert f(4, 64, 64, good, good, None, 0, 0, None, x, None, None, 0, None) == -1
        assert i(4, 64, 64, good, good, 0, None, x, None, 0, None) == -1
        assert w(4, 64, 64, good, good, x, None, None, 0, None) == -1
        if x is not None:
            assert f(4, 64, 64, good, good, None, 0, 0, x, good, None, None, 0, None) == -1
    for k in BAD_KEPT[1:]:
        assert f(4, 64, 64, good, good, None, 0, 0, None, good, k, None, 0, None) == -1
    for sizes in ((-1, 64, 64), (4, -1, 64), (4, 64, -1), (4, 1 << 23, 64), (4, 64, 1 << 23), (1 << 31, 64, 64)):
        assert f(*sizes, good, good, None, 0, 0, None, good, None, None, 0, None) == -1
        assert i(*sizes, good, good, 0, None, good, None, 0, None) == -1
        assert w(*sizes, good, good, good, None, None, 0, None) == -1
        assert lib.moc_linear_work(*sizes) == -1
    for act in (-1, 4):
        assert f(4, 64, 64, good, good, None, 0, act, None, good, None, None, 0, None) == -1
        assert i(4, 64, 64, good, good, act, good, good, None, 0, None) == -1
    assert i(4, 64, 64, good, good, 2, None, good, None, 0, None) == -1            # an activation without its argument
    assert i(4, 64, 64, good, good, 2, mat(F16), good, None, 0, None) == -1
    assert i(4, 64, 64, good, good, 2, mat(I8, scale_stride=1), good, None, 0, None) == -1
    assert w(4, 64, 64, good, mat(F32), good, None, None, 0, None) == -1 and w(4, 64, 64, good, mat(F16), good, None, None, 0, None) == -1
    assert w(4, 64, 64, good, good, good, A + 2, None, 0, None) == -1
    assert f(4, 64, 64, good, good, A, 4, 0, None, good, None, None, 0, None) == -1   # bias as a checkpoint
    none = mat(BF16, data=None)
    assert f(0, 64, 64, none, good, None, 0, 0, None, none, None, None, 0, None) == 0
    assert i(0, 64, 64, none, good, 0, None, none, None, 0, None) == 0
    assert w(4, 64, 0, mat(BF16, cols=0, stride=64), good, none, None, None, 0, None) == 0


def test_tensors_off_the_gpu_are_refused():
    import torch

    from paper_2304_14463_amd import training as tr
    x = torch.zeros(4, 64)
    for call in (lambda: tr.moc_checkpoint_write(x), lambda: tr.moc_norm_forward(x), lambda: tr.moc_linear_forward(x.bfloat16(), x.bfloat16()),
                 lambda: tr.moc_checkpoint_read(tr.empty_checkpoint(4, 64, "int8", "cpu"), torch.float32), lambda: tr.Checkpoint(x, x, "fp4")):
        with pytest.raises(ValueError):
            call()
