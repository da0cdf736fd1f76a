"""What the C ABI of the operators around a plan's layers refuses before anything touches a device.  No GPU."""
import ctypes

import pytest

F32, F16, BF16, E4M3, I8 = range(5)
A = 1 << 20   # an aligned address; nothing looks at it
P, I32, I64, U64, D, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_double, ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    from paper_2304_14463_amd import training
    return training.lib()


class Tensor(ctypes.Structure):
    """moc_adamw_tensor"""
    _fields_ = [("param", P), ("grad", P), ("m", P), ("v", P), ("m_scales", P), ("v_scales", P), ("copy", P), ("count", I64), ("param_type", I32), ("grad_type", I32),
                ("moment_type", I32), ("copy_type", I32), ("decay", F), ("reserved", I32)]


class Rule(ctypes.Structure):
    """moc_adamw_rule"""
    _fields_ = [("lr", D), ("beta1", D), ("beta2", D), ("eps", D), ("grad_scale", D), ("step", I64), ("seed", U64), ("lr_at", P), ("grad_scale_at", P), ("step_at", P)]


class Read(ctypes.Structure):
    """moc_moments_tensor"""
    _fields_ = [("m", P), ("v", P), ("m_scales", P), ("v_scales", P), ("m_values", P), ("v_values", P), ("count", I64), ("moment_type", I32), ("value_type", I32)]


def test_adamw(lib):
    def call(tensors=1, rule=None, **changed):
        t = Tensor(A, A, A, A, A, A, None, 64, F32, BF16, E4M3, F16, 0.1, 0)
        r = Rule(1e-3, 0.9, 0.999, 1e-8, 1.0, 1, 0, None, None, None)
        for k, v in changed.items():
            setattr(r if k in dict(Rule._fields_) else t, k, v)
        return lib.moc_adamw_step(tensors, ctypes.byref(t), ctypes.byref(r) if rule is None else rule, None)

    nan, inf = float("nan"), float("inf")
    for bad in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(m_scales=None), dict(v_scales=None), dict(param=A + 2), dict(grad=A + 1), dict(param_type=E4M3), dict(grad_type=5),
                dict(moment_type=F16), dict(moment_type=I8), dict(moment_type=F32, m=A + 2), dict(moment_type=F32, v=A + 1), dict(copy=A, copy_type=F32), dict(copy=A + 1), dict(count=-1),
                dict(count=(1 << 40) + 1), dict(decay=-0.1), dict(decay=nan), dict(decay=inf), dict(reserved=1), dict(lr=nan), dict(lr=1e300), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.5), dict(beta2=nan),
                dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-50), dict(eps=nan), dict(grad_scale=inf), dict(step=0), dict(step=-5), dict(lr_at=A + 2), dict(step_at=A + 4), dict(grad_scale_at=A + 1),
                dict(tensors=-1)):
        assert call(**bad) == -1, bad
    assert lib.moc_adamw_step(1, None, ctypes.byref(Rule(1e-3, 0.9, 0.999, 1e-8, 1.0, 1)), None) == -1
    assert lib.moc_adamw_step(1, ctypes.byref(Tensor()), None, None) == -1
    # nothing to do: no device is asked
    assert call(tensors=0) == 0 and call(count=0, param=None, m=None) == 0


def test_moments_read(lib):
    def call(tensors=1, **changed):
        t = Read(A, A, A, A, A, A, 64, E4M3, BF16)
        for k, v in changed.items():
            setattr(t, k, v)
        return lib.moc_moments_read(tensors, ctypes.byref(t), None)

    for bad in (dict(m=None), dict(v=None), dict(m_scales=None), dict(v_scales=None), dict(m_values=None), dict(v_values=None), dict(m_values=A + 1), dict(v_values=A + 2, value_type=F32), dict(count=-1),
                dict(moment_type=BF16), dict(value_type=E4M3), dict(value_type=-1), dict(moment_type=F32, m=A + 2), dict(tensors=-1)):
        assert call(**bad) == -1, bad
    assert lib.moc_moments_read(1, None, None) == -1
    assert call(count=0, m=None) == 0 and call(tensors=0) == 0


class RowNorm(ctypes.Structure):
    """moc_row_norm"""
    _fields_ = [("kind", I32), ("param_type", I32), ("gamma", P), ("beta", P), ("mean", P), ("rstd", P), ("eps", F), ("reserved", I32)]


class Grads(ctypes.Structure):
    """moc_residual_grads"""
    _fields_ = [("before_gamma", P), ("before_beta", P), ("after_gamma", P), ("after_beta", P), ("gate", P)]


def mat(type_=BF16, cols=64, stride=None, data=A, reserved=0, scales=A):
    from paper_2304_14463_amd.training import Matrix
    return Matrix(data, scales if type_ in (E4M3, I8) else None, cols if stride is None else stride, 2, type_, reserved)


def row_norm(kind=1, **changed):
    n = RowNorm(kind, F32, A, A if kind == 1 else None, A, A, 1e-5, 0)
    for k, v in changed.items():
        setattr(n, k, v)
    return ctypes.byref(n)


BAD_NORMS = [dict(kind=3), dict(kind=-1), dict(param_type=E4M3), dict(param_type=-1), dict(gamma=A + 2), dict(beta=A + 1), dict(kind=2, beta=A), dict(mean=None), dict(rstd=None), dict(mean=A + 2), dict(rstd=A + 1),
             dict(eps=-1.0), dict(eps=float("nan")), dict(reserved=1)]
BAD_MATRICES = [mat(7), mat(-1), mat(stride=63), mat(data=None), mat(data=A + 1), mat(F32, data=A + 2), mat(stride=1 << 23), mat(reserved=1)]


def test_residual(lib):
    def forward(rows=8, cols=64, x=mat(), block=mat(), gate=mat(), gates=2, scale=1.0, after=row_norm(), before=row_norm(2), r=mat(), n=mat(), kept=None):
        return lib.moc_residual_forward(rows, cols, x, block, gate, gates, scale, after, before, r, n, kept, None)

    def backward(rows=8, cols=64, dr=mat(), dn=mat(), r=mat(), block=mat(), gate=mat(), gates=2, scale=1.0, after=row_norm(), before=row_norm(), dx=mat(), dblock=mat(),
                 grads=Grads(A, A, A, A, A), work=A, work_bytes=0):
        return lib.moc_residual_backward(rows, cols, dr, dn, r, block, gate, gates, scale, after, before, dx, dblock, None if grads is None else ctypes.byref(grads), work, work_bytes, None)

    sizes = [dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=16385), dict(gates=-1), dict(gates=3), dict(gates=16), dict(gates=0), dict(gate=None)]
    for bad in sizes + [dict(scale=float("nan")), dict(scale=float("inf"))] + [dict(after=row_norm(**k)) for k in BAD_NORMS] + [dict(before=row_norm(**k)) for k in BAD_NORMS] + [dict(gate=mat(E4M3))]:
        assert forward(**bad) == -1 and backward(**bad) == -1, bad
    for k in ("x", "block", "gate", "r", "n"):
        for m in BAD_MATRICES:
            assert forward(**{k: m}) == -1, k
    for k in ("dr", "dn", "r", "block", "gate", "dx", "dblock"):
        for m in BAD_MATRICES:
            assert backward(**{k: m}) == -1, k
    for bad in (dict(block=None), dict(x=mat(I8)), dict(r=mat(E4M3)), dict(n=mat(E4M3)), dict(n=None), dict(before=None), dict(before=row_norm(0)), dict(r=None, n=None, before=None), dict(kept=mat()),
                dict(kept=mat(I8, data=None)), dict(kept=mat(I8, scales=None)), dict(kept=mat(I8), n=None, before=None)):
        assert forward(**bad) == -1, bad
    for bad in (dict(dn=None), dict(before=None), dict(dr=None, dn=None, before=None), dict(r=None), dict(block=None), dict(dr=mat(E4M3)), dict(dn=mat(I8)), dict(dx=mat(E4M3)), dict(dblock=mat(I8)),
                dict(grads=Grads(A + 2)), dict(grads=Grads(None, A + 1)), dict(grads=Grads(None, None, A + 2)), dict(grads=Grads(None, None, None, None, A + 2)), dict(before=row_norm(2)), dict(after=row_norm(2)),
                dict(after=None), dict(gate=None, gates=0), dict(block=None, after=None, grads=Grads(None, None, None, None, A))):
        assert backward(**bad) == -1, bad
    none = mat(data=None)
    assert forward(rows=0, x=none, block=none, r=none, n=none, gates=1) == 0
    assert backward(rows=0, dr=none, dn=none, r=none, block=none, dx=none, dblock=none, gates=1, grads=None) == 0
    for bad in ((-1, 64, 0), (8, 0, 0), (8, 64, 3), (8, 16385, 0), (8, 64, -1)):
        assert lib.moc_residual_backward_work(*bad) == -1


def test_logprob(lib):
    def forward(rows=4, vocab=64, logits=mat(), tokens=A, bytes_=8, scale=1.0, top=5, logp=A, lse=A, entropy=A, top_logp=A, top_tokens=A):
        return lib.moc_logprob_forward(rows, vocab, logits, tokens, bytes_, scale, top, logp, lse, entropy, top_logp, top_tokens, None, 0, None)

    def backward(rows=4, vocab=64, logits=mat(), lse=A, entropy=A, tokens=A, bytes_=8, dlogp=A, dentropy=A, scale=1.0, out=mat()):
        return lib.moc_logprob_backward(rows, vocab, logits, lse, entropy, tokens, bytes_, dlogp, dentropy, scale, out, None)

    matrices = [None, mat(7), mat(E4M3), mat(I8), mat(stride=63), mat(data=None), mat(data=A + 1), mat(F32, data=A + 2), mat(stride=1 << 23), mat(reserved=1)]
    nan, inf = float("nan"), float("inf")
    for bad in [dict(logits=x) for x in matrices] + [dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=-1), dict(vocab=1 << 23), dict(bytes_=2), dict(tokens=A + 4), dict(tokens=A + 2, bytes_=4),
                                                     dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(scale=inf), dict(scale=1e30), dict(scale=1e-30)]:
        assert forward(**bad) == -1 and backward(**bad) == -1, bad
    for bad in (dict(top=-1), dict(top=65), dict(vocab=4, logits=mat(cols=4)), dict(logp=None), dict(tokens=None), dict(lse=None), dict(entropy=None), dict(top_logp=None), dict(top_tokens=None),
                dict(logp=A + 2), dict(lse=A + 1), dict(entropy=A + 2), dict(top_logp=A + 2), dict(top_tokens=A + 4)):
        assert forward(**bad) == -1, bad
    for bad in [dict(out=x) for x in matrices] + [dict(out=mat(F16)), dict(lse=None), dict(lse=A + 2), dict(tokens=None), dict(dlogp=None), dict(dlogp=A + 1), dict(entropy=None), dict(entropy=A + 2), dict(dentropy=A + 2)]:
        assert backward(**bad) == -1, bad
    none = mat(data=None)
    assert forward(rows=0, logits=none, tokens=None, logp=None, lse=None, entropy=None) == 0 and backward(rows=0, logits=none, out=none, lse=None) == 0
    for sizes in ((-1, 64, 0), (4, 0, 0), (4, 64, 65), (4, 8, 9), (4, 64, -1)):
        assert lib.moc_logprob_forward_work(*sizes) == -1


def test_what_is_on_no_gpu(lib):
    import torch

    from paper_2304_14463_amd import training as tr
    x = torch.zeros(64)
    with pytest.raises(ValueError):
        tr.moc_adamw_step([x], [x], [tr.zero_moments(x)], 1e-3, 1)
    with pytest.raises(ValueError):
        tr.moc_moments_read([tr.zero_moments(x)])
    with pytest.raises(ValueError):
        tr.zero_moments(x, 16)
    assert tr.zero_moments(x).nbytes == 132 and tr.zero_moments(x, 32).nbytes == 512
    m = torch.zeros(4, 64)
    for call in (lambda: tr.moc_residual_forward(m, m.clone()), lambda: tr.moc_residual_backward(m, None), lambda: tr.moc_logprob_forward(m), lambda: tr.moc_logprob_backward(m, x[:4])):
        with pytest.raises(ValueError):
            call()
    for bad in (None, 3, [1.0], "x"):
        for call in (lambda: tr.moc_residual_forward(None, bad), lambda: tr.moc_residual_backward(bad, bad), lambda: tr.moc_logprob_forward(bad), lambda: tr.moc_logprob_backward(bad, bad)):
            with pytest.raises(TypeError):
                call()
    for bad in (None, 3, [3], [x, "y"]):
        with pytest.raises((TypeError, ValueError)):
            tr.moc_adamw_step(bad, [x], [tr.zero_moments(x)], 1e-3, 1)
