"""The training operators inside torch's autograd: results are tensors of their own, and what a call writes to counts as changed."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2304_14463_amd import training
    training.lib()
    return training


def test_log_probabilities_are_tensors_of_their_own(tr):
    """Returned by one function of autograd, each may be changed in place, and a change of one leaves what is saved of another alone."""
    class LogProbs(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, tokens):
            f = tr.moc_logprob_forward(logits, tokens)
            ctx.save_for_backward(logits, tokens, f.lse, f.entropy)
            return f.logp, f.entropy

        @staticmethod
        def backward(ctx, dlogp, dentropy):
            logits, tokens, lse, entropy = ctx.saved_tensors
            return tr.moc_logprob_backward(logits, lse, tokens, dlogp.contiguous(), entropy, dentropy.contiguous()), None

    for rows in (1, 5):
        x, tokens = torch.randn(rows, 100, device="cuda", requires_grad=True), torch.arange(rows, device="cuda")
        f = tr.moc_logprob_forward(x, tokens, top=2)
        assert len({t.untyped_storage().data_ptr() for t in f}) == 5 and not any(t._is_view() for t in f)
        f.logp.add_(1)
        assert f.logp._version == 1 and f.lse._version == f.entropy._version == 0
        logp, entropy = LogProbs.apply(x, tokens)
        logp.mul_(2.0)
        (logp.sum() + 0.5 * entropy.sum()).backward()
        y = x.detach().double().requires_grad_()
        logs = torch.log_softmax(y, 1)
        (2 * logs.gather(1, tokens[:, None]).sum() - 0.5 * (logs.exp() * logs).sum()).backward()
        assert float((x.grad - y.grad).abs().max()) < 1e-5   # 2^-24 by some ten roundings of values below 8


def test_what_a_step_writes_counts_as_changed(tr):
    """A graph that was recorded before a step of AdamW is refused afterwards, as after an update by torch; all that is written has a
    new version, what is read has not."""
    for bits in (32, 8):
        w, x = torch.randn(64, 64, device="cuda", requires_grad=True), torch.randn(8, 64, device="cuda", requires_grad=True)
        copy, moments, grad = torch.empty_like(w, dtype=torch.bfloat16, requires_grad=False), tr.zero_moments(w, bits), torch.randn_like(w)
        y = (x @ w).square().sum()
        tr.moc_adamw_step([w], [grad], [moments], 1e-3, 1, copies=[copy])
        assert w._version == copy._version == 1 and grad._version == 0
        assert all(t._version == 1 for t in (moments.m, moments.v, moments.m_scales, moments.v_scales) if t is not None)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
        (x @ w).sum().backward()
        values = tr.moc_moments_read([moments])
        assert moments.m._version == 1
        tr.moc_moments_read([moments], out=values)
        assert all(t._version == 1 for t in values[0])


def test_outputs_that_are_given_count_as_changed(tr):
    """One version more for each call that writes to them, none where it is refused."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x, y, w, stats = (torch.randn(*s, generator=g, device="cuda").half() for s in ((4, 64), (4, 64), (64, 64), (4,)))
    gamma, v, n = torch.ones(64, device="cuda"), stats.float().abs() + 1, tr.Norm("rms")
    out, kept, given = torch.empty_like(x), tr.empty_checkpoint(4, 64, "int8", "cuda"), x.clone()
    square = torch.empty_like(w)

    def after(call, *tensors):
        before = [t._version for t in tensors + (x, y, w, gamma, v)]
        call()
        assert [t._version - b for t, b in zip(tensors + (x, y, w, gamma, v), before)] == [1] * len(tensors) + [0] * 5

    after(lambda: tr.moc_checkpoint_write(x, out=kept), kept.codes, kept.scales)
    after(lambda: tr.moc_checkpoint_read(kept, torch.float16, out=out), out)
    after(lambda: tr.moc_norm_forward(x, gamma, keep=kept, out=out), out, kept.codes, kept.scales)
    after(lambda: tr.moc_norm_backward(x, y, gamma, v, v, out=out), out)
    after(lambda: tr.moc_linear_forward(x, w, keep=kept, out=out), out, kept.codes, kept.scales)
    after(lambda: tr.moc_linear_backward_input(x, w, out=out), out)
    after(lambda: tr.moc_linear_backward_weight(x, y, out=square), square)
    after(lambda: tr.moc_residual_forward(x, y, before=n, keep=kept, out=given, out_norm=out), given, out, kept.codes, kept.scales)
    after(lambda: tr.moc_residual_backward(x, y, x, before=n, before_stats=(None, v), out_x=given, out_block=out), given, out)
    after(lambda: tr.moc_logprob_backward(x, v, out=out), out)
    with pytest.raises(ValueError):
        after(lambda: tr.moc_logprob_backward(x, v[:3], out=out))
    with torch.inference_mode():   # tensors without a version
        room = torch.empty_like(x)
        tr.moc_logprob_backward(x, v, out=room)
    tr.moc_logprob_backward(x, v, out=room)
