"""The training operators inside torch's autograd: results are tensors of their own."""
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
