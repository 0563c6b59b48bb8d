"""Tensors that a caller gives for results count as changed in place: a backward pass that needs
what they held before ends in autograd's error, not in gradients of the new values."""
import pytest

from test_gpu_q4 import sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def test_reordered_states(sq, torch):  # noqa: F811
    p = torch.tensor([[1, 0], [0, 0]]).cuda()
    x = torch.randn(4, 6).cuda().requires_grad_()
    state, other, to = x.exp(), torch.randn(4, 6).cuda(), torch.zeros(4, 6).cuda()   # exp keeps its result
    loss = (state * other).sum() + (x * to).sum()
    versions = [t._version for t in (state, other, to)]
    sq.beam_reorder([other], p)
    sq.beam_reorder([other], p, out=[to])
    sq.beam_reorder([state.detach()], p, out=[state.detach()])
    assert [t._version for t in (state, other, to)] == [versions[0] + 1, versions[1], versions[2] + 1]
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        s = torch.randn(4, 6).cuda()
        before = s.clone()
        assert torch.equal(sq.beam_reorder(s, p, out=s), before[[1, 0, 2, 2]])
    assert sq.beam_reorder([], p, out=[]) == []


def test_gradient_of_log_probabilities(sq, torch):  # noqa: F811
    x = torch.randn(5, 40).cuda().requires_grad_()
    logits = x.tanh()                                   # keeps its result
    tokens = torch.arange(5).cuda()
    held = logits.detach()
    r = sq.token_logprobs(held, tokens)
    g = torch.ones(5).cuda()
    fresh = sq.token_logprobs_backward(held, tokens, r.lse, grad_logprob=g)
    assert held._version == 0
    got = sq.token_logprobs_backward(held, tokens, r.lse, grad_logprob=g, out=held)
    assert got is held and torch.equal(got, fresh) and held._version == 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        logits.sum().backward()
