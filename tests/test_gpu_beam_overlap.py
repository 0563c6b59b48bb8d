"""Results of a reordering that share memory with something else of the call are refused before
anything is launched; those that only lie between its rows are not. On the GPU against the
oracle."""
import numpy as np
import pytest

from oracle import beam as obeam
from test_gpu_q4 import sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def test_results_that_overlap_are_refused(sq, torch):  # noqa: F811
    a, b, c = (torch.randn(4, 6).cuda() for _ in range(3))
    flat = torch.randn(60).cuda()
    wide = torch.randn(4, 2, 12).cuda()
    p = torch.tensor([[1, 0], [0, 0]]).cuda()
    tokens = torch.randint(9, (4,)).cuda()
    held = [t.clone() for t in (a, b, c, flat, wide, p, tokens)]
    for states, out in (([a, a], [a, b]), ([a, a], [b, a]),                 # a is read for b while it is moved
                        ([flat[:24].view(4, 6)], [flat[5:29].view(4, 6)]),  # begins inside its own state
                        ([a, flat[30:54].view(4, 6)], [flat[:24].view(4, 6), flat[23:47].view(4, 6)]),
                        ([a, b], [flat[:24].view(4, 6), flat[20:44].view(4, 6)]),
                        ([a, wide], [wide[:, 1, 3:9], torch.empty_like(wide)]),
                        ([wide[:, 0, :8]], [wide[:, 0, 4:]]),
                        ([wide, wide[:, 0]], [torch.empty_like(wide), wide[:, 0]]),
                        ([tokens], [p.view(-1)])):
        with pytest.raises(ValueError):
            sq.beam_reorder(states, p, out=out)
    for t, before in zip((a, b, c, flat, wide, p, tokens), held):
        assert torch.equal(t, before)


def test_results_between_rows_of_others(sq, torch):  # noqa: F811
    g = torch.Generator().manual_seed(1)
    p = torch.tensor([[1, 0, 1], [2, 2, 0]])
    cache = torch.randn(6, 5, 2, 3, 20, 16, generator=g).cuda()     # [rows][layer][key or value][heads][room][width]
    other = torch.zeros_like(cache)
    views = [cache[:, k, v, :, :11] for k in range(5) for v in range(2)]
    ref = [obeam.reorder(t.cpu().numpy(), p.numpy()) for t in views]
    before = cache.clone()
    to = [other[:, k, v, :, :11] for k in range(5) for v in range(2)]
    sq.beam_reorder(views, p.cuda(), out=to)                        # from one tensor's layers to another's
    assert torch.equal(cache, before) and (other[..., 11:, :] == 0).all()
    sq.beam_reorder(views, p.cuda(), out=views)                     # and where they are
    assert torch.equal(cache[..., 11:, :], before[..., 11:, :])
    for v, t, r in zip(views, to, ref):
        assert np.array_equal(v.cpu().numpy(), r) and np.array_equal(t.cpu().numpy(), r)
    sq.beam_reorder(cache[:, 0], p.cuda(), out=cache[:, 1])         # one layer's rows into the next's
    assert np.array_equal(cache[:, 1].cpu().numpy(), obeam.reorder(cache[:, 0].cpu().numpy(), p.numpy()))
    # one state for two results, and shared states that nothing writes
    got = sq.beam_reorder([cache, cache], p.cuda(), out=[torch.empty_like(cache), torch.empty_like(cache)])
    assert torch.equal(got[0], got[1])
