"""Beam search's selection and reordering on the GPU against the oracle.

Bars: a row's sum of exponentials errs by less than 2e-7 of itself (an exponential in fp32 by
one unit, its argument by 2^-24 of x - m, at most 16 to 32 of them added in fp32, the rest in
fp64; what is far from the maximum, whose argument errs more, is as much smaller), so totals
err by that and the score's rounding to fp32, 2^-24 of it. Beams and tokens are the
oracle's wherever its neighbours lie further apart than twice that."""
import numpy as np
import pytest

from oracle import beam as obeam
from test_gpu_q4 import TYPES, sq, torch  # noqa: F401

pytestmark = pytest.mark.gpu

FAR = 4e-7


def check(step, x, scores, finished, pad, top):
    x = x.double().cpu().numpy()
    scores, batch, beams = scores.cpu().numpy(), *scores.shape
    finished = None if finished is None else finished.cpu().numpy()
    got = [t.cpu().numpy() for t in (step.score, step.parent, step.token)]
    for i in range(batch):
        more = obeam.select(x[i * beams:(i + 1) * beams], scores[i], None if finished is None else finished[i],
                            pad, top + 1)
        for r in range(top):
            total, beam, token = more[r]
            if np.isnan(total) or total == -np.inf:
                assert got[0][i, r] == total or (np.isnan(total) and np.isnan(got[0][i, r]))
                assert got[1][i, r] == got[2][i, r] == -1
                continue
            assert abs(got[0][i, r] - total) <= 2e-7 + 2.0 ** -24 * abs(total) * 1.001, (i, r)
            near = [o for o in (more[r - 1] if r else None, more[r + 1]) if o is not None
                    and o[1] != beam and abs(o[0] - total) <= FAR]
            if not near:
                assert (got[1][i, r], got[2][i, r]) == (beam, token), (i, r)


def sample(torch, seed, batch, beams, vocab, dtype, pad=0):  # noqa: F811
    g = torch.Generator().manual_seed(seed)
    x = 3 * torch.randn(batch * beams, vocab + pad, generator=g)
    x[:, torch.randint(vocab, (vocab // 50 + 1,), generator=g)] = float("-inf")
    scores = torch.randn(batch, beams, generator=g) - 10
    return x.to(getattr(torch, dtype)).cuda()[:, :vocab], scores.cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,beams,vocab,top", [(1, 1, 1, 1), (1, 1, 7, 4), (2, 4, 9, 32), (3, 5, 1000, 10),
                                                   (1, 32, 2001, 32), (17, 3, 300, 1), (2, 8, 32003, 16),
                                                   (1, 4, 131072, 8), (1, 1, 131072, 32), (40, 16, 515, 32),
                                                   (1, 31, 40000, 31), (5, 2, 16384, 32), (600, 1, 70, 2)])
def test_select(sq, torch, batch, beams, vocab, top, dtype):  # noqa: F811
    x, scores = sample(torch, batch + vocab, batch, beams, vocab, dtype, pad=5 * (vocab % 2))
    check(sq.beam_select(x, scores, top), x, scores, None, 0, top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [50, 3001, 70000])
def test_select_of_finished_dead_and_masked_beams(sq, torch, vocab, dtype):  # noqa: F811
    batch, beams, top = 8, 6, 12
    x, scores = sample(torch, vocab, batch, beams, vocab, dtype)
    x = x.contiguous()
    finished = torch.zeros(batch, beams, dtype=torch.bool)
    finished[0, 2] = finished[1, :] = finished[2, 5] = finished[4, 1] = True
    finished = finished.cuda()
    scores[2, 0] = scores[2, 5] = float("-inf")       # dead, one of them finished
    scores[3, 1:] = float("-inf")                     # the first step
    scores[5] = float("-inf")                         # nothing left of the sequence
    x[6 * beams:7 * beams] = float("-inf")            # masks that leave nothing
    x[7 * beams + 3] = float("-inf")
    x[7 * beams + 4, 1:] = float("-inf")              # one token left
    lowest = torch.finfo(x.dtype).min
    x[7 * beams + 5] = lowest                         # a mask of the type's lowest value: uniform
    scores[0, 2] = scores[0].max() + 3                # a finished beam before everything
    # what is not read may hold anything
    x[0 * beams + 2] = float("nan")
    x[2 * beams + 0] = float("inf")
    r = sq.beam_select(x, scores, top, finished=finished, pad_token=vocab + 7)
    check(r, x, scores, finished, vocab + 7, top)
    assert r.token[0, 0] == vocab + 7 and r.parent[0, 0] == 2 and r.score[0, 0] == scores[0, 2]
    assert (r.token[5] == -1).all() and (r.token[6] == -1).all()
    again = sq.beam_select(x, scores, top, finished=finished.to(torch.uint8) * 3, pad_token=vocab + 7)
    assert torch.equal(again.token, r.token) and torch.equal(again.score, r.score)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [50, 40000])
def test_select_of_what_is_no_distribution(sq, torch, vocab, dtype):  # noqa: F811
    batch, beams, top = 6, 3, 7
    x, scores = sample(torch, vocab, batch, beams, vocab, dtype)
    x = x.contiguous()
    ref = sq.beam_select(x, scores, top)
    x[1 * beams + 1, vocab - 1] = float("nan")
    x[2 * beams, 3] = float("inf")
    scores[3, 2], scores[4, 0] = float("nan"), float("inf")
    r = sq.beam_select(x, scores, top)
    for i in (1, 2, 3, 4):
        assert torch.isnan(r.score[i]).all() and (r.parent[i] == -1).all() and (r.token[i] == -1).all()
    for i in (0, 5):
        assert torch.equal(r.score[i], ref.score[i]) and torch.equal(r.token[i], ref.token[i])


@pytest.mark.parametrize("vocab", [40, 4096, 33000])
def test_ties_go_to_the_lower_beam_and_token(sq, torch, vocab):  # noqa: F811
    # rows alike and scores alike: every total is met again in every beam
    batch, beams, top = 2, 4, 32
    row = torch.randint(-3, 4, (batch, 1, vocab), generator=torch.Generator().manual_seed(2)).bfloat16()
    x = row.expand(batch, beams, vocab).reshape(batch * beams, vocab).cuda()
    scores = torch.full((batch, beams), -2.5).cuda()
    r = sq.beam_select(x, scores, top)
    for i in range(batch):
        best = torch.sort(row[i, 0].float(), descending=True, stable=True)
        want = [(b, t, v) for v in sorted(set(best.values.tolist()), reverse=True) for b in range(beams)
                for t in best.indices[best.values == v].tolist()][:top]
        assert [(int(p), int(t)) for p, t in zip(r.parent[i], r.token[i])] == [w[:2] for w in want]
    # nothing but equal logits: the first tokens of the first beam
    same = torch.zeros(batch * beams, vocab, device="cuda")
    r = sq.beam_select(same, scores, top)
    assert (r.parent == 0).all() and torch.equal(r.token.cpu(), torch.arange(32).repeat(2, 1))


def test_select_of_rows_anywhere_on_another_stream_and_in_a_graph(sq, torch):  # noqa: F811
    batch, beams, vocab, top = 3, 4, 1501, 8
    base = torch.randn(batch * beams * 1601 + 9, generator=torch.Generator().manual_seed(3)).half().cuda()
    x = base[5:5 + batch * beams * 1601].view(-1, 1601)[:, 7:7 + vocab]
    scores = torch.randn(batch, beams).cuda()
    ref = sq.beam_select(x.contiguous(), scores, top)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [sq.beam_select(x, scores, top), sq.beam_select(x.flip(1).contiguous().flip(1), scores, top),
           sq.beam_select(x, scores, top, stream=side)]
    side.synchronize()
    for r in got:
        assert torch.equal(r.score, ref.score) and torch.equal(r.token, ref.token)
    state = torch.randn(batch * beams, 33, device="cuda")

    def step():
        r = sq.beam_select(x, scores, beams)
        return r.score, r.token, sq.beam_reorder(state, r.parent)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step()
    for seed in range(3):
        base.copy_(torch.randn(base.shape, generator=torch.Generator().manual_seed(seed)))
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, step()):
            assert torch.equal(a, b)


# ---------------------------------------------------------------- reordering

@pytest.mark.parametrize("batch,beams,out_beams", [(1, 1, 1), (1, 4, 4), (3, 5, 5), (2, 1, 6), (4, 8, 3),
                                                   (1, 32, 32), (2, 16, 17)])
def test_reorder(sq, torch, batch, beams, out_beams):  # noqa: F811
    g = torch.Generator().manual_seed(batch * beams)
    rows = batch * beams
    parents = torch.randint(beams, (batch, out_beams), generator=g)
    cache = torch.randn(rows, 3, 50, 16, generator=g)
    states = [cache.cuda()[:, :, :37], cache.bfloat16().cuda()[:, 1, 3:8],
              torch.randint(100, (rows,), generator=g).cuda(), torch.randint(2, (rows, 7), generator=g).bool().cuda(),
              torch.randn(rows, 33, generator=g).half().cuda(), torch.randn(rows, 5, 3, generator=g).double().cuda(),
              torch.zeros(rows, 0).cuda(), cache.transpose(1, 2).cuda(), cache.cuda().permute(0, 3, 2, 1),
              torch.randint(99, (3, rows), generator=g).to(torch.uint8).cuda().t(),
              torch.randn(rows, 20, 300, generator=g).cuda()[:, ::2, ::3]]
    got = sq.beam_reorder(states, parents.cuda())
    for s, o in zip(states, got):
        assert o.dtype == s.dtype and o.is_contiguous()
        v = s.float() if s.dtype == torch.bfloat16 else s
        ref = obeam.reorder(v.cpu().numpy(), parents.numpy())
        assert np.array_equal((o.float() if s.dtype == torch.bfloat16 else o).cpu().numpy(), ref)
    one = sq.beam_reorder(states[0], parents.cuda())
    assert torch.equal(one, got[0])
    # into a part of a larger cache, whose other elements stay
    room = torch.full((batch * out_beams, 3, 50, 16), 7.0, device="cuda")
    sq.beam_reorder([states[0]], parents.cuda(), out=[room[:, :, :37]])
    assert torch.equal(room[:, :, :37], got[0]) and (room[:, :, 37:] == 7).all()


@pytest.mark.parametrize("batch,beams", [(1, 2), (3, 5), (2, 12), (1, 32)])
def test_reorder_in_place(sq, torch, batch, beams):  # noqa: F811
    g = torch.Generator().manual_seed(batch * beams)
    rows = batch * beams
    for kind in ("random", "shift", "swap", "same", "none"):
        j = torch.arange(beams).expand(batch, beams)
        parents = {"random": torch.randint(beams, (batch, beams), generator=g), "shift": (j + 1) % beams,
                   "swap": beams - 1 - j, "same": j, "none": torch.where(j == 0, -1, j)}[kind].contiguous()
        cache = torch.randn(rows, 3, 50, 17, generator=g).cuda()
        tokens = torch.randint(1000, (rows, 5), generator=g).cuda()
        states = [cache[:, :, :41], tokens, tokens[:, 0].clone()]
        before = cache.clone()
        ref = [obeam.reorder(s.cpu().numpy(), parents.numpy()) for s in states]
        got = sq.beam_reorder(states, parents.cuda(), out=states)
        for s, o, r in zip(states, got, ref):
            assert o is s and np.array_equal(s.cpu().numpy(), r)
        assert torch.equal(cache[:, :, 41:], before[:, :, 41:])


def test_reorder_refuses(sq, torch):  # noqa: F811
    a, b = torch.randn(4, 6).cuda(), torch.randn(4, 6).cuda()
    p = torch.tensor([[1, 0], [0, 0]]).cuda()
    wide = torch.randn(4, 12).cuda()
    before = [a.clone(), b.clone()]
    for states, out in (([a, a], [a, a]), ([a, b], [b, a]), ([a, b], [wide[:, :6], wide[:, :6]]), ([a], [a[:2]]),
                        ([a], [a.double()]), ([a], [a.cpu()]), ([a], []), ([a, b[:2]], None), ([a.cpu()], None),
                        ([a[:3]], None), ([a], [torch.empty_like(a)[:1].expand(4, 6)])):
        with pytest.raises((ValueError, sq.SeedqError)):
            sq.beam_reorder(states, p, out=out)
    with pytest.raises(ValueError):
        sq.beam_reorder(a, torch.zeros(4, 1, dtype=torch.int64).cuda(), out=a.t())
    with pytest.raises(ValueError):
        sq.beam_reorder(torch.randn(4, 6).cuda(), torch.zeros(2, 3, dtype=torch.int64).cuda(), out=a)
    with pytest.raises(ValueError):
        sq.beam_reorder(a, p.int())
    assert torch.equal(a, before[0]) and torch.equal(b, before[1])
    across = torch.zeros(6, 4).cuda().t()              # rows between each other's pieces
    sq.beam_reorder(a, p, out=across)
    assert torch.equal(across, sq.beam_reorder(a, p))


def test_reorder_of_parents_that_are_none(sq, torch):  # noqa: F811
    state = torch.randn(8, 70, device="cuda")
    parents = torch.tensor([[-1, 0, 4, 3], [1 << 40, -(1 << 62), 2, 2]]).cuda()
    got = sq.beam_reorder(state, parents)
    assert np.array_equal(got.cpu().numpy(), obeam.reorder(state.cpu().numpy(), parents.cpu().numpy()))


def test_reorder_of_complex_states(sq, torch):  # noqa: F811
    state = torch.randn(6, 5, dtype=torch.complex64, device="cuda")
    parents = torch.tensor([[2, 0, 2], [1, 1, 0]]).cuda()
    at = torch.tensor([2, 0, 2, 4, 4, 3]).cuda()
    # conjugates and their imaginary parts are marks on the same memory
    states = [state, state.conj(), state.conj().imag]
    for s, o in zip(states, sq.beam_reorder(states, parents)):
        assert torch.equal(o, s.resolve_conj()[at])
    for s in states[1:]:
        with pytest.raises(ValueError):
            sq.beam_reorder(s, parents, out=s)


def test_reorder_of_many_states_and_sequences(sq, torch):  # noqa: F811
    g = torch.Generator().manual_seed(5)
    parents = torch.randint(3, (2, 3), generator=g).cuda()
    states = [torch.randn(6, 5 + k, generator=g).cuda() for k in range(131)]
    for s, o in zip(states, sq.beam_reorder(states, parents)):
        assert np.array_equal(o.cpu().numpy(), obeam.reorder(s.cpu().numpy(), parents.cpu().numpy()))
    batch = 70000
    parents = torch.randint(2, (batch, 2), generator=g).cuda()
    state = torch.randint(1 << 40, (2 * batch, 3), generator=g).cuda()
    at = parents + 2 * torch.arange(batch, device="cuda")[:, None]
    assert torch.equal(sq.beam_reorder(state, parents), state[at.view(-1)])
    assert sq.beam_reorder(state[:0], parents[:0]).shape == (0, 3)
    assert sq.beam_reorder([], parents) == []


def test_reorder_past_32_bits(sq, torch):  # noqa: F811
    # rows of 2^31 + 40 bytes: one piece is cut, and offsets pass 32 bits
    n = (1 << 31) + 40
    state = torch.empty(3, n, dtype=torch.uint8, device="cuda")
    for r in range(3):
        state[r] = r + 1
    state[:, -3:] += 10
    parents = torch.tensor([[2, 0, 2]]).cuda()
    got = sq.beam_reorder(state, parents)
    for j, p in enumerate((2, 0, 2)):
        assert torch.equal(got[j], state[p])
    sq.beam_reorder(state, parents, out=state)
    assert torch.equal(state, got)


def test_more_sequences_than_a_launch(sq, torch):  # noqa: F811
    batch, beams, vocab, top = 65536 + 9, 2, 24, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(batch * beams, vocab, generator=g, device="cuda")
    scores = torch.randn(batch, beams, generator=g, device="cuda")
    finished = torch.rand(batch, beams, generator=g, device="cuda") < 0.2
    r = sq.beam_select(x, scores, top, finished=finished, pad_token=5)
    for lo, hi in ((0, 40), (65530, batch)):
        part = sq.BeamStep(r.score[lo:hi], r.parent[lo:hi], r.token[lo:hi])
        check(part, x[lo * beams:hi * beams], scores[lo:hi], finished[lo:hi], 5, top)


def test_many_offers_of_equal_total(sq, torch):  # noqa: F811
    # every beam offers the same: the bounds of the join cut nothing away that counts
    for beams, vocab, top in ((32, 70000, 32), (31, 40, 32), (16, 33000, 32), (5, 131072, 32), (32, 3, 17)):
        x = torch.zeros(beams, vocab, device="cuda", dtype=torch.float16)
        r = sq.beam_select(x, torch.zeros(1, beams, device="cuda"), top)
        want = [(b, v) for b in range(beams) for v in range(min(vocab, top))][:top]
        assert [(int(p), int(t)) for p, t in zip(r.parent[0], r.token[0])] == want
