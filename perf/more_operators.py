"""Operators on weights held as microscaled 4-bit floats, and on the beams that a head's logits extend.

``listed()`` names the calls that a user makes of them, ``draw(rng)`` gives more of the same ranges,
``prepare`` makes what a program has in hand, ``run`` is one pass: the plain form in torch operations
where ``own`` is false, the library's entry points where it is true. ``exact`` is the definition in
64 bits.

* round: a weight matrix to codes and back (what a comparison of codecs does per tensor).
* gemv: products of the coded matrix with one vector, a batch, or a prompt in 16 or 32 bits.
* matmul: products of coded rows with a coded matrix.
* select: the best continuations of every sequence over its beams and the vocabulary.
* reorder: states of beams, caches among them, moved to the beams that continue them.

Codes are 32-bit words of eight 4-bit floats (sign, two exponent bits, one mantissa bit: 0, 0.5, 1,
1.5, 2, 3, 4, 6), lowest bits first, each row padded to 16 bytes; a byte e a row and block of 32
columns scales them by 2^(e - 127).
"""
import math
from types import SimpleNamespace

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 32


def listed():
    return [
        # A key or value projection of 8 shared heads, coded and decoded: the small tensor.
        dict(name="round_kv", kind="round", rows=1024, cols=4096, type="f32"),
        # An MLP up-projection kept in 16 bits.
        dict(name="round_mlp", kind="round", rows=4096, cols=14336, type="bf16"),
        # One token against an attention projection: launch and latency bound.
        dict(name="gemv_token", kind="gemv", rows=4096, cols=4096, nvec=1, type="bf16", out="bf16"),
        # Three vectors in 32 bits against an odd shape whose last block is short.
        dict(name="gemv_ragged", kind="gemv", rows=1001, cols=2056, nvec=3, type="f32", out="f32"),
        # Eight sequences' tokens against the largest layer: bound by the reading of the codes.
        dict(name="gemv_batch", kind="gemv", rows=8192, cols=28672, nvec=8, type="f16", out="f16"),
        # The logits of a prompt: a coded head of 32000 tokens, bound by the matrix core.
        dict(name="gemv_prompt", kind="gemv", rows=32000, cols=4096, nvec=512, type="bf16", out="f32"),
        # Four coded tokens against a coded projection.
        dict(name="matmul_tokens", kind="matmul", rows=4096, cols=4096, nvec=4, out="bf16"),
        # The logits of a long prompt from coded hidden states and the coded head.
        dict(name="matmul_prompt", kind="matmul", rows=32000, cols=4096, nvec=2048, out="bf16"),
        # One sequence's four beams, one of them finished, an odd vocabulary inside a padded one.
        dict(name="select_step", kind="select", batch=1, beams=4, vocab=32003, pad=61, type="f32", top=8),
        # Sixty-four sequences of eight beams over a wide vocabulary.
        dict(name="select_batch", kind="select", batch=64, beams=8, vocab=131072, pad=0, type="bf16",
             top=16),
        # The tokens, lengths and small odd states of one sequence's five beams.
        dict(name="reorder_tokens", kind="reorder", batch=1, beams=5, layers=1, heads=3, room=77,
             used=67, dim=33, type="f32"),
        # The keys and values of 16 layers, of which the used part moves.
        dict(name="reorder_cache", kind="reorder", batch=4, beams=4, layers=16, heads=8, room=2048,
             used=1500, dim=128, type="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("round", "gemv", "gemv", "gemv", "matmul", "matmul", "select", "select",
                       "reorder"))
    if kind == "select":
        beams = rng.choice((1, 2, 3, 4, 5, 8, 12, 16))
        vocab = _log(rng, 500, 131072)
        batch = _log(rng, 1, max(1, min(64, 2 ** 25 // (vocab * beams))))
        return dict(kind=kind, batch=batch, beams=beams, vocab=vocab, pad=rng.choice((0, 0, 1, 8, 37)),
                    type=rng.choice(("f32", "f16", "bf16", "bf16")), top=rng.choice((beams, 2 * beams)))
    if kind == "reorder":
        case = dict(kind=kind, batch=_log(rng, 1, 16), beams=rng.choice((1, 2, 3, 4, 5, 8, 12, 16)),
                    layers=_log(rng, 1, 16), heads=_log(rng, 1, 8), dim=rng.choice((33, 64, 80, 128)),
                    type=rng.choice(("f32", "f16", "bf16", "bf16")))
        row = 2 * case["layers"] * case["batch"] * case["beams"] * case["heads"] * case["dim"]
        case["room"] = _log(rng, 16, max(17, min(4096, 2 ** 28 // row)))
        case["used"] = rng.randint(1, case["room"])
        return case
    case = dict(kind=kind, rows=_log(rng, 64, 32000), cols=8 * _log(rng, 16, 3584))
    case["cols"] = min(case["cols"], 8 * ((4 if kind == "gemv" else 2) * 10 ** 6 // case["rows"]))
    case["type"] = rng.choice(("f32", "f16", "bf16", "bf16"))
    if kind == "gemv":
        case["nvec"] = rng.choice((1, 1, 1, _log(rng, 2, 16), _log(rng, 2, 16), _log(rng, 16, 512)))
        case["out"] = rng.choice((case["type"], case["type"], "f32"))
    if kind == "matmul":
        case["nvec"] = rng.choice((_log(rng, 1, 16), _log(rng, 16, 2048), _log(rng, 16, 2048)))
        case["out"] = case.pop("type")
    return case


# ---------------------------------------------------------------- inputs

def _weights(rows, cols, g):
    """N(0, 0.02^2) with one heavy-tailed weight at a random place of every 1000."""
    w = torch.randn(rows, cols, device="cuda", generator=g).mul_(0.02)
    m = max(1, rows * cols // 1000)
    at = torch.arange(m, device="cuda") * 1000 + torch.randint(1000, (m,), device="cuda", generator=g)
    z = torch.randn(4, m, device="cuda", generator=g)
    w.view(-1)[at.clamp_(max=rows * cols - 1)] = 0.1 * z[0] / (z[1:].square().sum(0) / 3).sqrt()
    return w


def _hidden(rows, cols, g):
    """Rows of a normed hidden state, some channels larger."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    return x * torch.randn(cols, device="cuda", generator=g).mul_(0.3).exp_()


def _pack(u):
    """Codes 0..15 [rows, cols] to words [rows, row_words]."""
    rows, cols = u.shape
    u = torch.nn.functional.pad(u, (0, -cols % BLOCK)).view(rows, -1, 8)
    w = torch.zeros(u.shape[:2], dtype=torch.int32, device=u.device)
    for i in range(8):
        w |= u[:, :, i].to(torch.int32) << (4 * i)
    return w


def _prepare_select(s, case, g, seed):
    rows, vocab = case["batch"] * case["beams"], case["vocab"]
    x = torch.randn(rows, vocab + case["pad"], device="cuda", generator=g).mul_(3.0)
    likely = torch.randint(vocab, (rows, 4), device="cuda", generator=g)
    x.scatter_add_(1, likely, 6.0 + 3.0 * torch.randn(rows, 4, device="cuda", generator=g))
    barred = torch.randint(vocab, (max(1, vocab // 100),), device="cuda", generator=g)
    x[:, barred] = float("-inf")                                       # tokens that are never allowed
    if rows >= 16:
        x[seed % rows] = float("-inf")                                 # a beam whose mask leaves nothing
    s.logits = x.to(TYPES[case["type"]])[:, :vocab]
    s.scores = torch.randn(case["batch"], case["beams"], device="cuda", generator=g).mul_(1.5).sub_(20.0)
    s.finished = torch.rand(case["batch"], case["beams"], device="cuda", generator=g) < 1 / 8
    s.finished[0, case["beams"] // 2] = case["beams"] > 1
    if case["batch"] > 3:
        s.scores[1, 1:] = float("-inf")                                # a sequence at its first step
    s.pad_token = 2


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = SimpleNamespace(case=case, kind=case["kind"])
    if s.kind == "round":
        s.W = _weights(case["rows"], case["cols"], g).to(TYPES[case["type"]])
    elif s.kind in ("gemv", "matmul"):
        u, s.scale = _quantize(_weights(case["rows"], case["cols"], g))
        s.codes = _pack(u)
        x = _hidden(case["nvec"], case["cols"], g)
        if s.kind == "gemv":
            s.x = x.to(TYPES[case["type"]])
        else:
            u, s.xscale = _quantize(x)
            s.xcodes = _pack(u)
    elif s.kind == "select":
        _prepare_select(s, case, g, seed)
    else:   # caches with room for more tokens than are used, the tokens and lengths themselves
        rows = case["batch"] * case["beams"]
        caches = [torch.randn(rows, case["heads"], case["room"], case["dim"], device="cuda", generator=g,
                              dtype=TYPES[case["type"]]) for _ in range(2 * case["layers"])]
        s.states = [c[:, :, :case["used"]] for c in caches]
        s.states.append(torch.randint(32000, (rows, case["room"]), device="cuda", generator=g))
        s.states.append(torch.randint(case["room"], (rows,), device="cuda", generator=g))
        s.parents = torch.randint(case["beams"], (case["batch"], case["beams"]), device="cuda",
                                  generator=g)
    return s


# ---------------------------------------------------------------- the plain forms

def _blocks(w):
    """[rows, nblocks, 32] with zeros after the last column."""
    rows, cols = w.shape
    return torch.nn.functional.pad(w, (0, -cols % BLOCK)).view(rows, -1, BLOCK)


def _power(k):
    """2^k of whole numbers in 32 bits, -127 among them."""
    return torch.where(k < -126, torch.full_like(k, 1 << 22), (k + 127) << 23).view(torch.float32)


def _quantize(w):
    """Codes 0..15 and the biased exponents of the scales, uint8. The largest magnitude of a block
    lies in the last binade of the codes, 4 to 8; what is above 6 is 6."""
    cols = w.shape[1]
    b = _blocks(w.float())
    e = ((b.abs().amax(2).view(torch.int32) >> 23) - 2).clamp(min=0)
    half = (127 - e) // 2   # in two steps: 2^127 and more are no factors
    t = b * _power(half)[..., None] * _power(127 - e - half)[..., None]
    a = t.abs()
    a = torch.where(a < 2, torch.round(2 * a) / 2,
                    torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2))).clamp(max=6)
    u = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    u |= (b.view(torch.int32) < 0).to(torch.uint8) << 3
    return u.view(len(w), -1)[:, :cols], e.to(torch.uint8)


def _values(words, scale, cols):
    """The weights in 32 bits."""
    u = ((words[..., None] >> (4 * torch.arange(8, device=words.device, dtype=torch.int32))) & 15)
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6],
                         device=words.device)
    w = table[u.view(len(words), -1, BLOCK)]
    return (w * _power(scale.to(torch.int32) - 127)[..., None]).view(len(words), -1)[:, :cols]


def _order_keys(x):
    """64-bit keys in the order of (value, lower index first); all different."""
    b = (x.float() + 0.0).view(torch.int32)
    b = b ^ ((b >> 31) & 0x7FFFFFFF)
    n = x.shape[1]
    return (b.to(torch.int64) << 32) + (n - 1 - torch.arange(n, device=x.device))


def _select(s):
    """Totals in 64 bits, since those of different beams may lie next to each other."""
    case = s.case
    batch, beams, top, vocab = case["batch"], case["beams"], case["top"], case["vocab"]
    each = min(top, vocab)
    none = float("-inf")
    token = torch.topk(_order_keys(s.logits), each, dim=1).indices
    x = s.logits.double()
    m = x.amax(1, keepdim=True)
    lse = m + torch.where(m == none, torch.full_like(x, none), x - m).exp().sum(1, keepdim=True).log()
    logp = x.gather(1, token) - lse
    logp = torch.where(m == none, torch.full_like(logp, none), logp).view(batch, beams, each)
    token = token.view(batch, beams, each)
    first = torch.arange(each, device=x.device) == 0
    done = s.finished[..., None]
    logp = torch.where(done, torch.where(first, 0.0, none).double(), logp)
    token = torch.where(done, torch.full_like(token, s.pad_token), token)
    total = (s.scores.double()[..., None] + logp).view(batch, -1)
    total, at = torch.sort(total, dim=1, descending=True, stable=True)
    total, at = total[:, :top], at[:, :top]
    gone = total == none
    if total.shape[1] < top:
        raise ValueError("fewer tokens than continuations")
    parent = torch.where(gone, torch.full_like(at, -1), at // each)
    token = torch.where(gone, torch.full_like(at, -1), token.view(batch, -1).gather(1, at))
    return {"score": total.float(), "parent": parent, "token": token}


def _plain(s):
    case, kind = s.case, s.kind
    if kind == "select":
        return _select(s)
    if kind == "reorder":
        batch, beams = s.parents.shape
        at = (s.parents + beams * torch.arange(batch, device=s.parents.device)[:, None]).view(-1)
        return [t[at] for t in s.states]
    cols = case["cols"]
    if kind == "round":
        u, scale = _quantize(s.W)
        return {"W": _values(_pack(u), scale, cols).to(s.W.dtype), "exponent": scale}
    x = s.x.float() if kind == "gemv" else _values(s.xcodes, s.xscale, cols)
    return (x @ _values(s.codes, s.scale, cols).t()).to(TYPES[case["out"]])


def run(s):
    if not own:
        return _plain(s)
    import paper_2609_38477_amd as sq
    case, kind = s.case, s.kind
    if kind == "round":
        q = sq.mx4_quantize(s.W)
        return {"W": sq.mx4_dequantize(q, s.W.dtype), "exponent": q.scale}
    if kind == "select":
        r = sq.beam_select(s.logits, s.scores, case["top"], finished=s.finished, pad_token=s.pad_token)
        return {"score": r.score, "parent": r.parent, "token": r.token}
    if kind == "reorder":
        return sq.beam_reorder(s.states, s.parents)
    q = sq.Mx4Weights(s.codes, s.scale, case["rows"], case["cols"])
    if kind == "gemv":
        return sq.mx4_gemv(q, s.x, TYPES[case["out"]])
    return sq.mx4_matmul(sq.Mx4Weights(s.xcodes, s.xscale, case["nvec"], case["cols"]), q,
                         TYPES[case["out"]])


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    kind = case["kind"]
    size = 4 if case.get("type") == "f32" else 2
    if kind == "select":   # a difference, an exponential and a sum for each logit
        rows = case["batch"] * case["beams"]
        n = rows * case["vocab"]
        return {"bytes": size * n + 5 * rows + 20 * case["batch"] * case["top"], "flops": 4.0 * n}
    if kind == "reorder":   # every beam has a continuation at the most; the least is written once
        rows = case["batch"] * case["beams"]
        moved = 2 * case["layers"] * case["heads"] * case["used"] * case["dim"] * size \
            + 8 * case["room"] + 8
        kept = case["batch"] * case["beams"] * (1 - (1 - 1 / case["beams"]) ** case["beams"])
        return {"bytes": (rows + kept) * moved + 8 * rows, "flops": 0}
    rows, cols = case["rows"], case["cols"]
    coded = rows * cols / 2 + rows * -(-cols // BLOCK)
    if kind == "round":
        return {"bytes": 2 * size * rows * cols + coded, "flops": 4.0 * rows * cols}
    nvec = case["nvec"]
    osize = 4 if case["out"] == "f32" else 2
    x = size * nvec * cols if kind == "gemv" else nvec * cols / 2 + nvec * -(-cols // BLOCK)
    return {"bytes": coded + x + osize * nvec * rows, "flops": 2.0 * rows * cols * nvec}


# ---------------------------------------------------------------- 64-bit results

def _exact_power(k):
    """2^k of whole numbers in 64 bits."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _exact_values(codes, scale, cols):
    """Weights in 64 bits, from sign, exponent and mantissa, one nibble position at a time."""
    W = torch.empty(*codes.shape, 8, dtype=torch.float64, device="cuda")
    for i in range(8):
        u = torch.bitwise_and(torch.bitwise_right_shift(codes, 4 * i), 15)
        ex, man = torch.bitwise_and(u, 7) // 2, (u % 2).double()
        mag = torch.where(ex == 0, man / 2, (1 + man / 2) * _exact_power(ex - 1))
        W[:, :, i] = torch.where(u >= 8, -mag, mag)
    W = W.reshape(codes.shape[0], -1)[:, :cols]
    of = torch.div(torch.arange(cols, device="cuda"), BLOCK, rounding_mode="floor")
    return W.mul_(_exact_power(scale.int() - 127)[:, of])


def _exact_round(W):
    """Column block by column block: the nearest of the eight magnitudes, the even code of two."""
    rows, cols = W.shape
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device="cuda")   # even codes win ties
    out = torch.empty(rows, cols, dtype=torch.float64, device="cuda")
    exps = []
    for c in range(0, cols, BLOCK):
        w = W[:, c:c + BLOCK].double()
        big = w.abs().max(1).values
        e = torch.where(big > 0, torch.frexp(big).exponent - 3, -127).clamp(min=-127)
        s = _exact_power(e)[:, None]
        t = w / s
        d = (t.abs()[..., None] - grid[order]).abs()
        mag = grid[order[d.argmin(2)]]
        out[:, c:c + BLOCK] = torch.copysign(mag, t) * s
        exps.append((e + 127).to(torch.uint8))
    return {"W": out, "exponent": torch.stack(exps, 1)}


def _exact_select(s):
    """Every total of a sequence, those that reach the last selected one in order."""
    case = s.case
    beams, top, vocab = case["beams"], case["top"], case["vocab"]
    out = {"score": [], "parent": [], "token": []}
    for b in range(case["batch"]):
        x = s.logits[b * beams:(b + 1) * beams].double()
        total = torch.log_softmax(x, 1) + s.scores[b].double()[:, None]
        total = torch.nan_to_num(total, nan=float("-inf"), neginf=float("-inf"))
        for i in torch.nonzero(s.finished[b]).flatten().tolist():
            total[i] = float("-inf")
            total[i, s.pad_token] = s.scores[b, i].double()
        flat = total.flatten()
        last = torch.kthvalue(-flat, top).values
        at = torch.nonzero(flat >= -last).flatten()
        v, i = torch.sort(-flat[at], stable=True)
        v, at = -v[:top], at[i[:top]]
        none = torch.isinf(v)
        out["score"].append(v)
        out["parent"].append((at // vocab).masked_fill(none, -1))
        out["token"].append((at % vocab).masked_fill(none, -1))
    return {k: torch.stack(v) for k, v in out.items()}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "select":
        return _exact_select(s)
    if kind == "reorder":
        out = []
        for t in s.states:
            rows = t.reshape(case["batch"], case["beams"], *t.shape[1:])
            out.append(torch.cat([rows[b].index_select(0, s.parents[b]) for b in range(case["batch"])]))
        return out
    if kind == "round":
        return _exact_round(s.W)
    cols = case["cols"]
    x = s.x.double() if kind == "gemv" else _exact_values(s.xcodes, s.xscale, cols)
    return torch.matmul(x, _exact_values(s.codes, s.scale, cols).t())
