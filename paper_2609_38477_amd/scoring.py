"""What a coded language-model head answers: perplexity, entropy and the likeliest
tokens of the head in 4 bits with group scales and of the seed-coded head, next to
the head they were made from; the measured counterpart of the data-free gradient
size; and single-bit faults of the 4-bit form.

* ``score`` takes logits and the tokens that came next: mean negative log
  likelihood, perplexity and entropy, and the likeliest tokens. Rows with a negative
  token (padding, a prompt) are in no mean.
* The head in 4 bits gives its logits straight from the codes (``q4_gemv``), the
  seed-coded head from its decoded weights.
* ``measured_rho`` is the gradient size at the head's input that the data itself
  gives, rho_j = sum_r W_rj^2 E[g_r^2] with g the gradient of the negative log
  likelihood at the logits; the importance front end takes E[g_r^2] = 1.
* ``fault_study`` flips single bits of a code, a scale and a zero point: the
  footprint of eq. (security_metrics) and the log likelihood after it. A code's bit
  changes one weight, a scale's or zero point's a whole group.

    python -m paper_2609_38477_amd.scoring [--vocab 8192 --d 1024 --tokens 256]

prints one JSON line.
"""
from __future__ import annotations

import argparse
import json
import math
import sys

import numpy as np

from . import (Q4Weights, footprint, q4_dequantize, q4_gemv, q4_quantize, token_logprobs,
               token_logprobs_backward)


def score(logits, tokens, top: int = 5) -> dict:
    """Figures of logits [n, vocab] against the tokens [n] that came next, means over the
    rows whose token is not negative (NaN if there is none)."""
    s = token_logprobs(logits, tokens, top=top)
    asked = tokens >= 0
    nll = -s.logprob[asked].double().mean().item()
    return {"nll": nll, "perplexity": math.inf if nll >= 700 else math.exp(nll),   # NaN stays NaN
            "entropy": s.entropy[asked].double().mean().item(), "top": s.top_token}


def measured_rho(W, logits, tokens):
    """rho (fp64 [d]) of the head W (fp32 [vocab, d]) on these logits and tokens, the mean
    over the rows whose token is not negative (NaN if there is none)."""
    import torch
    from .frontend import sq_gemv
    s = token_logprobs(logits, tokens)
    minus = torch.full_like(s.lse, -1.0)
    g = token_logprobs_backward(logits, tokens, s.lse, grad_logprob=minus)   # 0 in the other rows
    return sq_gemv(W, (g.float() ** 2).sum(0) / (tokens >= 0).sum(), transpose=True)


def next_token(q: Q4Weights, h, top: int = 5):
    """The likeliest tokens after one hidden state h [d] and their log probabilities:
    one product with one vector and one row of logits."""
    s = token_logprobs(q4_gemv(q, h, _fp32()).unsqueeze(0), top=top)
    return s.top_token[0], s.top_logprob[0]


def _fp32():
    import torch
    return torch.float32


def bits_per_weight(q: Q4Weights) -> float:
    """Stored bits a weight, scales and zero points included."""
    parts = [q.codes, q.scale] + ([] if q.zero is None else [q.zero])
    return 8.0 * sum(t.numel() * t.element_size() for t in parts) / (q.nrows * q.ncols)


def flip_bit(q: Q4Weights, part: str, index: int, bit: int) -> Q4Weights:
    """q with one bit of an element of ``part`` (codes, scale or zero) flipped."""
    import torch
    t = getattr(q, part).clone()
    n = t.element_size()
    bytes_ = t.view(-1).view(torch.uint8)
    bytes_[index * n + bit // 8] ^= 1 << (bit % 8)
    return Q4Weights(**{**q.__dict__, part: t})


def fault_study(q: Q4Weights, h, tokens) -> list:
    """Footprint and negative log likelihood of one fault of every kind, in the row of the
    first token that is one."""
    some = tokens[(tokens >= 0) & (tokens < q.nrows)]
    if some.numel() == 0:
        raise ValueError("tokens: none of them is one of the head's")
    clean = q4_dequantize(q)
    row = int(some[0].item())
    words, groups = q.codes.shape[1], q.scale.shape[1]
    kinds = [("lowest bit of a code", "codes", row * words, 0),
             ("highest bit of a code", "codes", row * words, 3),
             ("lowest bit of a scale", "scale", row * groups, 0),
             ("highest exponent bit of a scale", "scale", row * groups, 14)]
    if q.zero is not None:
        kinds.append(("bit 3 of a zero point", "zero", row * groups, 3))
    rows = []
    for name, part, index, bit in kinds:
        bad = flip_bit(q, part, index, bit)
        n, p, eta = footprint(clean, q4_dequantize(bad))
        nll = score(q4_gemv(bad, h, _fp32()), tokens, 0)["nll"]
        rows.append({"fault": name, "N_flip": n, "p_flip": p, "eta": eta, "nll": nll})
    return rows


def study(W, h, tokens, group: int = 128, zeros: bool = False, target_bpw: float = 4.0) -> dict:
    """The head W (fp32 [vocab, d]) and its two coded forms on the hidden states h
    (fp32 [n, d]) and the tokens that came next."""
    from .faults import Encoded
    base = h @ W.t()
    q = q4_quantize(W, group, zeros=zeros)
    enc = Encoded(W, ((12, 2), (16, 3), (20, 4)), (4.0, 1.0, 0.25), target_bpw,
                  np.ones(W.shape[1], dtype=np.float32))
    W_seed = enc.decode()
    forms = {"original": (32.0, W, base), "q4": (bits_per_weight(q), q4_dequantize(q), q4_gemv(q, h)),
             "seed": (32.0 * enc.words.numel() / W.numel(), W_seed, h @ W_seed.t())}
    out, first = {}, None
    for name, (bits, W_hat, logits) in forms.items():
        s = score(logits, tokens)
        top = s.pop("top")
        first = top[:, 0] if first is None else first
        err = ((W_hat - W).double() ** 2).sum() / (W.double() ** 2).sum()
        out[name] = {"bits_per_weight": bits, "relative_sq_error": err.item(), **s,
                     "same_first_token": (top[:, 0] == first).double().mean().item()}
    rho = {name: measured_rho(W, logits, tokens) for name, (_, _, logits) in forms.items()}
    free = (W.double() ** 2).sum(0).cpu().numpy()
    token, logprob = next_token(q, h[0])
    return {"heads": out,
            "rho_measured": {"correlation_with_data_free": float(np.corrcoef(rho["original"], free)[0, 1]),
                             "q4_relative_difference": _relative(rho["q4"], rho["original"]),
                             "seed_relative_difference": _relative(rho["seed"], rho["original"])},
            "next_token": {"tokens": token.tolist(), "logprobs": logprob.tolist()},
            "q4_faults": fault_study(q, h, tokens)}


def _relative(a, b) -> float:
    return float(np.linalg.norm(a - b) / np.linalg.norm(b))


def sample(vocab: int, d: int, n: int, key: int = 9):
    """A synthetic head, hidden states, and tokens drawn from the head's own softmax."""
    import torch
    import synthetic
    W = torch.from_numpy(synthetic.weights(vocab, d, 0.02, key * 16 + 7, 0.001)).cuda()
    h = torch.from_numpy(synthetic.normal(key, 41, n * d).reshape(n, d).astype(np.float32)).cuda()
    h *= 4.0 / (h * h).mean(1, keepdim=True).sqrt()
    u = torch.from_numpy(synthetic.uniform(key, 42, n).astype(np.float32)).cuda()
    cdf = torch.softmax((h @ W.t()).double(), 1).cumsum(1)
    tokens = torch.searchsorted(cdf, u.double().unsqueeze(1)).squeeze(1).clamp_(max=vocab - 1)
    return W, h, tokens


def main(argv=None) -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--vocab", type=int, default=8192)
    ap.add_argument("--d", type=int, default=1024)
    ap.add_argument("--tokens", type=int, default=256)
    ap.add_argument("--group", type=int, default=128)
    ap.add_argument("--zeros", action="store_true", help="zero points too")
    ap.add_argument("--target-bpw", type=float, default=4.0, help="of the seed-coded head")
    args = ap.parse_args(argv)
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    if root not in sys.path:
        sys.path.insert(0, root)
    W, h, tokens = sample(args.vocab, args.d, args.tokens)
    res = study(W, h, tokens, args.group, args.zeros, args.target_bpw)
    print(json.dumps({"head": [args.vocab, args.d], "tokens": args.tokens, "group": args.group,
                      "zeros": args.zeros, **res}), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
