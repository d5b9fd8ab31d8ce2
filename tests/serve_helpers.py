"""Plain 64-bit implementations of the calls around the decode step, and how far a right kernel may be off."""
import math

import numpy as np
import torch

from paper_1906_11024_b200 import binding as B

DH = 64


def dtype_of(name):
    return (torch.bfloat16, B.SAN_BF16) if name == "bf16" else (torch.float32, B.SAN_F32)


def randn(gen, *shape, dtype):
    """N(0, 1) rounded to `dtype`, on the host."""
    return torch.randn(*shape, generator=gen).to(dtype)


def to_planes(x):
    """Rows [..., position, 64] in order -> as the cache keeps them (16-byte chunks of a bf16 row permuted by position)."""
    if x.dtype != torch.bfloat16:
        return x.clone()
    T = x.shape[-2]
    out = torch.empty_like(x)
    y, o = x.view(*x.shape[:-1], 8, 8), out.view(*x.shape[:-1], 8, 8)
    for pos in range(T):
        for c in range(8):
            o[..., pos, c ^ (pos & 7), :] = y[..., pos, c, :]
    return out


def attend(q, k, v):
    """One query row: q [64], k [n][64], v [L][n][64] (64 bits) -> outputs [L][64] and, per output, how far an
    implementation in float32 may be off before its outputs are rounded."""
    n = k.shape[0]
    if n == 0:
        return torch.zeros(v.shape[0], DH, dtype=torch.float64), torch.zeros(v.shape[0], DH, dtype=torch.float64)
    z = k @ q / 8.0
    p = torch.softmax(z, 0)
    out = torch.einsum("n,lnd->ld", p, v)
    size = torch.einsum("n,lnd->ld", p, v.abs())
    # a score: 64 products and additions and the scale, each within 2^-24 of what it is applied to; the argument
    # of the exponential is a difference of two scores; the exponential within 2^-21 (the fast one within 2^-22
    # plus the argument's rounding, |z| log2(e) 2^-24, which the factor 66 + 4 covers); n additions of weights and outputs
    dz = 70 * 2.0 ** -24 * float((k.abs() @ q.abs()).max()) / 8.0
    return out, size * (4 * dz + 2.0 ** -20 + 2 * n * 2.0 ** -24)


def check_outputs(got, want, slack, size_bf16, dtype, where=""):
    """got (kernel) against want (64 bits).  bf16: the weights and the outputs are rounded once each, by at
    most half a step (2^-8) relative."""
    got = got.double()
    if dtype == torch.bfloat16:
        bound = slack + 2.0 ** -8 * size_bf16 + 2.0 ** -8 * (want.abs() + 2.0 ** -8 * size_bf16) * 1.01 + 1e-30
    else:
        bound = slack + 2.0 ** -23 * want.abs() + 1e-30
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), (where, int(bad.sum()), float((off / bound.clamp_min(1e-30)).max()))


def weighted_size(q, k, v):
    if k.shape[0] == 0:
        return torch.zeros(v.shape[0], DH, dtype=torch.float64)
    p = torch.softmax(k @ q / 8.0, 0)
    return torch.einsum("n,lnd->ld", p, v.abs())


def select(logits, score, length, done, tokens, eos, alpha, beam):
    """Beam selection in 64 bits, candidate by candidate; NaN logits are masked."""
    rows, V = logits.shape
    S = rows // beam
    x = logits.double().numpy().copy()
    x[np.isnan(x)] = -np.inf
    out = dict(score=np.full(rows, -np.inf), len=np.array(length), done=np.ones(rows, np.int32),
               parent=np.tile(np.arange(beam), S).astype(np.int32), next=np.full(rows, max(eos, 0), np.int32),
               tokens=[list(tokens[r][:length[r]]) for r in range(rows)])
    gap = np.inf                                # the least distance of two candidates that the choice turned on
    for s in range(S):
        found = []
        for b in range(beam):
            r = s * beam + b
            if not np.isfinite(score[r]):
                continue
            if done[r]:
                found.append((-(float(score[r]) / ((5.0 + length[r]) / 6.0) ** alpha), b, max(eos, 0), float(score[r])))
                continue
            top = x[r].max()
            if top == -np.inf:
                continue
            d = np.where(x[r] == top, 0.0, x[r] - top)
            logp = d - math.log(np.exp(d).sum())
            norm = ((5.0 + length[r] + 1) / 6.0) ** alpha
            for v in np.lexsort((np.arange(V), -x[r]))[:beam + 1]:
                if logp[v] > -np.inf:
                    found.append((-(float(score[r]) + logp[v]) / norm, b, int(v), float(score[r]) + logp[v]))
        found.sort(key=lambda f: f[:3])
        for i in range(1, min(len(found), beam + 1)):
            if found[i][1] != found[i - 1][1]:
                gap = min(gap, found[i][0] - found[i - 1][0])
        for i, (_, b, v, t) in enumerate(found[:beam]):
            r, q = s * beam + i, s * beam + b
            out["score"][r], out["parent"][r], out["next"][r] = t, b, v
            out["len"][r] = length[q] + (0 if done[q] else 1)
            out["done"][r] = int(bool(done[q]) or v == eos)
            out["tokens"][r] = list(tokens[q][:length[q]]) + ([] if done[q] else [v])
    out["gap"] = gap
    return out
