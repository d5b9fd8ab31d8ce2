"""Plain 64-bit implementations of the calls for long prompts and caches that are kept small, and how far a right kernel may be off."""
import math

import numpy as np
import torch

DH = 64
U32, UBF = 2.0 ** -24, 2.0 ** -8            # half a step, relative
TRUNC = 2.0 ** -23                          # a step of a tensor-core sum may be cut off instead of rounded


def rounding(dtype):
    return UBF if dtype == torch.bfloat16 else U32


# ------------------------------------------------------------------------------------------- packed prompts
def packed(q, k, v, dtype):
    """One sequence: q [t][H][64], k [t][Hk][64], v [L][t][Hk][64] -> outputs [L][t][H][64] in 64 bits and how far each may be off."""
    t, H = q.shape[:2]
    r = H // k.shape[1]
    dev = q.device
    want = torch.zeros(v.shape[0], t, H, DH, dtype=torch.float64, device=dev)
    bound = torch.zeros_like(want)
    hide = torch.ones(t, t, dtype=torch.bool, device=dev).triu_(1)
    n = torch.arange(1, t + 1, dtype=torch.float64, device=dev)[:, None]
    for h in range(H):
        qh, kh, vh = q[:, h].double(), k[:, h // r].double(), v[:, :, h // r].double()
        z = (qh @ kh.T / 8.0).masked_fill_(hide, -math.inf)
        p = torch.softmax(z, -1)
        want[:, :, h] = p @ vh
        size = p @ vh.abs()
        # a score: 64 exact products whose sums are cut off or rounded some 64 times at most, and the scale; the exponential's argument is a
        # difference of two of them; the fast exponential 2^-22 + |z| log2(e) 2^-24 (in the factor); sums of n weights, twice
        dz = 70 * TRUNC * (qh.abs() @ kh.abs().T / 8.0).masked_fill_(hide, 0.0).amax(-1, keepdim=True)
        off = size * (4 * dz + 2.0 ** -20 + 2 * n * TRUNC)
        bound[:, :, h] = off + UBF * size + UBF * (want[:, :, h].abs() + UBF * size) * 1.01 + 1e-30      # weights and outputs in bf16
    assert dtype == torch.bfloat16
    return want, bound


# ------------------------------------------------------------------------------------------- four bits
def _bf16(x, up):
    """float64 number -> the bf16 number next to it, not below (up) or not above it; inf where there is none."""
    if x == 0 or not np.isfinite(x):
        return float(x)
    m, e = math.frexp(abs(x))                               # abs(x) = m 2^e, m in [0.5, 1)
    e = max(e, -125)
    unit = math.ldexp(1.0, e - 8)                           # distance of bf16 numbers there
    away = up == (x > 0)
    k = abs(x) / unit                                       # exact: a power of two
    k = math.ceil(k) if away else math.floor(k)
    y = k * unit
    y = math.inf if y >= 2.0 ** 128 else y
    return math.copysign(y, x)


def quantise_row(x):
    """64 numbers -> (codes list, step, low); step = low = NaN for a row that cannot be held."""
    x = [float(v) for v in x]
    if not all(abs(v) < 2.0 ** 40 for v in x):
        return [0] * DH, math.nan, math.nan
    low = _bf16(min(x), False)
    step = _bf16((max(x) - low) / 15.0, True)
    step = max(step, 2.0 ** -50) if step > 0 else step
    codes = []
    for v in x:
        t = (v - low) / step if step > 0 else 0.0
        codes.append(int(min(max(round(t), 0), 15)))        # round(): half to even
    return codes, step, low


def pack(codes):
    return [codes[2 * i] | codes[2 * i + 1] << 4 for i in range(DH // 2)]


def numbers(codes, scales):
    """Bytes [..., 32] and (step, low) [..., 2] -> what they stand for, 64 bits."""
    x = torch.stack([codes % 16, codes // 16], -1).reshape(*codes.shape[:-1], DH).double()
    return scales[..., 1:].double() + scales[..., :1].double() * x


def quant_attend(q, codes, scales, dtype):
    """One item: q [H][64], codes [1 + L][Hk][t][32], scales [1 + L][Hk][t][2] -> outputs [L][H][64], weights [H][t] and their bounds."""
    H, Hk, t = q.shape[0], codes.shape[1], codes.shape[2]
    L, r = codes.shape[0] - 1, H // codes.shape[1]
    if t == 0:
        z = torch.zeros(L, H, DH, dtype=torch.float64, device=q.device)
        return z, z + 1e-30, z[0, :, :0], z[0, :, :0]
    x = numbers(codes, scales).repeat_interleave(r, 1)                          # [1 + L][H][t][64]
    step = scales[..., 0].double().repeat_interleave(r, 1)
    mid = scales[..., 1].double().repeat_interleave(r, 1) + 8 * step
    whole = (x - mid[..., None]).abs()                                          # step |n'|
    qd = q.double()
    z = (x[0] @ qd[:, :, None])[..., 0] / 8.0
    p = torch.softmax(z, -1)
    out = (p[None, :, None] @ x[1:])[:, :, 0]
    # a score: sums of 64 products (float32 queries: of three parts each), cut off or rounded some 80 times at most, of the size of its two halves
    qa = qd.abs()
    dz = 80 * TRUNC * ((whole[0] @ qa[:, :, None])[..., 0] + mid[0].abs() * qa.sum(-1, keepdim=True)).amax(-1) / 8.0      # [H]
    rel = 4 * dz + 2.0 ** -20 + 2 * t * TRUNC
    size = (p[None, :, None] @ (whole[1:] + mid[1:].abs()[..., None]))[:, :, 0]
    bound = size * rel[None, :, None] + rounding(dtype) * out.abs() * 1.01 + 1e-30
    if dtype == torch.bfloat16:
        bound = bound + UBF * (p[None, :, None] @ whole[1:])[:, :, 0] * 1.01                                # weights times step in bf16
    return out, bound, p, p * rel[:, None] + 1e-37


# ------------------------------------------------------------------------------------------- mass and eviction
def keep(mass, length, n_keep, n_sink, n_recent):
    """Rows that stay, ascending."""
    if length <= n_keep:
        return list(range(length))
    m = [-math.inf if math.isnan(v) else v for v in mass]
    free = sorted(range(n_sink, length - n_recent), key=lambda j: (-m[j], j))[:n_keep - n_sink - n_recent]
    return list(range(n_sink)) + sorted(free) + list(range(length - n_recent, length))
