"""Measured cases of the calls for long prompts and a cache that is kept small.

  packed   san_packed_block: causal attention of whole prompts laid end to end, without padding, query heads in groups
  store    san_quant_append, san_quant_read: rows into a cache of four bits a number, and back as numbers
  attn     san_quant_attn: one decode step of attention over such a cache, with the weights where they are wanted
  mass     san_weight_mass: what the cached rows have received of the weights so far
  evict    san_cache_evict: the rows that received most, the first and the last ones stay, in every layer of a block

``own`` is false: ``run`` computes them from elementary torch operations.  ``own`` is true: it calls the
library.  ``exact`` is the definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
DH = 64


# ------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the latency of one short question in front of a decoder
        dict(name="packed one question", op="packed", n=1, len_lo=37, len_hi=37, log=False, heads=8, kv_heads=8, layers=1, fused=False),
        # what a server has waiting: prompts of one token to some thousand, from one fused projection
        dict(name="packed mixed", op="packed", n=48, len_lo=1, len_hi=4096, log=True, heads=16, kv_heads=4, layers=1, fused=True),
        # long documents, a block of two layers
        dict(name="packed long", op="packed", n=2, len_lo=7777, len_hi=8192, log=False, heads=8, kv_heads=8, layers=2, fused=False),
        # the rows of one decode step of a batch, a block of four layers
        dict(name="store step", op="store", dtype="bf16", n=128, rows=1, kv_heads=8, layers=4, cap=600),
        # the rows of prompts, at once
        dict(name="store prompts", op="store", dtype="f32", n=5, rows=4001, kv_heads=8, layers=2, cap=4096),
        # one request far into a long document, query heads in groups of four
        dict(name="attn one row", op="attn", dtype="bf16", n=1, len_lo=32001, len_hi=32001, heads=16, kv_heads=4, layers=1, weights=False),
        # a batch at mixed lengths, a block of four layers
        dict(name="attn batch", op="attn", dtype="bf16", n=128, len_lo=1, len_hi=4096, heads=8, kv_heads=8, layers=4, weights=False),
        # float32 decoding, with the weights for the mass of the rows
        dict(name="attn f32 weights", op="attn", dtype="f32", n=33, len_lo=1, len_hi=1500, heads=12, kv_heads=4, layers=2, weights=True),
        # the weights of one step of a batch, heads in groups of two
        dict(name="mass step", op="mass", n=128, rows=1, len_lo=1, len_hi=4096, heads=16, kv_heads=8, decay=0.99),
        # the weights of whole prompts, as their full attention gives them
        dict(name="mass prompts", op="mass", n=16, rows=512, len_lo=300, len_hi=512, heads=8, kv_heads=8, decay=1.0),
        # one request's cache in four bits is cut to half
        dict(name="evict one", op="evict", dtype="q4", n=1, len_lo=4096, len_hi=4096, keep=2048, sink=4, recent=256, kv_heads=8, layers=1),
        # the caches of a batch that have grown over their bound, a block of four layers
        dict(name="evict batch", op="evict", dtype="bf16", n=48, len_lo=900, len_hi=2304, keep=1023, sink=4, recent=128, kv_heads=8, layers=4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["packed", "store", "attn", "mass", "evict"])
    heads = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
    kv_heads = rng.choice([k for k in (1, 2, 3, 4, 8, 16) if heads % k == 0] + [heads])
    layers = rng.choice([1, 1, 2, 3, 4, 5])
    while True:
        lo = _log(rng, 1, 6000)
        hi = min(8192, lo + rng.choice([0, lo // 3, lo, 20 * lo]))
        if op == "packed":
            c = dict(op=op, n=_log(rng, 1, 200), len_lo=lo, len_hi=hi, log=rng.random() < 0.5, heads=heads, kv_heads=kv_heads,
                     layers=layers, fused=rng.random() < 0.5)
            if c["n"] * hi ** 2 * heads * (1 + layers) <= 2 * 8192 ** 2 * 8 * 3 and c["n"] * hi * heads <= 300000:
                return c
        elif op == "store":
            rows = _log(rng, 1, 4096)
            c = dict(op=op, dtype=rng.choice(["bf16", "f32"]), n=_log(rng, 1, 256), rows=rows, kv_heads=kv_heads, layers=layers,
                     cap=rows + rng.randrange(0, 500))
            if c["n"] * c["cap"] * kv_heads * (1 + layers) <= 5 * 4096 * 8 * 3:
                return c
        elif op == "attn":
            c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), n=_log(rng, 1, 256), len_lo=lo * rng.choice([0, 1, 1, 4]), len_hi=hi * 4,
                     heads=heads, kv_heads=kv_heads, layers=layers, weights=rng.random() < 0.4)
            if c["n"] * c["len_hi"] * kv_heads * (1 + layers) <= 128 * 4096 * 8 * 5 and c["n"] * c["len_hi"] * heads <= 128 * 4096 * 8:
                return c
        elif op == "mass":
            rows = rng.choice([1, 1, rng.randrange(2, 33), _log(rng, 33, 600)])
            c = dict(op=op, n=_log(rng, 1, 256), rows=rows, len_lo=lo * rng.choice([0, 1, 1]), len_hi=hi, heads=heads, kv_heads=kv_heads,
                     decay=rng.choice([1.0, 0.99, 0.5, 0.0]))
            if c["n"] * rows * hi * heads <= 16 * 512 * 512 * 8:
                return c
        else:
            keep = _log(rng, 1, 4000)
            sink = min(keep // 2, rng.choice([0, 1, 4, 5, 64]))
            c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32", "q4"]), n=_log(rng, 1, 128), len_lo=lo * rng.choice([0, 1]), len_hi=hi,
                     keep=keep, sink=sink, recent=min(keep - sink, rng.choice([0, 1, 16, 100, 1000])), kv_heads=kv_heads, layers=layers)
            if keep <= hi and c["n"] * hi * kv_heads * (1 + layers) * (2 if c["dtype"] == "f32" else 1) <= 48 * 2304 * 8 * 5:
                return c


def _spread(n, lo, hi):
    """n lengths over lo..hi in no order, the same for every seed (the work of a case depends on them)."""
    return [lo + (i * 7919 + 13) % (hi - lo + 1) for i in range(n)]


def _lens(case):
    n, lo, hi = case["n"], case["len_lo"], case["len_hi"]
    if case.get("log"):
        at = _spread(n, 0, max(n - 1, 1))
        return [max(lo, min(hi, int(round(lo * (hi / lo) ** (a / max(n - 1, 1)))))) for a in at]
    return _spread(n, lo, hi)


def _elem(case):
    return {"bf16": 2, "f32": 4}[case.get("dtype", "bf16")]


def work(case):
    op = case["op"]
    if op == "mass":
        T = _lens(case)
        rows = [min(case["rows"], t) if case["rows"] > 32 else case["rows"] for t in T]
        n = sum(r * t for r, t in zip(rows, T)) * case["heads"]
        return {"bytes": 4.0 * n + 8.0 * sum(T) * case["kv_heads"], "flops": 1.0 * n}
    Hk, L = case["kv_heads"], case["layers"]
    if op == "store":
        n = case["n"] * case["rows"] * Hk * (1 + L)
        return {"bytes": n * (2 * DH * _elem(case) + 2 * 36.0), "flops": 6.0 * DH * n}
    T = _lens(case)
    if op == "evict":
        row = 36 if case["dtype"] == "q4" else DH * _elem(case)
        moved = sum(max(0, case["keep"] - case["sink"]) for t in T if t > case["keep"])
        back = (36 + DH * 4) * sum(min(t, case["keep"]) for t in T) if case["dtype"] == "q4" else 0
        return {"bytes": Hk * (1 + L) * (2.0 * moved * row + back) + 4.0 * Hk * sum(T), "flops": 4.0 * Hk * sum(T)}
    H = case["heads"]
    if op == "attn":
        s = 4.0 * sum(T) * H if case["weights"] else 0.0
        return {"bytes": 36.0 * sum(T) * Hk * (1 + L) + len(T) * H * DH * (1 + L) * _elem(case) + s, "flops": 2.0 * sum(T) * H * DH * (1 + L)}
    pairs = sum(t * (t + 1) // 2 for t in T)
    return {"bytes": 2.0 * sum(T) * DH * (1 + L) * (H + Hk), "flops": 2.0 * pairs * H * DH * (1 + L)}


# ------------------------------------------------------------------------------------------- inputs
def _codes(gen, *shape):
    """Bytes of two codes each, 0..15, the middle ones more often than the outer ones (as codes of a projection's rows are)."""
    r = lambda m: torch.randint(0, 256, shape, generator=gen, device=DEV, dtype=torch.uint8).bitwise_and_(m)      # noqa: E731
    return r(0x77).add_(r(0x77)).add_(r(0x11))


def _scales(gen, *shape):
    """(step, low) of rows that reach from some -2.5 to 2.5."""
    step = 0.25 + 0.15 * torch.rand(*shape, 1, generator=gen, device=DEV)
    low = -7.5 * step + 0.3 * torch.randn(*shape, 1, generator=gen, device=DEV)
    return torch.cat([step, low], -1).bfloat16()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op = case["op"]
    dt = torch.float32 if case.get("dtype") == "f32" else torch.bfloat16
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV, dtype=torch.float32)            # noqa: E731
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)                                # noqa: E731
    st = {"case": case, "seed": seed, "dt": dt}
    n = case["n"]
    ids = torch.randperm(n, generator=gen, device=DEV).to(torch.int32)
    if op == "packed":
        H, Hk, L = case["heads"], case["kv_heads"], case["layers"]
        T = _lens(case)
        N = sum(T)
        first = [0]
        for t in T:
            first.append(first[-1] + t)
        st.update(lens=T, first=i32(first), max_len=max(T), out=torch.zeros(L, N, H, DH, dtype=dt, device=DEV))
        if case["fused"]:                                 # q, k and v of a token side by side, as one projection leaves them
            qkv = randn(L, N, H + 2 * Hk, DH).to(dt)      # (of the layers above the first only the values are used)
            st["q"], st["k"], st["v"] = qkv[0, :, :H], qkv[0, :, H:H + Hk], qkv[:, :, H + Hk:]
        else:
            st["q"], st["k"], st["v"] = randn(N, H, DH).to(dt), randn(N, Hk, DH).to(dt), randn(L, N, Hk, DH).to(dt)
    elif op == "store":
        Hk, L, R, cap = case["kv_heads"], case["layers"], case["rows"], case["cap"]
        wide = 0.5 + torch.rand(Hk, DH, generator=gen, device=DEV) * 1.5           # dims of a projection differ in size and middle
        mid = randn(Hk, DH) * 0.5
        st["k"], st["v"] = (randn(n, R, Hk, DH) * wide + mid).to(dt), (randn(L, n, R, Hk, DH) * wide).to(dt)
        st["pos"] = i32([(i * 31) % (cap - R + 1) for i in range(n)])
        st["codes"] = torch.zeros(1 + L, n, Hk, cap, DH // 2, dtype=torch.uint8, device=DEV)
        st["scales"] = torch.zeros(1 + L, n, Hk, cap, 2, dtype=torch.bfloat16, device=DEV)
        st["k_back"], st["v_back"] = torch.zeros_like(st["k"]), torch.zeros_like(st["v"])
    elif op == "attn":
        H, Hk, L = case["heads"], case["kv_heads"], case["layers"]
        T = _lens(case)
        cap = max(max(T), 1)
        st.update(lens=i32(T), max_len=cap, q=randn(n, H, DH).to(dt), codes=_codes(gen, 1 + L, n, Hk, cap, DH // 2),
                  scales=_scales(gen, 1 + L, n, Hk, cap), out=torch.zeros(L, n, H, DH, dtype=dt, device=DEV))
        st["S"] = torch.zeros(n, H, cap, device=DEV) if case["weights"] else None
    elif op == "mass":
        H, Hk, R = case["heads"], case["kv_heads"], case["rows"]
        T = _lens(case)
        cap = max(max(T), 1)
        st.update(lens=i32(T), max_len=cap, mass=torch.rand(n, Hk, cap, generator=gen, device=DEV) * 3.0)
        if R > 32:                                        # prompts: [sequence][head][row][position], causal
            z = randn(n, H, R, cap).mul_(1.5).exp_()
            z.mul_(torch.arange(cap, device=DEV) <= torch.arange(R, device=DEV)[:, None])
            st["S"], st["rows"], st["begin"] = z, i32([min(R, t) for t in T]), i32([0] * n)
            st["strides"] = (H * R * cap, cap, R * cap)
        else:                                             # steps: [item][row][head][position]; the newest position has none yet
            z = randn(n, R, H, cap).mul_(1.5).exp_()
            st["S"], st["rows"], st["begin"] = z, None, i32([max(0, t - 1) for t in T])
            st["strides"] = (R * H * cap, H * cap, cap)
        st["S"].div_(st["S"].sum(-1, keepdim=True).clamp_min(1e-20))
    else:
        Hk, L = case["kv_heads"], case["layers"]
        T = _lens(case)
        cap = max(max(T), 1)
        st.update(lens=i32(T), max_len=cap, mass=torch.exp(randn(n, Hk, cap) * 1.5) * 0.1, lens_out=i32([0] * n),
                  kept=torch.full((n, Hk, case["keep"]), -1, dtype=torch.int32, device=DEV))
        if case["dtype"] == "q4":
            st["codes"], st["scales"] = _codes(gen, 1 + L, n, Hk, cap, DH // 2), _scales(gen, 1 + L, n, Hk, cap)
            st["back"] = torch.zeros(1 + L, n, case["keep"], Hk, DH, device=DEV)
            st["back_rows"], st["back_pos"] = i32([min(t, case["keep"]) for t in T]), i32([0] * n)
        else:                                             # cache planes as the library keeps them
            st["planes"] = randn(1 + L, n, Hk, cap, DH).to(dt)
    st["ids"] = ids
    if own:
        st["call"] = _plan(st)
    return st


def _plan(st):
    """The argument blocks and the workspace that a user's program keeps beside its buffers."""
    from paper_1906_11024_b200 import binding as B
    case, op, n = st["case"], st["case"]["op"], st["case"]["n"]
    code = B.SAN_F32 if case.get("dtype") == "f32" else B.SAN_BF16
    room = lambda b: torch.empty(max(b, 1), dtype=torch.uint8, device=DEV)       # noqa: E731

    def planes(x, kind, scales=None):
        step = dict(d_k_scale=scales[0], d_v_scale=scales[1:]) if scales is not None else {}
        return B.planes(dtype=kind, n_kv_heads=x.shape[2], n_layers=x.shape[0] - 1, d_k=x[0], d_v=x[1:],
                        v_stride=x.shape[1] * x.shape[2] * x.shape[3] * DH, max_ids=x.shape[1], cap_len=x.shape[3], **step)

    if op == "packed":
        q, k, v = st["q"], st["k"], st["v"]
        a = B.packed_args(dtype=code, n_heads=case["heads"], n_kv_heads=case["kv_heads"], n_layers=case["layers"], d_q=q, ld_q=q.stride(0),
                          d_k=k, ld_k=k.stride(0), d_v=v, ld_v=v.stride(1), v_stride=v.stride(0), d_first=st["first"], n_seq=n,
                          n_tokens=q.shape[0], max_len=st["max_len"], d_out=st["out"])
        rc, b = B.san_packed_block_bytes(a)
        B.check(rc)
        ws = room(b)
        return lambda: B.san_packed_block(a, ws, b)
    if op == "store":
        p = planes(st["codes"], B.SAN_Q4, st["scales"])

        def store():
            rc = B.san_quant_append(p, code, st["k"], st["v"], st["ids"], st["pos"], None, n, case["rows"])
            return rc or B.san_quant_read(p, code, st["k_back"], st["v_back"], st["ids"], st["pos"], None, n, case["rows"])
        return store
    if op == "attn":
        p = planes(st["codes"], B.SAN_Q4, st["scales"])
        a = B.step_rows(dtype=code, n_heads=case["heads"], d_q=st["q"], d_ids=st["ids"], d_lens=st["lens"], n_items=n, max_len=st["max_len"],
                        d_S=st["S"], ld_s=st["max_len"], d_out=st["out"])
        rc, b = B.san_quant_attn_bytes(p, a)
        B.check(rc)
        ws = room(b)
        return lambda: B.san_quant_attn(p, a, ws, b)
    if op == "mass":
        a = B.mass_args(n_heads=case["heads"], n_kv_heads=case["kv_heads"], d_S=st["S"], item_stride=st["strides"][0], row_stride=st["strides"][1],
                        head_stride=st["strides"][2], n_rows=case["rows"], d_rows=st["rows"], d_ids=st["ids"], d_lens=st["lens"], d_begin=st["begin"],
                        n_items=n, max_len=st["max_len"], decay=case["decay"], d_mass=st["mass"], ld_mass=st["max_len"], max_ids=n)
        return lambda: B.san_weight_mass(a)
    q4 = case["dtype"] == "q4"
    p = planes(st["codes"], B.SAN_Q4, st["scales"]) if q4 else planes(st["planes"], code)
    a = B.evict_args(d_ids=st["ids"], d_lens=st["lens"], n_items=n, max_len=st["max_len"], n_keep=case["keep"], n_sink=case["sink"],
                     n_recent=case["recent"], d_mass=st["mass"], ld_mass=st["max_len"], d_kept=st["kept"], ld_kept=case["keep"],
                     d_lens_out=st["lens_out"])
    rc, b = B.san_cache_evict_bytes(p, a)
    B.check(rc)
    ws = room(b)

    def evict():
        rc = B.san_cache_evict(p, a, ws, b)
        if rc or not q4:
            return rc
        return B.san_quant_read(p, B.SAN_F32, st["back"][0], st["back"][1:], st["ids"], st["back_pos"], st["back_rows"], n, case["keep"])
    return evict


# ------------------------------------------------------------------------------------------- one pass
def run(st):
    op = st["case"]["op"]
    if own:
        if st["call"]() != 0:
            raise RuntimeError("the call was refused")
    else:
        {"packed": _packed, "store": _store, "attn": _attn, "mass": _mass, "evict": _evict}[op](st)
    if op == "packed":
        return st["out"]
    if op == "store":
        return {"k": st["k_back"], "v": st["v_back"]}
    if op == "attn":
        return {"out": st["out"]} | ({"S": st["S"]} if st["case"]["weights"] else {})
    if op == "mass":
        return st["mass"]
    rows = {"rows": st["back"]} if st["case"]["dtype"] == "q4" else {"planes": st["planes"]}
    return rows | {"mass": st["mass"], "lens": st["lens_out"], "kept": st["kept"]}


def _softmax(z, seen):
    """Weights over the last axis where `seen`; a row that sees nothing gets zeros."""
    z = torch.where(seen, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = (z - torch.where(top == -math.inf, 0.0, top)).exp()
    return p / p.sum(-1, keepdim=True).clamp_min(1e-30)


def _packed(st):
    case, T = st["case"], st["lens"]
    H, Hk, L, N = case["heads"], case["kv_heads"], case["layers"], st["q"].shape[0]
    q, k, v = st["q"].float() / 8.0, st["k"].float(), st["v"].float()

    def attend(q, k, v):                                  # [batch][position][heads][64]
        n, t = q.shape[:2]
        at = torch.arange(t, device=DEV)
        z = torch.einsum("iahrd,ibhd->ihrab", q.reshape(n, t, Hk, H // Hk, DH), k)
        p = _softmax(z, at[None, :] <= at[:, None])
        return torch.einsum("ihrab,libhd->liahrd", p, v).reshape(L, n, t, H, DH)

    if len(T) * max(T) ** 2 * H <= 1 << 27:               # all at once, padded: later positions are seen by padding alone
        at = (st["first"][:-1, None] + torch.arange(max(T), device=DEV)).clamp_max(N - 1).long()
        real = torch.arange(max(T), device=DEV)[None, :] < (st["first"][1:] - st["first"][:-1])[:, None]
        st["out"].copy_(attend(q[at], k[at], v[:, at])[:, real])
        return
    a = 0
    for t in T:
        st["out"][:, a:a + t] = attend(q[None, a:a + t], k[None, a:a + t], v[:, None, a:a + t])[:, 0]
        a += t


def _quantise(x):
    """Rows [..., 64] -> codes, (step, low), decided in 64 bits."""
    bits = lambda y: y.float().contiguous().view(torch.int32)                                     # noqa: E731
    real = lambda b: b.view(torch.float32)                                                        # noqa: E731
    least, most = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    b = bits(least)                                       # to bf16, down: cut off, or away from zero
    low = real(torch.where(b >= 0, b, b + 0xffff) & -0x10000).double()
    wide = (most.double() - low) / 15.0
    step = wide.float()
    step = torch.where(step.double() < wide, torch.nextafter(step, torch.full_like(step, math.inf)), step)
    step = real((bits(step) + 0xffff) & -0x10000).double()          # to bf16, up
    codes = torch.where(step > 0, torch.round((x.double() - low) / step), 0.0).clamp(0, 15)
    return codes.to(torch.uint8), torch.cat([step, low], -1).bfloat16()


def _numbers(codes, scales):
    """Bytes [..., 32] and (step, low) [..., 2] -> the numbers that they stand for, float32."""
    n = torch.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], DH)
    return scales[..., 1:].float() + scales[..., :1].float() * n.float()


def _store(st):
    case = st["case"]
    R, Hk = case["rows"], case["kv_heads"]
    pos = st["pos"].long()[:, None] + torch.arange(R, device=DEV)                                 # [n][rows]
    at = (st["ids"].long()[:, None, None], torch.arange(Hk, device=DEV), pos[:, :, None])
    for y, x in enumerate([st["k"], *st["v"]]):           # [n][rows][heads][64]
        codes, scales = _quantise(x)
        st["codes"][y].index_put_(at, codes[..., 0::2] | codes[..., 1::2] << 4)
        st["scales"][y].index_put_(at, scales)
    st["k_back"].copy_(_numbers(st["codes"][0][at], st["scales"][0][at]))
    for y in range(case["layers"]):
        st["v_back"][y].copy_(_numbers(st["codes"][1 + y][at], st["scales"][1 + y][at]))


def _attn(st):
    case = st["case"]
    H, Hk, L, n, T = case["heads"], case["kv_heads"], case["layers"], case["n"], st["max_len"]
    ids = st["ids"].long()
    q = st["q"].float().view(n, Hk, H // Hk, DH) / 8.0
    z = torch.einsum("ihrd,ihtd->ihrt", q, _numbers(st["codes"][0][ids], st["scales"][0][ids]))
    seen = torch.arange(T, device=DEV) < st["lens"][:, None]
    p = _softmax(z, seen[:, None, None])
    for y in range(L):
        st["out"][y] = torch.einsum("ihrt,ihtd->ihrd", p, _numbers(st["codes"][1 + y][ids], st["scales"][1 + y][ids])).reshape(n, H, DH)
    if case["weights"]:                                   # entries behind a row's length stay as they are
        st["S"].copy_(torch.where(seen[:, None], p.view(n, H, T), st["S"]))


def _mass(st):
    case = st["case"]
    H, Hk, n, R, T = case["heads"], case["kv_heads"], case["n"], case["rows"], st["max_len"]
    at, ids = torch.arange(T, device=DEV), st["ids"].long()
    S = st["S"] if R > 32 else st["S"].transpose(1, 2)    # [n][head][row][position]
    if st["rows"] is not None:
        S = torch.where((torch.arange(R, device=DEV) < st["rows"][:, None])[:, None, :, None], S, 0.0)
    got = S.reshape(n, Hk, H // Hk * R, T).sum(2)
    old = torch.where((at < st["begin"][:, None])[:, None], st["mass"][ids], 0.0)
    st["mass"][ids] = torch.where((at < st["lens"][:, None])[:, None], case["decay"] * old + got, st["mass"][ids])


def _evict(st):
    case = st["case"]
    n, Hk, K, T = case["n"], case["kv_heads"], case["keep"], st["max_len"]
    ids, lens, at = st["ids"].long(), st["lens"].long()[:, None, None], torch.arange(T, device=DEV)
    full = lens > K                                       # shorter ones stay as they are
    mass = st["mass"][ids]
    key = torch.where(torch.isnan(mass), -math.inf, mass).double()
    # what stays in any case before the others, what is not there behind them; ties: the lowest position
    order = torch.where(at >= lens, 2, torch.where((at < case["sink"]) | (at >= lens - case["recent"]), 0, 1))
    rank = torch.sort(key, dim=-1, descending=True, stable=True).indices
    rank = rank.gather(-1, torch.sort(order.expand_as(key).gather(-1, rank), dim=-1, stable=True).indices)
    pick = torch.sort(rank[..., :min(K, T)], dim=-1).values
    if pick.shape[-1] < K:
        pick = torch.nn.functional.pad(pick, (0, K - pick.shape[-1]))
    to = torch.arange(K, device=DEV).expand(n, Hk, K)
    pick = torch.where(full, pick, to.clamp_max(T - 1))
    alive = to < lens.clamp_max(K)
    st["kept"].copy_(torch.where(alive, pick, st["kept"]).int())
    st["lens_out"].copy_(lens.clamp_max(K)[:, 0, 0].int())
    i, h, a = torch.nonzero(full & alive, as_tuple=True)
    src, dst, head = pick[i, h, a], a, h
    st["mass"][ids[i], head, dst] = st["mass"][ids[i], head, src]
    if case["dtype"] == "q4":
        for x in (st["codes"], st["scales"]):
            x[:, ids[i], head, dst] = x[:, ids[i], head, src]
        rows = _numbers(st["codes"][:, ids, :, :K], st["scales"][:, ids, :, :K]).transpose(2, 3)            # [1 + L][n][keep][heads][64]
        st["back"][:, :, :rows.shape[2]] = torch.where((torch.arange(rows.shape[2], device=DEV) < st["back_rows"][:, None])[None, :, :, None, None],
                                                       rows, st["back"][:, :, :rows.shape[2]])
        return
    rows = st["planes"][:, ids[i], head, src]
    if case["dtype"] == "bf16":                           # chunk c of the row at position p sits at chunk c ^ (p & 7)
        chunk = torch.arange(8, device=DEV)[None, :] ^ (src & 7)[:, None] ^ (dst & 7)[:, None]
        rows = torch.take_along_dim(rows.view(*rows.shape[:2], 8, 8), chunk[None, :, :, None], 2).reshape(rows.shape)
    st["planes"][:, ids[i], head, dst] = rows


# ------------------------------------------------------------------------------------------- definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"packed": _exact_packed, "store": _exact_store, "attn": _exact_attn, "mass": _exact_mass, "evict": _exact_evict}[case["op"]](st)


def _exact_packed(st):
    """Sequence by sequence, head by head, a run of query rows at a time."""
    case = st["case"]
    H, Hk, L = case["heads"], case["kv_heads"], case["layers"]
    out = st["out"].double()
    a = 0
    for t in st["lens"]:
        for h in range(H):
            q, k = st["q"][a:a + t, h].double(), st["k"][a:a + t, h // (H // Hk)].double()
            v = st["v"][:, a:a + t, h // (H // Hk)].double()
            for b in range(0, t, 2048):
                e = min(t, b + 2048)
                z = q[b:e] @ k[:e].T / math.sqrt(DH)
                z.masked_fill_(torch.ones_like(z, dtype=torch.bool).triu_(b + 1), -math.inf)
                out[:, a + b:a + e, h] = torch.softmax(z, -1) @ v[:, :e]
        a += t
    return out


def _bf16_grid(x, up):
    """The bf16 number next to each x that is not below it (up) or not above it."""
    y = x.bfloat16()
    wrong = (y.double() < x) if up else (y.double() > x)
    bits = y.contiguous().view(torch.int16)               # neighbours are one apart; negative numbers run downwards
    moved = bits + torch.where((y > 0) == up, 1, -1).to(torch.int16)
    moved = torch.where(y == 0, torch.full_like(bits, 1 if up else -0x7fff), moved)
    return torch.where(wrong, moved, bits).view(torch.bfloat16).double()


def _exact_store(st):
    def back(x):
        x = x.double()
        low = _bf16_grid(x.amin(-1, keepdim=True), False)
        step = _bf16_grid((x.amax(-1, keepdim=True) - low) / 15, True)
        t = torch.where(step > 0, (x - low) / step, torch.zeros_like(x))
        n = torch.floor(t)
        n = n + ((t - n > 0.5) | ((t - n == 0.5) & (n % 2 == 1))).double()
        return low + step * n.clamp(0, 15)
    return {"k": back(st["k"]), "v": torch.stack([back(v) for v in st["v"]])}


def _row_numbers(codes, scales):
    x = torch.empty(*codes.shape[:-1], DH, dtype=torch.float64, device=DEV)
    x[..., 0::2], x[..., 1::2] = (codes % 16).double(), (codes // 16).double()
    return x * scales[..., 0:1].double() + scales[..., 1:2].double()


def _exact_attn(st):
    """Row by row over the rows that it sees."""
    case = st["case"]
    r = case["heads"] // case["kv_heads"]
    out = torch.zeros(case["layers"], case["n"], case["heads"], DH, dtype=torch.float64, device=DEV)
    S = st["S"].double() if case["weights"] else None
    for i, (b, t) in enumerate(zip(st["ids"].tolist(), st["lens"].tolist())):
        if t == 0:
            continue
        k = _row_numbers(st["codes"][0, b, :, :t], st["scales"][0, b, :, :t])
        v = _row_numbers(st["codes"][1:, b, :, :t], st["scales"][1:, b, :, :t])
        p = torch.softmax(st["q"][i].double().view(-1, r, DH) @ k.transpose(1, 2) / math.sqrt(DH), -1)       # [key heads][group][t]
        out[:, i] = (p[None] @ v).reshape(case["layers"], case["heads"], DH)
        if S is not None:
            S[i, :, :t] = p.reshape(case["heads"], t)
    return {"out": out} | ({"S": S} if case["weights"] else {})


def _exact_mass(st):
    case = st["case"]
    r = case["heads"] // case["kv_heads"]
    mass = st["mass"].double()
    for i, (b, t, new) in enumerate(zip(st["ids"].tolist(), st["lens"].tolist(), st["begin"].tolist())):
        rows = case["rows"] if st["rows"] is None else int(st["rows"][i])
        for h in range(case["kv_heads"]):
            mass[b, h, new:t] = 0
            mass[b, h, :t] *= case["decay"]
            for g in range(h * r, h * r + r):
                S = st["S"][i, g, :rows, :t] if case["rows"] > 32 else st["S"][i, :rows, g, :t]
                mass[b, h, :t] += S.double().sum(0)
    return mass


def _exact_evict(st):
    case = st["case"]
    K, sink, recent = case["keep"], case["sink"], case["recent"]
    q4 = case["dtype"] == "q4"
    mass, kept, lens_out = st["mass"].double(), st["kept"].clone(), st["lens_out"].clone()
    planes = None if q4 else st["planes"].double()
    back = st["back"].double() if q4 else None
    host = st["mass"].double().cpu().numpy()
    for i, (b, t) in enumerate(zip(st["ids"].tolist(), st["lens"].tolist())):
        lens_out[i] = min(t, K)
        for h in range(case["kv_heads"]):
            if t <= K:
                at = list(range(t))
            else:
                free = range(sink, t - recent)
                row = host[b, h]
                best = sorted(free, key=lambda j: (-row[j], j))[:K - sink - recent]
                at = list(range(sink)) + sorted(best) + list(range(t - recent, t))
            src = torch.tensor(at, dtype=torch.long, device=DEV)
            kept[i, h, :len(at)] = src.int()
            if q4:
                back[:, i, :len(at), h] = _row_numbers(st["codes"][:, b, h, src], st["scales"][:, b, h, src])
            if t <= K or not at:
                continue
            mass[b, h, :K] = st["mass"][b, h, src].double()
            if q4:
                continue
            x = st["planes"][:, b, h, src].double()
            if case["dtype"] == "bf16":
                dst = torch.arange(K, device=DEV)
                place = torch.arange(DH, device=DEV)[None, :] ^ (8 * ((src ^ dst) & 7))[:, None]
                x = torch.gather(x, -1, place.expand(x.shape))
            planes[:, b, h, :K] = x
    return ({"rows": back} if q4 else {"planes": planes}) | {"mass": mass, "lens": lens_out, "kept": kept}
