"""Measured cases of the serving operators around the shared-attention decode path.

Four calls, as a decoder that answers long prompts with a beam of hypotheses makes them:

  select        san_beam_select: the next hypotheses of every sentence, chosen over beam and vocabulary,
                with their token histories, lengths and scores carried over
  prefix        san_prefix_attn: one decode step of attention for rows that share long prefixes, each
                prefix read once for all of its rows, joined with every row's own cached rows
  window        san_window_attn: one decode step of attention over a sliding window of the cache and a
                few first rows that stay visible (sinks)
  window_block  san_window_block: the same visibility for a whole sequence at once (prompts)

``own`` is false: ``run`` computes them from elementary torch operations.  ``own`` is true: it calls the
library.  ``exact`` is the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DH = 64


# ------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the latency of one request's step: one sentence, beam 4, the first step (one live hypothesis)
        dict(name="select one sentence", op="select", dtype="f32", n_sent=1, beam=4, vocab=32000, pad=0, steps=1,
             history=64, alpha=0.0, done=0.0),
        # the translation batch of the base workload: 64 sentences, beam 4
        dict(name="select base", op="select", dtype="bf16", n_sent=64, beam=4, vocab=32000, pad=0, steps=30,
             history=66, alpha=0.6, done=0.2),
        # the widest beam of the beam sweep over an odd vocabulary: rows that start off 16-byte boundaries
        dict(name="select beam 20 odd", op="select", dtype="f32", n_sent=37, beam=20, vocab=50257, pad=0, steps=17,
             history=110, alpha=1.0, done=0.1),
        # the big workload with a large shared vocabulary
        dict(name="select large", op="select", dtype="bf16", n_sent=128, beam=4, vocab=128000, pad=64, steps=50,
             history=512, alpha=0.6, done=0.1),
        # one request, a sentence-sized forced prefix, a few rows decoded
        dict(name="prefix one sentence", op="prefix", dtype="bf16", n_prefix=1, group=4, ragged=False, heads=8,
             kv_heads=8, layers=1, prefix_lo=60, prefix_hi=60, own_lo=9, own_hi=9, cap=66),
        # the long workload: 32 prompts of 512 positions, beam 4, a block of four layers
        dict(name="prefix long", op="prefix", dtype="bf16", n_prefix=32, group=4, ragged=False, heads=8, kv_heads=8,
             layers=4, prefix_lo=512, prefix_hi=512, own_lo=1, own_hi=255, cap=512),
        # one system prompt in front of every hypothesis of a large batch
        dict(name="prefix one prompt for all", op="prefix", dtype="bf16", n_prefix=1, group=512, ragged=False, heads=16,
             kv_heads=16, layers=1, prefix_lo=8192, prefix_hi=8192, own_lo=20, own_hi=100, cap=110),
        # float32, a few prompts of odd lengths with unequal numbers of rows
        dict(name="prefix f32 ragged", op="prefix", dtype="f32", n_prefix=5, group=7, ragged=True, heads=8, kv_heads=8,
             layers=2, prefix_lo=33, prefix_hi=1001, own_lo=0, own_hi=70, cap=80),
        # a batch far into its targets: the window of the cache that is still read, a block of four layers
        dict(name="window step", op="window", dtype="bf16", n=128, heads=8, kv_heads=8, layers=4, len_lo=1,
             len_hi=4096, window=512, sink=4),
        # few rows over a very long window, query heads in groups of four
        dict(name="window step few rows", op="window", dtype="bf16", n=2, heads=16, kv_heads=4, layers=1,
             len_lo=30001, len_hi=32001, window=16384, sink=5),
        # a sentence-sized batch, a block of three layers
        dict(name="window block sentences", op="window_block", dtype="bf16", n=64, heads=8, kv_heads=8, layers=3,
             len_lo=10, len_hi=60, window=16, sink=1),
        # long prompts
        dict(name="window block prompts", op="window_block", dtype="bf16", n=2, heads=8, kv_heads=8, layers=2,
             len_lo=7777, len_hi=8192, window=1024, sink=4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["select", "prefix", "window", "window_block"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "select":
        while True:
            c = dict(op=op, dtype=dtype, n_sent=_log(rng, 1, 128), beam=rng.choice([1, 2, 4, 4, 5, 8, 12, 20, 32]),
                     vocab=_log(rng, 50, 130000), pad=rng.choice([0, 0, 1, 8, 64]), steps=_log(rng, 1, 200),
                     history=0, alpha=rng.choice([0.0, 0.6, 1.0]), done=rng.choice([0.0, 0.1, 0.5]))
            c["history"] = c["steps"] + _log(rng, 1, 64)
            if c["n_sent"] * c["beam"] * c["vocab"] <= 512 * 128000:
                return c
    heads = rng.choice([2, 3, 4, 6, 8, 12, 16])
    kv_heads = rng.choice([k for k in (1, 2, 3, 4, 8, 16) if heads % k == 0 and heads // k <= 8] + [heads, heads])
    layers = rng.choice([1, 1, 2, 3, 4, 5])
    if op == "prefix":
        while True:
            lo = _log(rng, 1, 4000)
            own = _log(rng, 1, 600)
            c = dict(op=op, dtype=dtype, n_prefix=_log(rng, 1, 32), group=_log(rng, 1, 256), ragged=rng.random() < 0.5,
                     heads=heads, kv_heads=kv_heads, layers=layers, prefix_lo=lo, prefix_hi=lo + rng.randrange(0, lo + 1),
                     own_lo=rng.randrange(0, own + 1), own_hi=own, cap=own + rng.randrange(0, 40))
            rows = c["n_prefix"] * c["group"]
            if rows * c["prefix_hi"] * heads * (1 + layers) <= 512 * 8192 * 16 * 2 and rows * c["cap"] * kv_heads * (1 + layers) <= 512 * 110 * 16 * 2:
                return c
    if op == "window":
        while True:
            lo = _log(rng, 1, 8000)
            c = dict(op=op, dtype=dtype, n=_log(rng, 1, 256), heads=heads, kv_heads=kv_heads, layers=layers, len_lo=lo,
                     len_hi=lo + rng.randrange(0, lo + 1), window=_log(rng, 1, 2048), sink=rng.choice([0, 1, 4, 5, 64]))
            if c["n"] * c["len_hi"] * kv_heads * (1 + layers) <= 128 * 4096 * 8 * 5:
                return c
    while True:
        lo = _log(rng, 1, 4000)
        c = dict(op=op, dtype="bf16", n=_log(rng, 1, 64), heads=heads, kv_heads=kv_heads, layers=layers, len_lo=lo,
                 len_hi=lo + rng.randrange(0, lo + 1), window=_log(rng, 1, 2048), sink=rng.choice([0, 1, 4, 5, 64]))
        if c["n"] * c["len_hi"] ** 2 * heads * (1 + layers) <= 2 * 8192 ** 2 * 8 * 3:
            return c


def _spread(n, lo, hi):
    """n lengths over lo..hi in no order, the same for every seed (the work of a case depends on them)."""
    return [lo + (i * 7919 + 13) % (hi - lo + 1) for i in range(n)]


def _groups(case):
    """Rows of each prefix: all alike, or 1 .. group."""
    n, g = case["n_prefix"], case["group"]
    return _spread(n, 1, g) if case["ragged"] else [g] * n


def _elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def work(case):
    e = _elem(case)
    if case["op"] == "select":
        rows = case["n_sent"] * case["beam"]
        live = _live_rows(case)
        return {"bytes": live * case["vocab"] * e + rows * (2 * 4 * (3 + min(case["steps"], case["history"])) + 8),
                "flops": 4.0 * live * case["vocab"]}
    H, Hk, L = case["heads"], case["kv_heads"], case["layers"]
    if case["op"] == "prefix":
        g = _groups(case)
        P = _spread(len(g), case["prefix_lo"], case["prefix_hi"])
        T = _spread(sum(g), case["own_lo"], case["own_hi"])
        kv = (sum(P) + sum(T)) * Hk * DH * (1 + L) * e
        pairs = sum(a * b for a, b in zip(g, P)) + sum(T)
        return {"bytes": kv + sum(g) * H * DH * (1 + L) * e, "flops": 2.0 * pairs * H * DH * (1 + L)}
    T = _spread(case["n"], case["len_lo"], case["len_hi"])
    w, s = case["window"], case["sink"]
    if case["op"] == "window":
        seen = sum(min(t, w) + min(s, max(0, t - w)) for t in T)
        return {"bytes": seen * Hk * DH * (1 + L) * e + len(T) * H * DH * (1 + L) * e, "flops": 2.0 * seen * H * DH * (1 + L)}
    pairs = 0
    for t in T:
        a = np.arange(1, t + 1, dtype=np.int64)
        pairs += int((np.minimum(a, w) + np.minimum(s, np.maximum(0, a - w))).sum())
    return {"bytes": sum(T) * DH * (1 + L) * (H + Hk) * e, "flops": 2.0 * pairs * H * DH * (1 + L)}


def _live_rows(case):
    """Hypotheses whose logits are read: neither finished nor without a score."""
    return int((~_done(case) & ~_dead(case)).sum())


def _dead(case):
    rows = np.arange(case["n_sent"] * case["beam"])
    return (rows % case["beam"] > 0) if case["steps"] == 1 else np.zeros(rows.shape, bool)   # first step: one live hypothesis


def _done(case):
    rows = np.arange(case["n_sent"] * case["beam"])
    return ((rows * 2654435761) % 1000 < 1000 * case["done"]) & ~_dead(case)


# ------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV, dtype=torch.float32).to(dt)     # noqa: E731
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)                    # noqa: E731
    st = {"case": case, "seed": seed, "dt": dt}
    if case["op"] == "select":
        rows, V = case["n_sent"] * case["beam"], case["vocab"]
        # a trained model's logits: a wide body and a few tokens that stand out
        x = torch.randn(rows, V + case["pad"], generator=gen, device=DEV) * 2.0
        peaks = torch.randint(0, V, (rows, min(8, V)), generator=gen, device=DEV)
        x.scatter_add_(1, peaks, 4.0 + 3.0 * torch.rand(peaks.shape, generator=gen, device=DEV))
        st["logits"] = x.to(dt)
        done, dead = torch.from_numpy(_done(case)).to(DEV), torch.from_numpy(_dead(case)).to(DEV)
        steps = case["steps"]
        n = torch.randint(max(1, steps // 2), steps + 1, (rows,), generator=gen, device=DEV)
        lens = torch.where(done, n, torch.full_like(n, steps))
        score = -(0.3 + 0.4 * torch.rand(rows, generator=gen, device=DEV)) * lens
        st["score"] = torch.where(dead, torch.full_like(score, -math.inf), score)
        st["len"], st["done"] = lens.to(torch.int32), done.to(torch.int32)
        st["tokens"] = torch.randint(0, V, (rows, case["history"]), generator=gen, device=DEV, dtype=torch.int32)
        st["eos"] = min(2, V - 1)
        st["score_out"], st["len_out"], st["done_out"] = (torch.empty_like(st[k]) for k in ("score", "len", "done"))
        st["tokens_out"] = torch.full_like(st["tokens"], -1)
        st["parent"], st["next"] = torch.empty_like(st["len"]), torch.empty_like(st["len"])
    else:
        H, Hk, L = case["heads"], case["kv_heads"], case["layers"]
        if case["op"] == "window_block":
            T = _spread(case["n"], case["len_lo"], case["len_hi"])
            cap = max(T)
            st["q"], st["k"] = randn(len(T), cap, H, DH), randn(len(T), cap, Hk, DH)
            st["v"] = randn(L, len(T), cap, Hk, DH)
            st["out"] = torch.zeros(L, len(T), cap, H, DH, dtype=dt, device=DEV)
        else:
            if case["op"] == "prefix":
                g = _groups(case)
                P = _spread(len(g), case["prefix_lo"], case["prefix_hi"])
                T, cap = _spread(sum(g), case["own_lo"], case["own_hi"]), case["cap"]
                st["pk"], st["pv"] = randn(len(g), max(P), Hk, DH), randn(L, len(g), max(P), Hk, DH)
                st["first"], st["plens"] = i32(np.concatenate([[0], np.cumsum(g)])), i32(P)
                st["max_group"] = max(g)
            else:
                T = _spread(case["n"], case["len_lo"], case["len_hi"])
                cap = max(T)
            # cache planes as the library keeps them: head-major, the 16-byte chunks of a bf16 row permuted by position
            st["q"], st["k"] = randn(len(T), H, DH), randn(len(T), Hk, cap, DH)
            st["v"] = randn(L, len(T), Hk, cap, DH)
            st["ids"] = torch.randperm(len(T), generator=gen, device=DEV).to(torch.int32)
            st["out"] = torch.zeros(L, len(T), H, DH, dtype=dt, device=DEV)
        st["lens"], st["max_len"] = i32(T), max(T)
    if own:
        st["call"] = _plan(st)
    return st


def _plan(st):
    """The argument blocks and the workspace that a user's program keeps beside its buffers."""
    from paper_1906_11024_b200 import binding as B
    case = st["case"]
    dtype = B.SAN_BF16 if case["dtype"] == "bf16" else B.SAN_F32
    room = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)       # noqa: E731
    if case["op"] == "select":
        rc, n = B.san_beam_select_bytes(case["n_sent"], case["beam"], case["vocab"])
        B.check(rc)
        ws = room(n)
        a = B.select_args(dtype=dtype, n_sent=case["n_sent"], beam=case["beam"], vocab=case["vocab"],
                          d_logits=st["logits"], ld_logits=st["logits"].shape[1], eos=st["eos"], alpha=case["alpha"],
                          d_score=st["score"], d_len=st["len"], d_done=st["done"], d_tokens=st["tokens"],
                          ld_tokens=case["history"], d_score_out=st["score_out"], d_len_out=st["len_out"],
                          d_done_out=st["done_out"], d_tokens_out=st["tokens_out"], d_parent=st["parent"],
                          d_next=st["next"], d_workspace=ws, workspace_bytes=n)
        return (B.san_beam_select, a, ws)
    if case["op"] == "window_block":
        a = (dtype, case["heads"], case["kv_heads"], case["layers"], case["window"], case["sink"], st["q"], st["k"], st["v"],
             st["lens"], case["n"], st["q"].shape[1], st["max_len"], st["out"])
        return (lambda args: B.san_window_block(*args), a, None)
    rows = B.cached_rows(dtype=dtype, n_heads=case["heads"], n_kv_heads=case["kv_heads"], n_layers=case["layers"], d_q=st["q"],
                         d_k=st["k"], d_v=st["v"], v_stride=st["v"][0].numel(), max_ids=st["k"].shape[0],
                         cap_len=st["k"].shape[2], d_ids=st["ids"], d_lens=st["lens"], n_items=st["q"].shape[0],
                         max_len=st["max_len"], d_out=st["out"])
    if case["op"] == "prefix":
        pre = B.shared_prefix(d_k=st["pk"], d_v=st["pv"], v_stride=st["pv"][0].numel(), n_prefix=st["pk"].shape[0],
                              cap_len=st["pk"].shape[1], d_lens=st["plens"], max_len=st["pk"].shape[1],
                              d_first=st["first"], max_group=st["max_group"])
        rc, n = B.san_prefix_attn_bytes(rows, pre)
        B.check(rc)
        ws = room(n)
        return (lambda a: B.san_prefix_attn(a, pre, ws, n), rows, ws)
    rc, n = B.san_window_attn_bytes(rows, case["window"], case["sink"])
    B.check(rc)
    ws = room(n)
    return (lambda a: B.san_window_attn(a, case["window"], case["sink"], ws, n), rows, ws)


# ------------------------------------------------------------------------------------------- one pass
def run(st):
    op = st["case"]["op"]
    if own:
        call, args, _ = st["call"]
        if call(args) != 0:
            raise RuntimeError("the call was refused")
        if op == "select":
            return {k: st[k + "_out"] for k in ("score", "len", "done", "tokens")} | {"parent": st["parent"], "next": st["next"]}
        return st["out"]
    return {"select": _select, "prefix": _prefix, "window": _window, "window_block": _window_block}[op](st)


def _select(st):
    case = st["case"]
    S, B, V = case["n_sent"], case["beam"], case["vocab"]
    x = st["logits"][:, :V].double()                      # scores are compared with one another: 64 bits
    x = torch.where(torch.isnan(x), -math.inf, x)
    top = x.amax(1, keepdim=True)
    lp = torch.where(x == top, 0.0, x - top)
    logp = lp - lp.exp().sum(1, keepdim=True).log()
    score, done = st["score"].double(), st["done"] != 0
    cand = score[:, None] + logp
    only = torch.full_like(cand, -math.inf)
    only[:, st["eos"]] = score
    cand = torch.where(done[:, None], only, cand)
    n_new = st["len"] + (~done).int()                     # a candidate's length
    rank = cand / ((5.0 + n_new.double()) / 6.0).pow(case["alpha"])[:, None]
    rank, at = torch.sort(rank.view(S, B * V), dim=1, descending=True, stable=True)     # ties: the lowest index first
    best, at = rank[:, :B], at[:, :B]
    none = best == -math.inf
    slot = torch.arange(B, device=DEV).expand(S, B)
    parent = torch.where(none, slot, at // V)
    row = (torch.arange(S, device=DEV)[:, None] * B + parent).view(-1)
    none = none.view(-1)
    keeps = done[row] | none
    nxt = torch.where(none, st["eos"], (at % V).view(-1))
    new = torch.where(none, -math.inf, cand.view(S, B * V).gather(1, at).view(-1))
    old_len = st["len"][row]
    length = old_len + (~keeps).int()
    pos = torch.arange(case["history"], device=DEV)[None, :]
    tokens = torch.where((pos == old_len[:, None]) & ~keeps[:, None], nxt[:, None].int(), st["tokens"][row])
    tokens = torch.where(pos < length[:, None], tokens, st["tokens_out"])
    return {"score": new.float(), "len": length.int(), "done": (keeps | (nxt == st["eos"])).int(), "tokens": tokens,
            "parent": parent.view(-1).int(), "next": nxt.int()}


def _natural(planes):
    """Cached rows [..., position, 64] with their elements in order."""
    if planes.dtype != torch.bfloat16:
        return planes.float()
    T = planes.shape[-2]
    chunk = torch.arange(8, device=DEV)[None, :] ^ (torch.arange(T, device=DEV)[:, None] & 7)
    x = planes.reshape(*planes.shape[:-1], 8, 8)
    return x[..., torch.arange(T, device=DEV)[:, None], chunk, :].reshape(planes.shape).float()


def _softmax(z, seen):
    """Weights over the last axis where `seen`; a row that sees nothing gets zeros."""
    z = torch.where(seen, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = (z - torch.where(top == -math.inf, 0.0, top)).exp()
    return p / p.sum(-1, keepdim=True).clamp_min(1e-30)


def _prefix(st):
    case, dt = st["case"], st["dt"]
    H, Hk, L = case["heads"], case["kv_heads"], case["layers"]
    n, r = st["q"].shape[0], H // Hk
    first, plens, ids, lens = st["first"].long(), st["plens"].long(), st["ids"].long(), st["lens"].long()
    item = torch.arange(n, device=DEV)
    g = torch.searchsorted(first[1:].contiguous(), item, right=True)
    at = item - first[g]
    G, R, P, T = plens.shape[0], st["max_group"], st["pk"].shape[1], st["max_len"]
    q = st["q"].float().view(n, Hk, r, DH) / 8.0
    qg = torch.zeros(G, R, Hk, r, DH, device=DEV)
    qg[g, at] = q
    zp = torch.einsum("gihrd,gphd->gihrp", qg, st["pk"].float())[g, at]
    k, v = _natural(st["k"][ids][:, :, :T]), _natural(st["v"][:, ids][:, :, :, :T])
    zo = torch.einsum("ihrd,ihtd->ihrt", q, k)
    seen = torch.cat([torch.arange(P, device=DEV) < plens[g][:, None], torch.arange(T, device=DEV) < lens[:, None]], 1)
    p = _softmax(torch.cat([zp, zo], -1), seen[:, None, None])
    pg = torch.zeros(G, R, Hk, r, P, device=DEV)
    pg[g, at] = p[..., :P]
    out = torch.einsum("gihrp,lgphd->lgihrd", pg, st["pv"].float())[:, g, at]
    return (out + torch.einsum("ihrt,lihtd->lihrd", p[..., P:], v)).reshape(L, n, H, DH).to(dt)


def _window(st):
    case, dt = st["case"], st["dt"]
    H, Hk, L, w, s = (case[k] for k in ("heads", "kv_heads", "layers", "window", "sink"))
    n, r = st["q"].shape[0], H // Hk
    ids, lens = st["ids"].long(), st["lens"].long()
    w, s = min(w, st["max_len"]), min(s, st["max_len"])
    # the rows that are seen, and no others: the first s, then the last w
    begin = (lens - w).clamp_min(0)
    pos = torch.cat([torch.arange(s, device=DEV).expand(n, s), begin[:, None] + torch.arange(w, device=DEV)], 1)
    seen = torch.cat([pos[:, :s] < begin[:, None], pos[:, s:] < lens[:, None]], 1)
    pos = pos.clamp_max(st["k"].shape[2] - 1)
    head = torch.arange(Hk, device=DEV)[None, :, None]
    k, v = st["k"][ids[:, None, None], head, pos[:, None]], st["v"][:, ids[:, None, None], head, pos[:, None]]
    if st["dt"] == torch.bfloat16:                        # chunks back in order
        chunk = (torch.arange(8, device=DEV) ^ (pos[..., None] & 7))[:, None, :, :, None]
        k = torch.take_along_dim(k.view(n, Hk, -1, 8, 8), chunk, 3).reshape(k.shape)
        v = torch.take_along_dim(v.view(L, n, Hk, -1, 8, 8), chunk[None], 4).reshape(v.shape)
    z = torch.einsum("ihrd,ihtd->ihrt", st["q"].float().view(n, Hk, r, DH) / 8.0, k.float())
    p = _softmax(z, seen[:, None, None])
    return torch.einsum("ihrt,lihtd->lihrd", p, v.float()).reshape(L, n, H, DH).to(dt)


def _window_block(st):
    case, dt = st["case"], st["dt"]
    H, Hk, L, w, s = (case[k] for k in ("heads", "kv_heads", "layers", "window", "sink"))
    n, cap = st["q"].shape[:2]
    a, b = torch.arange(cap, device=DEV)[:, None], torch.arange(cap, device=DEV)[None, :]
    lens = st["lens"].long()[:, None, None]
    seen = (b <= a) & ((b > a - w) | (b < s)) & (b < lens)
    z = torch.einsum("iahrd,ibhd->ihrab", st["q"].float().view(n, cap, Hk, H // Hk, DH) / 8.0, st["k"].float())
    p = _softmax(z, seen[:, None, None])
    out = torch.einsum("ihrab,libhd->liahrd", p, st["v"].float()).reshape(L, n, cap, H, DH).to(dt)
    # rows behind the end of a sequence stay as they were
    return torch.where((torch.arange(cap, device=DEV)[None, :] < lens[:, :, 0])[None, :, :, None, None], out, st["out"])


# ------------------------------------------------------------------------------------------- definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"select": _exact_select, "prefix": _exact_rows, "window": _exact_rows, "window_block": _exact_block}[case["op"]](st)


def _exact_select(st):
    case = st["case"]
    S, B, V, eos = case["n_sent"], case["beam"], case["vocab"], st["eos"]
    score, length, done = st["score"].double().cpu().numpy(), st["len"].cpu().numpy(), st["done"].cpu().numpy()
    tokens, out = st["tokens"].cpu().numpy(), st["tokens_out"].cpu().numpy().copy()
    got = {"score": np.empty(S * B), "len": np.empty(S * B, np.int32), "done": np.empty(S * B, np.int32),
           "parent": np.empty(S * B, np.int32), "next": np.empty(S * B, np.int32)}
    for i in range(S):
        found = []                                        # (-rank, slot, token, score)
        for b in range(B):
            j = i * B + b
            if score[j] == -math.inf:
                continue
            if done[j]:
                found.append((-score[j] / ((5.0 + length[j]) / 6.0) ** case["alpha"], b, eos, score[j]))
                continue
            x = st["logits"][j, :V].double()
            lse = torch.logsumexp(x, 0)
            kth = torch.topk(x, min(B, V)).values[-1]
            at = torch.nonzero(x >= kth)[:, 0]            # every token that could be chosen, ties among them
            total = (score[j] + (x[at] - lse)).cpu().numpy()
            lp = ((5.0 + length[j] + 1) / 6.0) ** case["alpha"]
            found += [(-t / lp, b, int(v), t) for t, v in zip(total, at.cpu().numpy())]
        found.sort(key=lambda f: f[:3])
        for b in range(B):
            j = i * B + b
            if b < len(found):
                _, p, tok, t = found[b]
                q = i * B + p
                n = length[q] + (0 if done[q] else 1)
                out[j, :length[q]] = tokens[q, :length[q]]
                if not done[q]:
                    out[j, length[q]] = tok
                got["score"][j], got["len"][j], got["done"][j] = t, n, int(bool(done[q]) or tok == eos)
                got["parent"][j], got["next"][j] = p, tok
            else:
                out[j, :length[j]] = tokens[j, :length[j]]
                got["score"][j], got["len"][j], got["done"][j], got["parent"][j], got["next"][j] = -math.inf, length[j], 1, b, eos
    got["tokens"] = out
    return got


def _plane(x, pos):
    """Rows `pos` of planes [..., position, 64] in 64 bits, elements in order."""
    bf16 = x.dtype == torch.bfloat16
    x = x[..., pos, :].double()
    if not bf16:
        return x
    place = (torch.arange(DH, device=DEV)[None, :] // 8 ^ (pos[:, None] % 8)) * 8 + torch.arange(DH, device=DEV)[None, :] % 8
    return torch.gather(x, -1, place.expand(x.shape))


def _attend(q, k, v):
    """q [h][64], k [h][t][64], v [l][h][t][64] -> [l][h][64]."""
    if k.shape[1] == 0:
        return torch.zeros(v.shape[0], q.shape[0], DH, dtype=torch.float64, device=DEV)
    p = torch.softmax((k @ q[:, :, None])[:, :, 0] / math.sqrt(DH), -1)
    return (p[None, :, None, :] @ v)[:, :, 0, :]


def _exact_rows(st):
    """Row by row: the rows that it sees, one after the other, in 64 bits."""
    case = st["case"]
    H, Hk = case["heads"], case["kv_heads"]
    n, r = st["q"].shape[0], H // Hk
    ids, lens = st["ids"].tolist(), st["lens"].tolist()
    out = torch.zeros(case["layers"], n, H, DH, dtype=torch.float64, device=DEV)
    first = st["first"].tolist() if case["op"] == "prefix" else None
    g = 0
    for i in range(n):
        t = lens[i]
        pos = torch.arange(t, device=DEV)
        if case["op"] == "window":
            pos = pos[(pos >= t - case["window"]) | (pos < case["sink"])]
        k, v = _plane(st["k"][ids[i]], pos), _plane(st["v"][:, ids[i]], pos)
        if first is not None:
            while i >= first[g + 1]:
                g += 1
            if i == first[g]:
                P = int(st["plens"][g])
                pk, pv = st["pk"][g, :P].double().transpose(0, 1), st["pv"][:, g, :P].double().transpose(1, 2)
            k, v = torch.cat([pk, k], 1), torch.cat([pv, v], 2)
        out[:, i] = _attend(st["q"][i].double(), k.repeat_interleave(r, 0), v.repeat_interleave(r, 1))
    return out


def _exact_block(st):
    """Head by head, a run of query rows at a time over the keys that the run can see."""
    case = st["case"]
    H, Hk, L, w, s = (case[k] for k in ("heads", "kv_heads", "layers", "window", "sink"))
    n, cap = st["q"].shape[:2]
    out = st["out"].double()
    for i, t in enumerate(st["lens"].tolist()):
        for a0 in range(0, t, 1024):
            a1 = min(t, a0 + 1024)
            lo = max(0, a0 - w + 1)
            lo = 0 if lo <= s else lo
            keys = torch.cat([torch.arange(min(s, lo), device=DEV), torch.arange(lo, a1, device=DEV)])
            a, b = torch.arange(a0, a1, device=DEV)[:, None], keys[None, :]
            hide = (b > a) | ((b <= a - w) & (b >= s))
            k = st["k"][i, keys].double().transpose(0, 1).repeat_interleave(H // Hk, 0)
            z = st["q"][i, a0:a1].double().transpose(0, 1) @ k.transpose(1, 2) / math.sqrt(DH)
            p = torch.softmax(z.masked_fill(hide[None], -math.inf), -1)
            v = st["v"][:, i][:, keys].double().transpose(1, 2).repeat_interleave(H // Hk, 1)
            out[:, i, a0:a1] = (p[None] @ v).transpose(1, 2)
    return out
