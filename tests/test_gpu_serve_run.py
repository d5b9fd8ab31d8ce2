"""The serving calls together, as a decoder with a forced prompt and a beam uses them: the prompt's rows through
san_full_block and san_window_block, steps through san_cache_append, san_prefix_attn and san_window_attn on the planes of
a context (san_cache_planes), san_beam_select, and san_beam_reorder by its parents.  Every step is followed on the host
in 64 bits."""
import numpy as np
import pytest
import torch

from paper_1906_11024_b200 import binding as B
from paper_1906_11024_b200 import build as san_build
from tests.serve_helpers import DH, attend, check_outputs, dtype_of, randn, select, weighted_size

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _context(code, L, H, S, beam, cap, blocks):
    cfg = B.san_config(n_layers=L, n_heads=H, d_head=DH, max_sent=S, beam=beam, max_tgt_len=cap, max_src_len=8, dtype=code,
                       self_is_aan=0, encdec_shared_context=0)
    rc, cb, wb = B.san_query_bytes(cfg, len(blocks), 1)
    B.check(rc)
    cache, ws = torch.empty(cb, dtype=torch.uint8, device=DEV), torch.empty(wb, dtype=torch.uint8, device=DEV)
    rc, ctx = B.san_create(cfg, blocks, [L], cache, cb, ws, wb)
    B.check(rc)
    return ctx, cache, ws


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_steps_selection_and_reorder(dtype):
    san_build.build()
    dt, code = dtype_of(dtype)
    L, H, S, beam, cap, V, steps, P, window, sink = 3, 2, 2, 4, 8, 90, 5, [37, 52], 3, 1
    blocks = [1, 2]
    n, pcap = S * beam, max(P)
    gen = torch.Generator().manual_seed(17)
    ctx, cache, ws = _context(code, L, H, S, beam, cap, blocks)
    # the prompt's rows as the projections of a prefill leave them, per block: keys of its first layer, values of each
    pk = [randn(gen, S, pcap, H, DH, dtype=dt) for _ in blocks]
    pv = [randn(gen, b, S, pcap, H, DH, dtype=dt) for b in blocks]
    dpk, dpv = [x.to(DEV) for x in pk], [x.to(DEV) for x in pv]
    plens = torch.tensor(P, dtype=torch.int32, device=DEV)
    if dtype == "bf16":
        # the prompt itself: windowed and full attention of its rows read the same buffers as the steps below
        pq = randn(gen, S, pcap, H, DH, dtype=dt).to(DEV)
        a, b = (torch.zeros(blocks[1], S, pcap, H, DH, dtype=dt, device=DEV) for _ in range(2))
        B.check(B.san_full_block(code, H, blocks[1], 1, pq, dpk[1], dpv[1], plens, S, pcap, 0, None, 0, a))
        B.check(B.san_window_block(code, H, H, blocks[1], pcap, 0, pq, dpk[1], dpv[1], plens, S, pcap, 0, b))
        torch.cuda.synchronize()
        for i, p in enumerate(P):
            assert (a[:, i, :p].double() - b[:, i, :p].double()).norm() <= 2.0 ** -7 * a[:, i, :p].double().norm()
    # the beam's state: one live hypothesis per sentence
    score = np.full(n, -np.inf, np.float32)
    score[::beam] = 0.0
    state = dict(score=score, len=np.zeros(n, np.int32), done=np.zeros(n, np.int32), tokens=np.zeros((n, cap), np.int32))
    dev = {k: torch.from_numpy(v.copy()).to(DEV) for k, v in state.items()}
    parent, nxt = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    logits = torch.zeros(n, V, device=DEV)
    rc, nb = B.san_beam_select_bytes(S, beam, V)
    sel_ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    sel = B.select_args(dtype=B.SAN_F32, n_sent=S, beam=beam, vocab=V, d_logits=logits, ld_logits=V, eos=1, alpha=0.6, d_score=dev["score"],
                        d_len=dev["len"], d_done=dev["done"], d_tokens=dev["tokens"], ld_tokens=cap, d_score_out=dev["score"],
                        d_len_out=dev["len"], d_done_out=dev["done"], d_tokens_out=dev["tokens"], d_parent=parent, d_next=nxt,
                        d_workspace=sel_ws, workspace_bytes=nb)
    ids = torch.arange(n, dtype=torch.int32, device=DEV)
    sent = torch.arange(S, dtype=torch.int32, device=DEV)
    first = torch.tensor([0, beam, 2 * beam], dtype=torch.int32, device=DEV)
    K = [[[] for _ in range(n)] for _ in blocks]                   # host: own rows of each sequence, per block / layer
    W = [[[] for _ in range(n)] for _ in range(L)]
    for step in range(steps):
        k_new, v_new = randn(gen, len(blocks), n, 1, H, DH, dtype=dt), randn(gen, L, n, 1, H, DH, dtype=dt)
        q = randn(gen, len(blocks), n, H, DH, dtype=dt)
        pos = torch.full((n,), step, dtype=torch.int32, device=DEV)
        lens = torch.full((n,), step + 1, dtype=torch.int32, device=DEV)
        dk, dv, dq = k_new.to(DEV), v_new.to(DEV), q.to(DEV)
        B.check(B.san_cache_append(ctx, B.SAN_SELF, 0, L, dk, dv, ids, pos, None, n, 1))
        for i in range(n):
            for b in range(len(blocks)):
                K[b][i] = K[b][i] + [k_new[b, i, 0]]
            for l in range(L):
                W[l][i] = W[l][i] + [v_new[l, i, 0]]
        layer = 0
        for b, size in enumerate(blocks):
            rc, kp, vp, stride = B.san_cache_planes(ctx, B.SAN_SELF, b)
            B.check(rc)
            out = torch.zeros(size, n, H, DH, dtype=dt, device=DEV)
            win = torch.zeros_like(out)
            make = lambda o: B.cached_rows(dtype=code, n_heads=H, n_kv_heads=H, n_layers=size, d_q=dq[b], d_k=kp, d_v=vp,   # noqa: E731
                                           v_stride=stride, max_ids=n, cap_len=cap, d_ids=ids, d_lens=lens, n_items=n, d_out=o)
            rows, wrows = make(out), make(win)
            pre = B.shared_prefix(d_k=dpk[b], d_v=dpv[b], v_stride=dpv[b][0].numel(), n_prefix=S, cap_len=pcap, d_lens=plens, d_first=first)
            rc, nw = B.san_prefix_attn_bytes(rows, pre)
            B.check(rc)
            at_ws = torch.empty(max(nw, B.san_window_attn_bytes(wrows, window, sink)[1], 1), dtype=torch.uint8, device=DEV)
            B.check(B.san_prefix_attn(rows, pre, at_ws, at_ws.numel()))
            B.check(B.san_window_attn(wrows, window, sink, at_ws, at_ws.numel()))
            torch.cuda.synchronize()
            for i in range(n):
                g = i // beam
                for h in range(H):
                    qi = q[b, i, h].double()
                    ko = torch.stack([r[h] for r in K[b][i]]).double()
                    vo = torch.stack([torch.stack([r[h] for r in W[layer + y][i]]) for y in range(size)]).double()
                    kk = torch.cat([pk[b][g, :P[g], h].double(), ko])
                    vv = torch.cat([pv[b][:, g, :P[g], h].double(), vo], 1)
                    want, slack = attend(qi, kk, vv)
                    check_outputs(out.cpu()[:, i, h], want, slack, weighted_size(qi, kk, vv), dt, ("prefix", step, i, h))
                    seen = [j for j in range(step + 1) if j >= step + 1 - window or j < sink]
                    want, slack = attend(qi, ko[seen], vo[:, seen])
                    check_outputs(win.cpu()[:, i, h], want, slack, weighted_size(qi, ko[seen], vo[:, seen]), dt, ("window", step, i, h))
            layer += size
        # selection, then every cache row follows its hypothesis
        x = torch.randn(n, V, generator=gen) * 3
        logits.copy_(x)
        want = select(x, state["score"], state["len"], state["done"], state["tokens"], 1, float(np.float32(0.6)), beam)
        B.check(B.san_beam_select(sel))
        B.check(B.san_beam_reorder(ctx, sent, parent, lens, S, 0))
        torch.cuda.synchronize()
        par = parent.cpu().numpy()
        assert np.array_equal(par, want["parent"]) and np.array_equal(nxt.cpu().numpy(), want["next"])
        assert np.array_equal(dev["len"].cpu().numpy(), want["len"]) and np.array_equal(dev["done"].cpu().numpy(), want["done"])
        state = {k: v.cpu().numpy() for k, v in dev.items()}
        for i in range(n):
            assert [int(t) for t in state["tokens"][i][:state["len"][i]]] == [int(t) for t in want["tokens"][i]]
        src = [i // beam * beam + par[i] for i in range(n)]
        K = [[K[b][src[i]] for i in range(n)] for b in range(len(blocks))]
        W = [[W[l][src[i]] for i in range(n)] for l in range(L)]
    rc, err, detail = B.san_device_status(ctx)
    assert (rc, err) == (B.SAN_OK, 0), detail
    B.san_destroy(ctx)


def test_cache_planes_of_every_block():
    """The addresses are those of the documented arena layout; bad blocks and kinds are refused."""
    san_build.build()
    L, H, S, beam, cap = 4, 2, 2, 2, 16
    ctx, cache, ws = _context(B.SAN_BF16, L, H, S, beam, cap, [1, 3])
    plane = (S * beam * H * cap * DH * 2 + 255) // 256 * 256
    for b, first in ((0, 0), (1, 1)):
        rc, k, v, stride = B.san_cache_planes(ctx, B.SAN_SELF, b)
        assert rc == B.SAN_OK and stride == plane // 2
        assert k == cache.data_ptr() + b * plane and v == cache.data_ptr() + (2 + first) * plane
    mem = (S * H * 8 * DH * 2 + 255) // 256 * 256
    rc, k, v, stride = B.san_cache_planes(ctx, B.SAN_ENCDEC, 0)
    base = cache.data_ptr() + (2 + L) * plane
    assert rc == B.SAN_OK and (k, v, stride) == (base, base + mem, mem // 2)
    assert B.san_cache_planes(ctx, B.SAN_SELF, 2)[0] == B.SAN_ERR_RANGE
    assert B.san_cache_planes(ctx, B.SAN_SELF, -1)[0] == B.SAN_ERR_RANGE
    assert B.san_cache_planes(ctx, 7, 0)[0] == B.SAN_ERR_RANGE
    B.san_destroy(ctx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_that_share_one_context(dtype):
    """Eq. 5: an encoder-decoder block has one value plane.  No distance to a second one is given, so that a call over the
    block's layers is refused; one over that plane answers with its values, the last block's too."""
    san_build.build()
    dt, code = dtype_of(dtype)
    L, H, S, src, enc = 4, 2, 3, 9, [1, 3]
    cfg = B.san_config(n_layers=L, n_heads=H, d_head=DH, max_sent=S, beam=2, max_tgt_len=4, max_src_len=src, dtype=code,
                       self_is_aan=0, encdec_shared_context=1)
    rc, cb, wb = B.san_query_bytes(cfg, 1, len(enc))
    B.check(rc)
    cache, ws = torch.zeros(cb, dtype=torch.uint8, device=DEV), torch.empty(wb, dtype=torch.uint8, device=DEV)
    rc, ctx = B.san_create(cfg, [L], enc, cache, cb, ws, wb)
    B.check(rc)
    gen = torch.Generator().manual_seed(3)
    lens, first = [9, 1, 4], [0, 1]
    k, v, q = (randn(gen, len(enc), *s, dtype=dt) for s in ((S, src, H, DH), (S, src, H, DH), (S, H, DH)))
    sent, pos = torch.arange(S, dtype=torch.int32, device=DEV), torch.zeros(S, dtype=torch.int32, device=DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    dk, dv, dq = k.to(DEV), v.to(DEV), q.to(DEV)
    for b in range(len(enc)):
        B.check(B.san_cache_append(ctx, B.SAN_ENCDEC, first[b], first[b] + 1, dk[b], dv[b], sent, pos, dl, S, src))
    for b, size in enumerate(enc):
        rc, kp, vp, stride = B.san_cache_planes(ctx, B.SAN_ENCDEC, b)
        assert (rc, stride) == (B.SAN_OK, 0)
        make = lambda layers, out: B.cached_rows(                                                # noqa: E731
            dtype=code, n_heads=H, n_kv_heads=H, n_layers=layers, d_q=dq[b], d_k=kp, d_v=vp, v_stride=stride, max_ids=S,
            cap_len=src, d_ids=sent, d_lens=dl, n_items=S, d_out=out)
        if size > 1:
            out = torch.full((size, S, H, DH), -7.0, dtype=dt, device=DEV)
            assert B.san_window_attn_bytes(make(size, out), src, 0)[0] == B.SAN_ERR_SHAPE
            assert B.san_window_attn(make(size, out), src, 0, None, 0) == B.SAN_ERR_SHAPE
            x = B.shared_prefix(d_k=dk, d_v=dk, v_stride=64, n_prefix=0, cap_len=1, d_lens=dl, d_first=dl)
            assert B.san_prefix_attn(make(size, out), x, None, 0) == B.SAN_ERR_SHAPE
        out = torch.full((1, S, H, DH), -7.0, dtype=dt, device=DEV)
        rows = make(1, out)
        assert B.san_window_attn_bytes(rows, src, 0) == (B.SAN_OK, 0)
        B.check(B.san_window_attn(rows, src, 0, None, 0))
        torch.cuda.synchronize()
        for i in range(S):
            for h in range(H):
                qq, kk, vv = q[b, i, h].double(), k[b, i, :lens[i], h].double(), v[b, None, i, :lens[i], h].double()
                want, slack = attend(qq, kk, vv)
                check_outputs(out.cpu()[:, i, h], want, slack, weighted_size(qq, kk, vv), dt, (b, i, h))
    rc, err, detail = B.san_device_status(ctx)
    assert (rc, err) == (B.SAN_OK, 0), detail
    B.san_destroy(ctx)
