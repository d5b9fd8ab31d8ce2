"""The calls for long prompts and small caches together, as a server uses them: prompts laid end to end through san_packed_block, their rows
into a cache of four bits (san_quant_append), steps over it with their weights (san_quant_attn), the mass of the rows
(san_weight_mass), and the cache cut back (san_cache_evict) whenever it has grown over its bound.  Then the same on a context's planes
with san_attn_weights, and prompts' weights from san_full_block.  Every step is followed on the host in 64 bits."""
import pytest
import torch

from paper_1906_11024_b200 import binding as B
from paper_1906_11024_b200 import build as san_build
from tests.keep_helpers import DH, keep, numbers, pack, packed, quant_attend, quantise_row

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    san_build.build()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def workspace(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_cache_steps_and_eviction(dtype):
    dt, code = (torch.bfloat16, B.SAN_BF16) if dtype == "bf16" else (torch.float32, B.SAN_F32)
    H, Hk, L, lens, steps, cap, n_keep, sink, recent, decay = 4, 2, 2, [37, 1, 150], 14, 160, 40, 2, 6, 0.9
    n, N = len(lens), sum(lens)
    gen = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=gen)                                          # noqa: E731
    # the prompts' projection, fused, and their attention
    qkv = r(L, N, H + 2 * Hk, DH).bfloat16().to(DEV)
    q, k, v = qkv[0, :, :H], qkv[0, :, H:H + Hk], qkv[:, :, H + Hk:]
    first = [0]
    for t in lens:
        first.append(first[-1] + t)
    d_first, out = i32(first), torch.zeros(L, N, H, DH, dtype=torch.bfloat16, device=DEV)
    a = B.packed_args(dtype=B.SAN_BF16, n_heads=H, n_kv_heads=Hk, n_layers=L, d_q=q, ld_q=q.stride(0), d_k=k, ld_k=k.stride(0), d_v=v, ld_v=v.stride(1),
                      v_stride=v.stride(0), d_first=d_first, n_seq=n, n_tokens=N, max_len=max(lens), d_out=out)
    rc, nb = B.san_packed_block_bytes(a)
    B.check(rc)
    ws = workspace(nb)
    B.check(B.san_packed_block(a, ws, nb))
    torch.cuda.synchronize()
    for s, t in enumerate(lens):
        want, bound = packed(q[first[s]:first[s + 1]], k[first[s]:first[s + 1]], v[:, first[s]:first[s + 1]], torch.bfloat16)
        assert not bool(((out[:, first[s]:first[s + 1]].double() - want).abs() > bound).any())
    # their rows into the cache, padded as an append takes them
    ids = [2, 0, 1]
    codes = torch.zeros(1 + L, n, Hk, cap, 32, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(1 + L, n, Hk, cap, 2, dtype=torch.bfloat16, device=DEV)
    cache = B.planes(dtype=B.SAN_Q4, n_kv_heads=Hk, n_layers=L, d_k=codes[0], d_v=codes[1:], v_stride=codes[0].numel() * 2, d_k_scale=scales[0],
                     d_v_scale=scales[1:], max_ids=n, cap_len=cap)
    R = max(lens)
    pk, pv = torch.zeros(n, R, Hk, DH, dtype=dt, device=DEV), torch.zeros(L, n, R, Hk, DH, dtype=dt, device=DEV)
    for s, t in enumerate(lens):
        pk[s, :t], pv[:, s, :t] = k[first[s]:first[s + 1]].to(dt), v[:, first[s]:first[s + 1]].to(dt)
    d_ids, d_lens, status = i32(ids), i32(lens), torch.zeros(8, dtype=torch.int32, device=DEV)
    B.check(B.san_quant_append(cache, code, pk, pv, d_ids, None, d_lens, n, R, status))
    hc, hs = codes.cpu(), scales.cpu()                              # the host's own cache, from here on
    for s, t in enumerate(lens):
        for y, x in enumerate([pk[s].cpu(), *pv[:, s].cpu()]):
            for j in range(0, t, 7):
                for h in range(Hk):
                    c, step, low = quantise_row(x[j, h].double().tolist())
                    assert hc[y, ids[s], h, j].tolist() == pack(c) and hs[y, ids[s], h, j].double().tolist() == [step, low]
    mass = torch.zeros(n, Hk, cap, device=DEV)
    host_mass, now = torch.zeros(n, Hk, cap, dtype=torch.float64), list(lens)
    out_n = torch.zeros(n, dtype=torch.int32, device=DEV)
    evicted = 0
    for step in range(steps):
        # this step's rows behind the others, then attention over all of them, weights, mass
        nk, nv, nq = r(n, 1, Hk, DH).to(dt), r(L, n, 1, Hk, DH).to(dt), r(n, H, DH).to(dt)
        B.check(B.san_quant_append(cache, code, nk.to(DEV), nv.to(DEV), d_ids, i32(now), None, n, 1, status))
        for s in range(n):
            for y, x in enumerate([nk[s, 0], *nv[:, s, 0]]):
                for h in range(Hk):
                    c, st, low = quantise_row(x[h].double().tolist())
                    hc[y, ids[s], h, now[s]] = torch.tensor(pack(c), dtype=torch.uint8)
                    hs[y, ids[s], h, now[s]] = torch.tensor([st, low]).bfloat16()
        begin = list(now)
        now = [t + 1 for t in now]
        dq, dn = nq.to(DEV), i32(now)
        o, S = torch.zeros(L, n, H, DH, dtype=dt, device=DEV), torch.zeros(n, H, cap, device=DEV)
        rows = B.step_rows(dtype=code, n_heads=H, d_q=dq, d_ids=d_ids, d_lens=dn, n_items=n, max_len=0, d_S=S, ld_s=cap, d_out=o, d_status=status)
        rc, nb = B.san_quant_attn_bytes(cache, rows)
        B.check(rc)
        ws = workspace(nb)
        B.check(B.san_quant_attn(cache, rows, ws, nb))
        d_begin = i32(begin)
        B.check(B.san_weight_mass(B.mass_args(n_heads=H, n_kv_heads=Hk, d_S=S, item_stride=H * cap, row_stride=H * cap, head_stride=cap, n_rows=1,
                                              d_ids=d_ids, d_lens=dn, d_begin=d_begin, n_items=n, max_len=cap, decay=decay, d_mass=mass, ld_mass=cap,
                                              max_ids=n, d_status=status)))
        torch.cuda.synchronize()
        for s in range(n):
            t, b = now[s], ids[s]
            want, bound, p, p_bound = quant_attend(nq[s], hc[:, b, :, :t], hs[:, b, :, :t], dt)
            assert not bool(((o[:, s].cpu().double() - want).abs() > bound).any())
            assert not bool(((S[s, :, :t].cpu().double() - p).abs() > p_bound).any())
            host_mass[b, :, t - 1] = 0
            host_mass[b, :, :t] = decay * host_mass[b, :, :t] + p.reshape(Hk, H // Hk, t).sum(1)
        got = mass.cpu().double()
        assert float((got - host_mass).abs().max()) <= 1e-5 * H         # float32 sums of weights, each within 1e-6 or so, over the steps
        # every fourth step caches over their bound are cut back, by the device's own mass
        if step % 4 == 3:
            kept = torch.full((n, Hk, n_keep), -1, dtype=torch.int32, device=DEV)
            e = B.evict_args(d_ids=d_ids, d_lens=dn, n_items=n, max_len=0, n_keep=n_keep, n_sink=sink, n_recent=recent, d_mass=mass, ld_mass=cap,
                             d_kept=kept, ld_kept=n_keep, d_lens_out=out_n, d_status=status)
            rc, nb = B.san_cache_evict_bytes(cache, e)
            B.check(rc)
            ws = workspace(nb)
            B.check(B.san_cache_evict(cache, e, ws, nb))
            torch.cuda.synchronize()
            for s in range(n):
                for h in range(Hk):
                    b, t = ids[s], now[s]
                    at = keep(got[b, h, :t].tolist(), t, n_keep, sink, recent)
                    assert kept[s, h, :len(at)].tolist() == at
                    if t > n_keep:
                        evicted += 1
                        hc[:, b, h, :n_keep], hs[:, b, h, :n_keep] = hc[:, b, h, at], hs[:, b, h, at]
                        host_mass[b, h, :n_keep] = host_mass[b, h, at]
            now = [min(t, n_keep) for t in now]
            assert out_n.tolist() == now
    assert evicted > 4 and status.tolist() == [0] * 8
    # the rows that are left, as numbers
    back_k, back_v = torch.zeros(n, cap, Hk, DH, device=DEV), torch.zeros(L, n, cap, Hk, DH, device=DEV)
    B.check(B.san_quant_read(cache, B.SAN_F32, back_k, back_v, d_ids, None, i32(now), n, cap))
    torch.cuda.synchronize()
    for s in range(n):
        want = numbers(hc[:, ids[s], :, :now[s]], hs[:, ids[s], :, :now[s]]).transpose(1, 2)
        got = torch.cat([back_k[None, s], back_v[:, s]])[:, :now[s]].cpu().double()
        assert bool(((got - want).abs() <= 2.0 ** -24 * want.abs()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_eviction_on_a_contexts_planes(dtype):
    """Weights of san_attn_weights over a context's cache, their mass, eviction in the planes of each block, and the step after: attention
    over the rows that were kept."""
    dt, code = (torch.bfloat16, B.SAN_BF16) if dtype == "bf16" else (torch.float32, B.SAN_F32)
    L, H, n, cap, blocks, n_keep = 3, 2, 3, 90, [1, 2], 30
    cfg = B.san_config(n_layers=L, n_heads=H, d_head=DH, max_sent=n, beam=1, max_tgt_len=cap, max_src_len=8, dtype=code, self_is_aan=0,
                       encdec_shared_context=0)
    rc, cb, wb = B.san_query_bytes(cfg, len(blocks), 1)
    B.check(rc)
    store, ws = torch.empty(cb, dtype=torch.uint8, device=DEV), torch.empty(wb, dtype=torch.uint8, device=DEV)
    rc, ctx = B.san_create(cfg, blocks, [L], store, cb, ws, wb)
    B.check(rc)
    gen = torch.Generator().manual_seed(6)
    lens = [90, 25, 61]
    k, v = (torch.randn(*s, generator=gen).to(dt) for s in ((len(blocks), n, cap, H, DH), (L, n, cap, H, DH)))
    ids, dl = i32([0, 1, 2]), i32(lens)
    dk, dv = k.to(DEV), v.to(DEV)
    B.check(B.san_cache_append(ctx, B.SAN_SELF, 0, L, dk, dv, ids, None, dl, n, cap))
    layer = 0
    for b, size in enumerate(blocks):
        q = torch.randn(n, H, DH, generator=gen).to(dt).to(DEV)
        S, mass = torch.zeros(n, H, cap, device=DEV), torch.zeros(n, H, cap, device=DEV)
        B.check(B.san_attn_weights(ctx, B.SAN_SELF, b, q, ids, dl, n, 0, S, cap))
        B.check(B.san_weight_mass(B.mass_args(n_heads=H, n_kv_heads=H, d_S=S, item_stride=H * cap, row_stride=0, head_stride=cap, n_rows=1, d_ids=ids,
                                              d_lens=dl, n_items=n, max_len=cap, decay=1.0, d_mass=mass, ld_mass=cap, max_ids=n)))
        rc, kp, vp, stride = B.san_cache_planes(ctx, B.SAN_SELF, b)
        B.check(rc)
        planes = B.planes(dtype=code, n_kv_heads=H, n_layers=size, d_k=kp, d_v=vp, v_stride=stride, max_ids=n, cap_len=cap)
        lens_out = torch.zeros(n, dtype=torch.int32, device=DEV)
        torch.cuda.synchronize()
        before = mass.cpu()
        assert torch.equal(before, S.cpu())
        e = B.evict_args(d_ids=ids, d_lens=dl, n_items=n, n_keep=n_keep, n_sink=1, n_recent=4, d_mass=mass, ld_mass=cap, d_lens_out=lens_out)
        rc, nb = B.san_cache_evict_bytes(planes, e)
        B.check(rc)
        room = workspace(nb)
        B.check(B.san_cache_evict(planes, e, room, nb))
        # the next step's weights and outputs, by the calls of the context
        S2, O = torch.zeros(n, H, cap, device=DEV), torch.zeros(size, n, H, DH, dtype=dt, device=DEV)
        B.check(B.san_attn_weights(ctx, B.SAN_SELF, b, q, ids, lens_out, n, 0, S2, cap))
        B.check(B.san_attn_apply(ctx, B.SAN_SELF, b, layer, layer + size, S2, cap, ids, None, lens_out, n, 0, O))
        torch.cuda.synchronize()
        for i, t in enumerate(lens):
            for h in range(H):
                at = keep(before[i, h, :t].tolist(), t, n_keep, 1, 4)
                z = k[b, i, at, h].double() @ q[i, h].cpu().double() / 8.0
                p = torch.softmax(z, 0)
                assert float((S2[i, h, :len(at)].cpu().double() - p).abs().max()) <= 1e-5
                want = torch.einsum("t,ltd->ld", p, v[layer:layer + size, i, at, h].double())
                size_of = torch.einsum("t,ltd->ld", p, v[layer:layer + size, i, at, h].double().abs())
                off = (O[:, i, h].cpu().double() - want).abs()
                assert bool((off <= (2.0 ** -8 * want.abs() if dtype == "bf16" else 0) + 1e-5 * size_of + 1e-30).all())
        assert lens_out.tolist() == [min(t, n_keep) for t in lens]
        layer += size
    rc, err, detail = B.san_device_status(ctx)
    assert (rc, err) == (B.SAN_OK, 0), detail
    B.san_destroy(ctx)


def test_mass_of_prompts_from_full_attention():
    """Column sums of the weights that san_full_block writes: what a prompt's rows have received before the first step."""
    n, H, cap, lens = 2, 3, 70, [70, 33]
    gen = torch.Generator().manual_seed(7)
    q, k, v = (torch.randn(n, cap, H, DH, generator=gen).bfloat16().to(DEV) for _ in range(3))
    S, out = torch.zeros(n, H, cap, 72, device=DEV), torch.zeros(1, n, cap, H, DH, dtype=torch.bfloat16, device=DEV)
    dl, ids, mass = i32(lens), i32([1, 0]), torch.zeros(n, H, cap, device=DEV)
    B.check(B.san_full_block(B.SAN_BF16, H, 1, 1, q, k, v[None].contiguous(), dl, n, cap, 0, S, 72, out))
    zero = i32([0, 0])
    B.check(B.san_weight_mass(B.mass_args(n_heads=H, n_kv_heads=H, d_S=S, item_stride=H * cap * 72, row_stride=72, head_stride=cap * 72, n_rows=cap,
                                          d_rows=dl, d_ids=ids, d_lens=dl, d_begin=zero, n_items=n, max_len=cap, decay=1.0, d_mass=mass, ld_mass=cap,
                                          max_ids=n)))
    torch.cuda.synchronize()
    for i, t in enumerate(lens):
        for h in range(H):
            z = (q[i, :t, h].double() @ k[i, :t, h].double().T / 8.0).masked_fill(torch.ones(t, t, dtype=torch.bool, device=DEV).triu_(1), -torch.inf)
            want = torch.softmax(z, -1).sum(0)
            assert bool(((mass[1 - i, h, :t].double() - want).abs() <= 2e-5 * want + 1e-7).all())
