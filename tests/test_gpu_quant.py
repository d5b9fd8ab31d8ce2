"""Rows in four bits (san_quant_append, san_quant_read) and step attention over them (san_quant_attn) against 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_1906_11024_b200 import binding as B
from paper_1906_11024_b200 import build as san_build
from tests.keep_helpers import DH, numbers, pack, quant_attend, quantise_row

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": (torch.bfloat16, B.SAN_BF16), "f32": (torch.float32, B.SAN_F32)}


@pytest.fixture(scope="module", autouse=True)
def _built():
    san_build.build()


def cache(ids, Hk, L, cap, fill=0):
    return (torch.full((1 + L, ids, Hk, cap, DH // 2), fill, dtype=torch.uint8, device=DEV),
            torch.full((1 + L, ids, Hk, cap, 2), -3.0, dtype=torch.bfloat16, device=DEV))


def planes(codes, scales):
    return B.planes(dtype=B.SAN_Q4, n_kv_heads=codes.shape[2], n_layers=codes.shape[0] - 1, d_k=codes[0], d_v=codes[1:],
                    v_stride=codes[0].numel() * 2, d_k_scale=scales[0], d_v_scale=scales[1:], max_ids=codes.shape[1], cap_len=codes.shape[3])


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------- rows
def special_rows(dt):
    gen = torch.Generator().manual_seed(3)
    r = lambda: torch.randn(DH, generator=gen)                                              # noqa: E731
    big = float(torch.finfo(dt).max)
    rows = [torch.zeros(DH), -torch.zeros(DH), torch.full((DH,), 1.7), torch.full((DH,), -1e-3), r(), r() * 1e-38, r() * 1e-42, r() * 1e30,
            torch.arange(DH).float() / 4 - 3, torch.arange(DH).float() % 31 * 0.5, r() + 1000, r() * 1e-6 - 5, -r().abs(), r().abs() * 3]
    x = r(); x[7] = math.nan; rows.append(x)
    x = r(); x[63] = math.inf; rows.append(x)
    x = r(); x[0] = -math.inf; rows.append(x)
    x = r(); x[0], x[1] = big, -big; rows.append(x)                     # float32: its low is beyond bf16
    x = r(); x[5] = 1.09e12; x[6] = -1.09e12; rows.append(x)                     # below 2^40; the next is not
    x = r(); x[9] = 1.1e12; rows.append(x)
    x = torch.zeros(DH); x[1] = 15.0; x[2:50] = torch.arange(48).float() * 0.25 + 0.5; rows.append(x)          # halves between codes
    x = torch.zeros(DH); x[0] = -2.25; x[1] = 5.25; x[2:] = 1e-12; rows.append(x)
    return torch.stack(rows).to(dt)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_of_every_kind_of_row(dtype):
    dt, code = TYPES[dtype]
    x = special_rows(dt)
    n = x.shape[0]
    codes, scales = cache(1, 1, 1, n)
    src = x.view(1, n, 1, DH).to(DEV)
    v = src.flip(1).contiguous()[None]
    B.check(B.san_quant_append(planes(codes, scales), code, src, v, i32([0]), None, None, 1, n))
    torch.cuda.synchronize()
    for plane, rows in ((0, x), (1, x.flip(0))):
        for j in range(n):
            want, step, low = quantise_row(rows[j].double().tolist())
            got = scales[plane, 0, 0, j].double().tolist()
            assert codes[plane, 0, 0, j].tolist() == pack(want), (plane, j)
            assert np.array_equal(got, [step, low], equal_nan=True), (plane, j, got, step, low)
            if math.isfinite(step):                         # no number is off by more than step / 2
                back = numbers(codes[plane, 0, 0, j].cpu(), scales[plane, 0, 0, j].cpu())
                assert float((back - rows[j].double()).abs().max()) <= step / 2 * (1 + 1e-12)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,R,Hk,L,cap", [(1, 1, 1, 1, 1), (5, 1, 3, 2, 9), (3, 17, 2, 1, 33), (2, 40, 1, 5, 40), (130, 1, 8, 4, 4)])
def test_rows_in_and_back(dtype, n, R, Hk, L, cap):
    dt, code = TYPES[dtype]
    gen = torch.Generator().manual_seed(n + R)
    k, v = (torch.randn(*s, generator=gen).to(dt) for s in ((n, R, Hk, DH), (L, n, R, Hk, DH)))
    ids = torch.randperm(n + 2, generator=gen)[:n].int()
    nrows = [(i * 5) % (R + 1) if R > 1 else 1 for i in range(n)]
    pos = [(i * 7) % (cap - nrows[i] + 1) for i in range(n)]
    codes, scales = cache(n + 2, Hk, L, cap, fill=0x5B)
    c0, s0 = codes.clone(), scales.clone()
    p = planes(codes, scales)
    status = torch.zeros(8, dtype=torch.int32, device=DEV)
    B.check(B.san_quant_append(p, code, k.to(DEV), v.to(DEV), ids.to(DEV), i32(pos), i32(nrows), n, R, status))
    back_k, back_v = torch.full_like(k, -9.0, device=DEV), torch.full_like(v, -9.0, device=DEV)
    B.check(B.san_quant_read(p, code, back_k, back_v, ids.to(DEV), i32(pos), i32(nrows), n, R, status))
    torch.cuda.synchronize()
    assert int(status[0]) == 0
    written = torch.zeros(codes.shape[:4], dtype=torch.bool)
    hc, hs = codes.cpu(), scales.cpu()
    for i in range(n):
        b = int(ids[i])
        written[:, b, :, pos[i]:pos[i] + nrows[i]] = True
        for y, x in enumerate([k, *v]):
            for r in range(nrows[i]):
                for h in range(Hk):
                    want, step, low = quantise_row(x[i, r, h].double().tolist())
                    assert hc[y, b, h, pos[i] + r].tolist() == pack(want) and hs[y, b, h, pos[i] + r].double().tolist() == [step, low]
    assert torch.equal(hc[~written], c0.cpu()[~written]) and torch.equal(hs[~written], s0.cpu()[~written])
    for y, got in enumerate([back_k.cpu(), *back_v.cpu()]):
        for i in range(n):
            a = pos[i]
            want = numbers(hc[y, int(ids[i]), :, a:a + nrows[i]], hs[y, int(ids[i]), :, a:a + nrows[i]]).transpose(0, 1)
            # float32: one rounding; bf16: that and its own
            assert bool(((got[i, :nrows[i]].double() - want).abs() <= want.abs() * (2.0 ** -24 + (2.0 ** -8 * 1.01 if dtype == "bf16" else 0))).all())
            assert bool((got[i, nrows[i]:] == -9.0).all())


def test_rows_bad_items_are_skipped_and_reported():
    gen = torch.Generator().manual_seed(1)
    k = torch.randn(4, 3, 2, DH, generator=gen).to(DEV)
    for call in (B.san_quant_append, B.san_quant_read):
        for ids, pos, nrows, bad in [([0, 9, 2, 3], [0] * 4, [3] * 4, (1, 9, 4)), ([0, 1, -1, 3], [0] * 4, [3] * 4, (2, -1, 4)),
                                     ([0, 1, 2, 3], [0, 0, 0, 8], [3] * 4, (3, 8, 10)), ([0, 1, 2, 3], [-1, 0, 0, 0], [3] * 4, (0, -1, 10)),
                                     ([0, 1, 2, 3], [0] * 4, [3, 4, 3, 3], (1, 4, 3)), ([0, 1, 2, 3], [0] * 4, [3, 3, -1, 3], (2, -1, 3)),
                                     ([0, 1, 2, 3], [0, 0, 0x7fffffff, 0], [3] * 4, (2, 0x7fffffff, 10))]:
            codes, scales = cache(4, 2, 1, 10, fill=0x11)
            out_k, out_v = k.clone().fill_(-9.0), k[None].clone().fill_(-9.0)
            status = torch.zeros(8, dtype=torch.int32, device=DEV)
            src = (k, k[None]) if call is B.san_quant_append else (out_k, out_v)
            B.check(call(planes(codes, scales), B.SAN_F32, *src, i32(ids), i32(pos), i32(nrows), 4, 3, status))
            torch.cuda.synchronize()
            assert status.tolist()[:5] == [B.SAN_ERR_DEVICE_CHECK, 14, *bad]
            good = [i for i in range(4) if i != bad[0]]
            if call is B.san_quant_append:
                assert bool((codes[:, [ids[i] for i in good], :, :3] != 0x11).any(-1).all())
                others = [b for b in range(4) if b not in [ids[i] for i in good]]
                assert bool((codes[:, others] == 0x11).all())
            else:
                assert bool((out_k[bad[0]] == -9.0).all()) and not bool((out_k[good] == -9.0).any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_wider_than_the_cache(dtype):
    """Buffers padded to more rows than the cache has: counts say what is real; more than the cache has room for is reported."""
    dt, code = TYPES[dtype]
    n, R, Hk, L, cap = 3, 70, 2, 2, 23
    gen = torch.Generator().manual_seed(9)
    k, v = (torch.randn(*s, generator=gen).to(dt).to(DEV) for s in ((n, R, Hk, DH), (L, n, R, Hk, DH)))
    ids, nrows = i32([2, 0, 1]), i32([23, 24, 11])
    codes, scales = cache(3, Hk, L, cap, fill=0x5B)
    p, status = planes(codes, scales), torch.zeros(8, dtype=torch.int32, device=DEV)
    B.check(B.san_quant_append(p, code, k, v, ids, None, nrows, n, R, status))
    back_k, back_v = torch.full_like(k, -9.0), torch.full_like(v, -9.0)
    B.check(B.san_quant_read(p, code, back_k, back_v, ids, None, nrows, n, R))
    torch.cuda.synchronize()
    assert status.tolist()[:5] == [B.SAN_ERR_DEVICE_CHECK, 14, 1, 0, 23]
    hc, hs = codes.cpu(), scales.cpu()
    assert bool((hc[:, 0] == 0x5B).all()) and bool((hc[:, 1, :, 11:] == 0x5B).all())
    for i, b, m in ((0, 2, 23), (2, 1, 11)):
        for y, x in enumerate([k.cpu(), *v.cpu()]):
            got = (back_k if y == 0 else back_v[y - 1])[i].cpu()
            for r in range(m):
                for h in range(Hk):
                    want, step, low = quantise_row(x[i, r, h].double().tolist())
                    assert hc[y, b, h, r].tolist() == pack(want) and hs[y, b, h, r].double().tolist() == [step, low]
            want = numbers(hc[y, b, :, :m], hs[y, b, :, :m]).transpose(0, 1)
            assert bool(((got[:m].double() - want).abs() <= want.abs() * (2.0 ** -24 + (2.0 ** -8 * 1.01 if dtype == "bf16" else 0))).all())
            assert bool((got[m:] == -9.0).all())
    assert bool((back_k[1] == -9.0).all()) and bool((back_v[:, 1] == -9.0).all())


# ------------------------------------------------------------------------------------------- attention
def filled(n_ids, Hk, L, cap, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    codes = torch.randint(0, 256, (1 + L, n_ids, Hk, cap, DH // 2), generator=gen, device=DEV, dtype=torch.uint8)
    step = 0.02 + 0.4 * torch.rand(1 + L, n_ids, Hk, cap, 1, generator=gen, device=DEV)
    low = -7.5 * step + torch.randn(1 + L, n_ids, Hk, cap, 1, generator=gen, device=DEV)
    return codes, torch.cat([step, low], -1).bfloat16()


def attention(codes, scales, q, ids, lens, dtype, weights=False, room=None, max_len=0, stream=None):
    n, H, L = q.shape[0], q.shape[1], codes.shape[0] - 1
    out = torch.full((L, n, H, DH), -7.0, dtype=q.dtype, device=DEV)
    S = torch.full((n, H, codes.shape[3] + 3), -5.0, device=DEV) if weights else None
    status = torch.zeros(8, dtype=torch.int32, device=DEV)
    p = planes(codes, scales)
    d_ids, d_lens = i32(ids), i32(lens)
    a = B.step_rows(dtype=TYPES[dtype][1], n_heads=H, d_q=q, d_ids=d_ids, d_lens=d_lens, n_items=n, max_len=max_len, d_S=S,
                    ld_s=codes.shape[3] + 3, d_out=out, d_status=status)
    rc, nb = B.san_quant_attn_bytes(p, a)
    B.check(rc)
    nb = nb if room is None else min(nb, room)
    ws = torch.full((max(nb, 256),), 0xAB, dtype=torch.uint8, device=DEV)
    B.check(B.san_quant_attn(p, a, ws, nb, stream))
    torch.cuda.synchronize()
    return out, S, status.tolist()


def check_items(out, S, codes, scales, q, ids, lens, skip=()):
    for i, (b, t) in enumerate(zip(ids, lens)):
        if i in skip:
            assert bool((out[:, i] == -7.0).all()) and (S is None or bool((S[i] == -5.0).all()))
            continue
        want, bound, p, p_bound = quant_attend(q[i], codes[:, b, :, :t], scales[:, b, :, :t], q.dtype)
        off = (out[:, i].double() - want).abs()
        bad = ~(off <= bound)
        assert not bool(bad.any()), (i, b, t, int(bad.sum()), float((off / bound).max()))
        if S is not None:
            off = (S[i, :, :t].double() - p).abs()
            assert bool((off <= p_bound).all()), (i, t, float((off / p_bound).max()))
            assert bool((S[i, :, t:] == -5.0).all())


CASES = [
    (1, 1, 1, 1, [1]), (1, 4, 4, 1, [60]), (3, 8, 2, 1, [0, 1, 2]), (4, 8, 8, 4, [63, 64, 65, 127]), (5, 12, 1, 3, [15, 16, 17, 128, 200]),
    (2, 20, 2, 9, [130, 77]), (1, 16, 4, 1, [5000]), (2, 6, 3, 5, [3001, 0]), (40, 8, 8, 2, [(i * 97) % 700 for i in range(40)]),
    (300, 2, 1, 1, [(i * 13) % 300 for i in range(300)]), (1, 1, 1, 2, [40001]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("n,H,Hk,L,lens", CASES)
def test_attention(n, H, Hk, L, lens, dtype, weights):
    gen = torch.Generator().manual_seed(n)
    codes, scales = filled(n + 1, Hk, L, max(lens) + 5, seed=n)
    ids = torch.randperm(n + 1, generator=gen)[:n].tolist()
    q = torch.randn(n, H, DH, generator=gen).to(TYPES[dtype][0]).to(DEV)
    for b, t in zip(ids, lens):                             # what lies behind the length does not matter
        scales[:, b, :, t:] = math.nan
    out, S, status = attention(codes, scales, q, ids, lens, dtype, weights)
    assert status[0] == 0
    check_items(out, S, codes, scales, q, ids, lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_items_of_one_id_and_a_bound(dtype):
    codes, scales = filled(2, 2, 2, 500, seed=4)
    ids, lens = [1, 1, 1, 0], [100, 220, 7, 333]
    q = torch.randn(4, 6, DH, generator=torch.Generator().manual_seed(5)).to(TYPES[dtype][0]).to(DEV)
    out, S, _ = attention(codes, scales, q, ids, lens, dtype, True, max_len=333)
    check_items(out, S, codes, scales, q, ids, lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("room", [0, 1, 3, 20])
def test_attention_with_less_workspace(dtype, room):
    """A workspace that has room for fewer partial results: rows are cut into fewer runs."""
    codes, scales = filled(2, 2, 2, 9000, seed=6)
    q = torch.randn(2, 4, DH, generator=torch.Generator().manual_seed(6)).to(TYPES[dtype][0]).to(DEV)
    for weights in (False, True):
        out, S, _ = attention(codes, scales, q, [1, 0], [9000, 6001], dtype, weights, room=256 + room * 8 * (8 + 2 * 256))
        check_items(out, S, codes, scales, q, [1, 0], [9000, 6001])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_large_and_small_numbers(dtype):
    """Steps over many magnitudes, scores far apart, rows far from zero."""
    codes, scales = filled(3, 1, 2, 300, seed=7)
    gen = torch.Generator().manual_seed(7)
    q = torch.randn(3, 4, DH, generator=gen)
    q[0] *= 30
    q[1] *= 1e-10
    q = q.to(TYPES[dtype][0]).to(DEV)
    scales[1, 0] *= 1e11
    scales[1, 1] *= 1e-12
    scales[2, 2, ..., 1] += 200
    scales[0, 2, ..., 0] = 0                                # rows of one number
    out, S, _ = attention(codes, scales, q, [0, 1, 2], [300, 299, 257], dtype, True)
    check_items(out, S, codes, scales, q, [0, 1, 2], [300, 299, 257])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_rows_and_queries_that_are_not_numbers(dtype):
    codes, scales = filled(4, 1, 2, 200, seed=8)
    q = torch.randn(4, 2, DH, generator=torch.Generator().manual_seed(8)).to(TYPES[dtype][0]).to(DEV)
    good, Sg, _ = attention(codes, scales, q, [0, 1, 2, 3], [150] * 4, dtype, True)
    scales[0, 0, :, 77] = math.nan                          # a key row of item 0
    scales[2, 1, :, 149] = math.nan                         # a value row of item 1, layer 1
    scales[:, 2, :, 150] = math.nan                         # behind item 2
    q[3, 1, 5] = math.inf                                   # one head of item 3
    out, S, _ = attention(codes, scales, q, [0, 1, 2, 3], [150] * 4, dtype, True)
    assert bool(out[:, 0].isnan().all()) and bool(S[0, :, :150].isnan().all())
    assert bool(out[1, 1].isnan().all()) and torch.equal(out[0, 1], good[0, 1]) and torch.equal(S[1], Sg[1])
    assert torch.equal(out[:, 2], good[:, 2]) and torch.equal(S[2], Sg[2])
    assert bool(out[:, 3, 1].isnan().all()) and torch.equal(out[:, 3, 0], good[:, 3, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_bad_items_are_skipped_and_reported(dtype):
    codes, scales = filled(3, 2, 1, 100, seed=9)
    q = torch.randn(3, 4, DH, generator=torch.Generator().manual_seed(9)).to(TYPES[dtype][0]).to(DEV)
    for ids, lens, bad in [([0, 3, 2], [9, 8, 7], (1, 3, 3)), ([-1, 1, 2], [9, 8, 7], (0, -1, 3)), ([0, 1, 2], [9, 8, 101], (2, 101, 100)),
                           ([0, 1, 2], [9, -2, 7], (1, -2, 100))]:
        out, S, status = attention(codes, scales, q, ids, lens, dtype, True)
        assert status[:5] == [B.SAN_ERR_DEVICE_CHECK, 13, *bad]
        check_items(out, S, codes, scales, q, ids, lens, skip=[bad[0]])


def test_attention_captured_replayed_and_beside_another_stream():
    """Two graphs with a workspace each, replayed at once, lengths changed between replays."""
    sets = []
    for seed, (n, H, Hk, L, t) in enumerate([(2, 8, 2, 2, 3000), (17, 4, 4, 3, 400)]):
        codes, scales = filled(n, Hk, L, t, seed=20 + seed)
        q = torch.randn(n, H, DH, generator=torch.Generator().manual_seed(seed)).bfloat16().to(DEV)
        out, S = torch.zeros(L, n, H, DH, dtype=torch.bfloat16, device=DEV), torch.full((n, H, t), -5.0, device=DEV)
        ids, lens = i32(list(range(n))[::-1]), i32([t] * n)
        p = planes(codes, scales)
        a = B.step_rows(dtype=B.SAN_BF16, n_heads=H, d_q=q, d_ids=ids, d_lens=lens, n_items=n, d_S=S, ld_s=t, d_out=out)
        nb = B.san_quant_attn_bytes(p, a)[1]
        ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            B.check(B.san_quant_attn(p, a, ws, nb))
        sets.append((graph, stream, codes, scales, q, out, S, lens, n, t, (ws, ids, a, p)))
    for turn in range(3):
        for graph, stream, codes, scales, q, out, S, lens, n, t, _ in sets:
            lens.copy_(i32([(t * 7 + i * 31 + turn * 13) % (t + 1) for i in range(n)]))
            S.fill_(-5.0)
        torch.cuda.synchronize()
        for _ in range(5):
            for graph, stream, *_ in sets:
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for graph, stream, codes, scales, q, out, S, lens, n, t, _ in sets:
            check_items(out, S, codes, scales, q, list(range(n))[::-1], lens.tolist())


def test_offsets_past_32_bits():
    """Planes of more than 4 GB: the last id of a cache whose value planes lie far apart."""
    cap, ids, L = 70000, 1000, 2
    codes = torch.empty((1 + L) * ids * cap * 32, dtype=torch.uint8, device=DEV).view(1 + L, ids, 1, cap, 32)
    scales = torch.zeros(1 + L, ids, 1, cap, 2, dtype=torch.bfloat16, device=DEV)
    c, s = filled(1, 1, L, cap, seed=30)
    codes[:, -1:], scales[:, -1:] = c, s
    q = torch.randn(1, 2, DH, generator=torch.Generator().manual_seed(30)).bfloat16().to(DEV)
    out, S, _ = attention(codes, scales, q, [ids - 1], [cap - 3], "bf16", True)
    check_items(out, S, codes, scales, q, [ids - 1], [cap - 3])
    k = torch.randn(1, 3, 1, DH, device=DEV)
    v = torch.randn(L, 1, 3, 1, DH, device=DEV)
    B.check(B.san_quant_append(planes(codes, scales), B.SAN_F32, k, v, i32([ids - 1]), i32([cap - 3]), None, 1, 3))
    back = torch.zeros_like(v)
    B.check(B.san_quant_read(planes(codes, scales), B.SAN_F32, k.clone(), back, i32([ids - 1]), i32([cap - 3]), None, 1, 3))
    torch.cuda.synchronize()
    want, step, low = quantise_row(v[1, 0, 2, 0].double().tolist())
    assert codes[2, -1, 0, -1].tolist() == pack(want) and scales[2, -1, 0, -1].double().tolist() == [step, low]
    assert float((back - v).abs().max()) <= float(scales[1:, -1, 0, -3:, 0].max()) / 2 * 1.001
