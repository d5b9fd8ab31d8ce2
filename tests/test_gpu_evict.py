"""Mass of cached rows (san_weight_mass) and eviction by it (san_cache_evict) against plain loops."""
import math

import pytest
import torch

from paper_1906_11024_b200 import binding as B
from paper_1906_11024_b200 import build as san_build
from tests.keep_helpers import DH, U32, keep
from tests.serve_helpers import to_planes

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    san_build.build()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------- mass
@pytest.mark.parametrize("layout", ["steps", "rows", "prompt"])
@pytest.mark.parametrize("n,H,Hk,R,lens,decay", [
    (1, 1, 1, 1, [1], 1.0), (3, 8, 2, 1, [0, 1, 300], 0.9), (2, 6, 3, 4, [257, 255], 0.0), (4, 4, 4, 40, [0, 31, 32, 40], 1.0),
    (2, 12, 1, 17, [513, 90], -0.5), (5, 2, 2, 200, [200, 1, 33, 199, 64], 0.99), (3, 8, 8, 0, [5, 6, 7], 0.5)])
def test_mass(n, H, Hk, R, lens, decay, layout):
    gen = torch.Generator().manual_seed(n + R)
    cap, ids = max(lens) + 3, torch.randperm(n + 2, generator=gen)[:n].tolist()
    mass = torch.rand(n + 2, Hk, cap + 2, generator=gen)
    if layout == "prompt":
        S = torch.rand(n, H, max(R, 1), cap, generator=gen)
        strides = (S.stride(0), S.stride(2), S.stride(1))
    else:
        S = torch.rand(n, max(R, 1), H, cap, generator=gen)
        strides = (S.stride(0), S.stride(1), S.stride(2))
    rows = None if layout == "steps" else [(i * 3) % (R + 1) for i in range(n)]
    begin = None if layout == "prompt" else [t // 2 if i % 2 else max(0, t - 1) for i, t in enumerate(lens)]
    want, bound = mass.double(), torch.zeros(mass.shape, dtype=torch.float64)
    for i, (b, t) in enumerate(zip(ids, lens)):
        count = R if rows is None else rows[i]
        x = (S[i, :, :count, :t] if layout == "prompt" else S[i, :count, :, :t].transpose(0, 1)).double()
        got = x.reshape(Hk, H // Hk * count, t).sum(1)
        old = want[b, :, :t].clone() * float(torch.tensor(decay, dtype=torch.float32))
        old[:, t if begin is None else begin[i]:] = 0
        want[b, :, :t] = old + got
        # a sum of k terms of one sign in any order, and the old mass, its product and the addition
        bound[b, :, :t] = U32 * ((H // Hk * count + 1) * got + 3 * (old.abs() + got)) + 1e-37
    # what is not read: positions behind a length, rows beyond an item's
    for i, t in enumerate(lens):
        S[i, ..., t:] = math.nan
        if rows is not None:
            (S[i, :, rows[i]:] if layout == "prompt" else S[i, rows[i]:]).fill_(math.nan)
    dm, dS, status = mass.to(DEV), S.to(DEV), torch.zeros(8, dtype=torch.int32, device=DEV)
    keepalive = [i32(ids), i32(lens), None if rows is None else i32(rows), None if begin is None else i32(begin)]
    B.check(B.san_weight_mass(B.mass_args(
        n_heads=H, n_kv_heads=Hk, d_S=dS, item_stride=strides[0], row_stride=strides[1], head_stride=strides[2], n_rows=R, d_rows=keepalive[2],
        d_ids=keepalive[0], d_lens=keepalive[1], d_begin=keepalive[3], n_items=n, max_len=cap, decay=decay, d_mass=dm, ld_mass=cap + 2,
        max_ids=n + 2, d_status=status)))
    torch.cuda.synchronize()
    assert int(status[0]) == 0
    assert bool(((dm.cpu().double() - want).abs() <= bound).all())


def test_mass_of_the_first_weights_does_not_look_at_the_old():
    """begin = 0: whatever was there, NaN among it, is replaced."""
    mass = torch.full((1, 2, 8), math.nan, device=DEV)
    S = torch.rand(1, 1, 4, 8, device=DEV)
    a = [i32([0]), i32([8]), i32([0])]
    B.check(B.san_weight_mass(B.mass_args(n_heads=4, n_kv_heads=2, d_S=S, item_stride=32, row_stride=32, head_stride=8, n_rows=1, d_ids=a[0],
                                          d_lens=a[1], d_begin=a[2], n_items=1, max_len=8, decay=1.0, d_mass=mass, ld_mass=8, max_ids=1)))
    torch.cuda.synchronize()
    assert torch.allclose(mass[0], S.view(2, 2, 8).sum(1), rtol=2.0 ** -22)


@pytest.mark.parametrize("n_rows", [1, 64])
def test_mass_bad_items_are_skipped_and_reported(n_rows):
    for ids, lens, rows, begin, bad in [([0, 3, 2], [5, 6, 7], [1] * 3, [0] * 3, (1, 3, 3)), ([0, 1, 2], [5, 9, 7], [1] * 3, [0] * 3, (1, 9, 8)),
                                        ([0, 1, 2], [5, 6, -1], [1] * 3, [0] * 3, (2, -1, 8)), ([0, 1, 2], [5, 6, 7], [n_rows + 1, 1, 1], [0] * 3, (0, n_rows + 1, n_rows)),
                                        ([0, 1, 2], [5, 6, 7], [1] * 3, [0, 7, 0], (1, 7, 6)), ([0, 1, 2], [5, 6, 7], [1] * 3, [0, 0, -1], (2, -1, 7))]:
        mass, S = torch.full((3, 2, 8), -3.0, device=DEV), torch.rand(3, n_rows, 2, 8, device=DEV)
        status, a = torch.zeros(8, dtype=torch.int32, device=DEV), [i32(x) for x in (ids, lens, rows, begin)]
        B.check(B.san_weight_mass(B.mass_args(n_heads=2, n_kv_heads=2, d_S=S, item_stride=16 * n_rows, row_stride=16, head_stride=8, n_rows=n_rows,
                                              d_rows=a[2], d_ids=a[0], d_lens=a[1], d_begin=a[3], n_items=3, max_len=8, decay=1.0, d_mass=mass,
                                              ld_mass=8, max_ids=3, d_status=status)))
        torch.cuda.synchronize()
        assert status.tolist()[:5] == [B.SAN_ERR_DEVICE_CHECK, 15, *bad]
        touched = {ids[i] for i in range(3) if i != bad[0]}
        for b in range(3):
            assert bool((mass[b, :, :5] >= 0).all()) if b in touched else bool((mass[b] == -3.0).all())


# ------------------------------------------------------------------------------------------- eviction
def masses(kind, gen, n, Hk, cap):
    if kind == "random":
        return torch.exp(torch.randn(n, Hk, cap, generator=gen) * 2)
    if kind == "ties":
        return torch.randint(0, 4, (n, Hk, cap), generator=gen).float() * 0.25
    if kind == "equal":
        return torch.full((n, Hk, cap), 0.125)
    if kind == "odd":                                       # both zeros, infinities, NaN, numbers of both signs, denormals
        pool = torch.tensor([0.0, -0.0, math.inf, -math.inf, math.nan, 1.0, -1.0, 1e-40, -1e-40, 3e38])
        return pool[torch.randint(0, len(pool), (n, Hk, cap), generator=gen)]
    return torch.arange(cap).float().flip(0).repeat(n, Hk, 1)      # falling: the first ones stay, nothing moves but the recent


def stored(fmt, gen, L, n, Hk, cap):
    """Planes with every element distinct enough, in the cache's layout, and a function that gives rows in order."""
    if fmt == "q4":
        codes = torch.randint(0, 256, (1 + L, n, Hk, cap, 32), generator=gen, dtype=torch.uint8)
        scales = torch.randn(1 + L, n, Hk, cap, 2, generator=gen).bfloat16()
        return [codes, scales]
    return [torch.randn(1 + L, n, Hk, cap, DH, generator=gen).to(torch.bfloat16 if fmt == "bf16" else torch.float32)]


def planes_of(fmt, x):
    ids, Hk, cap = x[0].shape[1:4]
    kw = dict(d_k_scale=x[1][0], d_v_scale=x[1][1:]) if fmt == "q4" else {}
    code = {"q4": B.SAN_Q4, "bf16": B.SAN_BF16, "f32": B.SAN_F32}[fmt]
    return B.planes(dtype=code, n_kv_heads=Hk, n_layers=x[0].shape[0] - 1, d_k=x[0][0], d_v=x[0][1:], v_stride=ids * Hk * cap * DH, max_ids=ids,
                    cap_len=cap, **kw)


def evict(fmt, rows, mass, ids, lens, n_keep, sink, recent, with_kept=True, in_place=False, max_len=0, stream=None):
    """Runs the call on copies; returns rows, mass, lens, kept, status."""
    dev = [(to_planes(x) if fmt == "bf16" else x).to(DEV) for x in rows]
    dm, n, Hk = mass.to(DEV), len(ids), mass.shape[1]
    d_ids, d_lens = i32(ids), i32(lens)
    out = d_lens if in_place else torch.full((n,), -9, dtype=torch.int32, device=DEV)
    kept = torch.full((n, Hk, n_keep + 1), -9, dtype=torch.int32, device=DEV) if with_kept else None
    status = torch.zeros(8, dtype=torch.int32, device=DEV)
    p = planes_of(fmt, dev)
    a = B.evict_args(d_ids=d_ids, d_lens=d_lens, n_items=n, max_len=max_len, n_keep=n_keep, n_sink=sink, n_recent=recent, d_mass=dm,
                     ld_mass=mass.shape[2], d_kept=kept, ld_kept=n_keep + 1, d_lens_out=out, d_status=status)
    rc, nb = B.san_cache_evict_bytes(p, a)
    B.check(rc)
    ws = torch.full((nb + 64,), 0xAB, dtype=torch.uint8, device=DEV)
    B.check(B.san_cache_evict(p, a, ws, nb, stream))
    torch.cuda.synchronize()
    assert bool((ws[nb:] == 0xAB).all())
    return dev, dm, out, kept, status.tolist()


def check(fmt, rows, mass, ids, lens, n_keep, sink, recent, got, skip=()):
    dev, dm, out, kept, _ = got
    want = [x.clone() for x in rows]
    wm = mass.clone()
    for i, (b, t) in enumerate(zip(ids, lens)):
        if i in skip:
            continue
        assert int(out[i]) == min(t, n_keep)
        for h in range(mass.shape[1]):
            at = keep(mass[b, h, :t].tolist(), t, n_keep, sink, recent)
            if kept is not None:
                assert kept[i, h].tolist() == at + [-9] * (n_keep + 1 - len(at)), (i, h)
            if t <= n_keep:
                continue
            wm[b, h, :n_keep] = mass[b, h, at]
            for x, y in zip(want, rows):
                x[:, b, h, :n_keep] = y[:, b, h, at]
    for x, y in zip(want, dev):
        x = to_planes(x) if fmt == "bf16" else x
        view = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()]
        assert torch.equal(x.view(view), y.cpu().view(view))
    assert torch.equal(wm.view(torch.int32), dm.cpu().view(torch.int32))


EVICT = [(1, 1, 1, 30, 10, 0, 0, [30]), (3, 2, 2, 40, 12, 3, 4, [40, 12, 13]), (4, 3, 1, 70, 64, 0, 64, [70, 0, 65, 63]), (2, 1, 3, 300, 299, 1, 2, [300, 299]),
         (2, 2, 1, 1500, 700, 64, 100, [1500, 1023]), (1, 2, 5, 3500, 1024, 4, 0, [3400]), (2, 1, 1, 2100, 5, 2, 3, [2100, 2048]), (1, 1, 1, 2, 1, 0, 0, [2])]


@pytest.mark.parametrize("fmt", ["q4", "bf16", "f32"])
@pytest.mark.parametrize("kind", ["random", "ties", "equal", "odd", "falling"])
@pytest.mark.parametrize("n,Hk,L,cap,n_keep,sink,recent,lens", EVICT)
def test_evict(n, Hk, L, cap, n_keep, sink, recent, lens, kind, fmt):
    gen = torch.Generator().manual_seed(cap)
    ids = torch.randperm(n + 1, generator=gen)[:n].tolist()
    rows, mass = stored(fmt, gen, L, n + 1, Hk, cap), masses(kind, gen, n + 1, Hk, cap)
    got = evict(fmt, rows, mass, ids, lens, n_keep, sink, recent, with_kept=cap != 300, in_place=cap == 40)
    assert got[4][0] == 0
    check(fmt, rows, mass, ids, lens, n_keep, sink, recent, got)


@pytest.mark.parametrize("fmt", ["q4", "bf16"])
@pytest.mark.parametrize("kind", ["random", "ties", "odd"])
@pytest.mark.parametrize("lens,n_keep", [([49999], 20000), ([16384, 4097], 4096), ([4096, 4095], 1500), ([16385], 16384)])
def test_evict_long(fmt, kind, lens, n_keep):
    """The bounds at which rows are chosen another way, and one row past them."""
    gen = torch.Generator().manual_seed(1)
    n, cap = len(lens), max(lens) + 1
    rows, mass = stored(fmt, gen, 1, n, 2, cap), masses(kind, gen, n, 2, cap)
    got = evict(fmt, rows, mass, list(range(n)), lens, n_keep, 4, 1000, max_len=max(lens))
    check(fmt, rows, mass, list(range(n)), lens, n_keep, 4, 1000, got)


def test_evict_two_streams_with_workspaces_of_their_own():
    gen = torch.Generator().manual_seed(9)
    sets = []
    for fmt, n, Hk, L, cap, n_keep in (("bf16", 9, 4, 3, 700, 300), ("q4", 2, 2, 1, 5000, 2000)):
        rows, mass = stored(fmt, gen, L, n, Hk, cap), masses("random", gen, n, Hk, cap)
        dev = [(to_planes(x) if fmt == "bf16" else x).to(DEV) for x in rows]
        lens = [cap - 7 * i for i in range(n)]
        dm, ids, dl, out = mass.to(DEV), i32(list(range(n))), i32(lens), torch.zeros(n, dtype=torch.int32, device=DEV)
        p = planes_of(fmt, dev)
        a = B.evict_args(d_ids=ids, d_lens=dl, n_items=n, n_keep=n_keep, n_sink=2, n_recent=9, d_mass=dm, ld_mass=cap, d_lens_out=out)
        nb = B.san_cache_evict_bytes(p, a)[1]
        sets.append((p, a, torch.empty(nb, dtype=torch.uint8, device=DEV), nb, torch.cuda.Stream(), (fmt, rows, mass, list(range(n)), lens, n_keep, 2, 9), dev, dm, out, ids, dl))
    torch.cuda.synchronize()
    for p, a, ws, nb, stream, *_ in sets:
        B.check(B.san_cache_evict(p, a, ws, nb, stream))
    torch.cuda.synchronize()
    for *_, about, dev, dm, out, ids, dl in sets:
        check(*about, (dev, dm, out, None, None))


@pytest.mark.parametrize("fmt", ["q4", "bf16", "f32"])
def test_evict_bad_items_are_skipped_and_reported(fmt):
    gen = torch.Generator().manual_seed(2)
    rows, mass = stored(fmt, gen, 2, 3, 2, 50), masses("random", gen, 3, 2, 50)
    for ids, lens, bad in [([0, 3, 2], [50, 40, 30], (1, 3, 3)), ([0, -5, 2], [50, 40, 30], (1, -5, 3)), ([0, 1, 2], [50, 51, 30], (1, 51, 50)),
                           ([0, 1, 2], [50, -1, 30], (1, -1, 50))]:
        got = evict(fmt, rows, mass, ids, lens, 20, 1, 5)
        assert got[4][:5] == [B.SAN_ERR_DEVICE_CHECK, 16, *bad]
        assert int(got[2][1]) == -9 and bool((got[3][1] == -9).all())
        check(fmt, rows, mass, ids, lens, 20, 1, 5, got, skip=[1])


def test_evict_captured_and_replayed():
    """A step's eviction in a graph: lengths and masses change, the graph does not."""
    gen = torch.Generator().manual_seed(3)
    n, Hk, L, cap, k = 6, 2, 2, 200, 90
    rows = stored("bf16", gen, L, n, Hk, cap)
    dev = [to_planes(x).to(DEV) for x in rows]
    start = [x.clone() for x in dev]
    dm, ids, lens, out = torch.zeros(n, Hk, cap, device=DEV), i32(list(range(n))), i32([cap] * n), i32([0] * n)
    p = planes_of("bf16", dev)
    a = B.evict_args(d_ids=ids, d_lens=lens, n_items=n, n_keep=k, n_sink=2, n_recent=20, d_mass=dm, ld_mass=cap, d_lens_out=out)
    nb = B.san_cache_evict_bytes(p, a)[1]
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        B.check(B.san_cache_evict(p, a, ws, nb))
    for turn in range(3):
        mass, t = masses("ties" if turn else "random", gen, n, Hk, cap), [(i * 53 + turn * 31) % (cap + 1) for i in range(n)]
        dm.copy_(mass)
        lens.copy_(i32(t))
        for x, y in zip(dev, start):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        check("bf16", rows, mass, list(range(n)), t, k, 2, 20, (dev, dm, out, None, None))


def test_evict_offsets_past_32_bits():
    cap, ids = 20000, 2000                                  # a plane of 5 GB
    dev = torch.zeros(2, ids, 1, cap, DH, dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator().manual_seed(4)
    rows = stored("bf16", gen, 1, 1, 1, cap)
    dev[:, -1:] = to_planes(rows[0]).to(DEV)
    mass = masses("random", gen, ids, 1, cap)
    dm, a = mass.to(DEV), [i32([ids - 1]), i32([cap])]
    p = planes_of("bf16", [dev])
    e = B.evict_args(d_ids=a[0], d_lens=a[1], n_items=1, n_keep=5000, n_sink=4, n_recent=50, d_mass=dm, ld_mass=cap, d_lens_out=a[1])
    nb = B.san_cache_evict_bytes(p, e)[1]
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    B.check(B.san_cache_evict(p, e, ws, nb))
    torch.cuda.synchronize()
    at = keep(mass[-1, 0].tolist(), cap, 5000, 4, 50)
    assert int(a[1][0]) == 5000 and torch.equal(dev[:, -1, 0, :5000].cpu(), to_planes(rows[0][:, :, :, at])[:, 0, 0])


@pytest.mark.parametrize("R", [1, 40])
def test_mass_without_a_bound(R):
    """max_len 0: whatever the mass holds; a longer length is reported."""
    n, H, Hk, ld = 3, 4, 2, 70
    S = torch.rand(n, R, H, ld, device=DEV)
    mass = torch.rand(n, Hk, ld, device=DEV)
    old, lens = mass.clone(), [70, 71, 33]
    status, a = torch.zeros(8, dtype=torch.int32, device=DEV), [i32([2, 0, 1]), i32(lens)]
    B.check(B.san_weight_mass(B.mass_args(n_heads=H, n_kv_heads=Hk, d_S=S, item_stride=R * H * ld, row_stride=H * ld, head_stride=ld, n_rows=R,
                                          d_ids=a[0], d_lens=a[1], n_items=n, max_len=0, decay=1.0, d_mass=mass, ld_mass=ld, max_ids=n, d_status=status)))
    torch.cuda.synchronize()
    assert status.tolist()[:5] == [B.SAN_ERR_DEVICE_CHECK, 15, 1, 71, 70]
    want, bound = old.double(), torch.zeros(n, Hk, ld, dtype=torch.float64, device=DEV)
    for i, b in ((0, 2), (2, 1)):
        t = lens[i]
        got = S[i, :, :, :t].double().view(R, Hk, H // Hk, t).sum((0, 2))
        want[b, :, :t] += got
        # terms of one sign in any order, the old mass and the addition
        bound[b, :, :t] = U32 * ((H // Hk * R + 1) * got + 3 * (old[b, :, :t] + got)) + 1e-37
    assert bool(((mass.double() - want).abs() <= bound).all())
