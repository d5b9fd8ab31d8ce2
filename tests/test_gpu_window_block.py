"""Windowed attention of whole sequences (san_window_block) against the rows that each query sees, in 64 bits."""
import pytest
import torch

from paper_1906_11024_b200 import binding as B
from paper_1906_11024_b200 import build as san_build
from tests.serve_helpers import DH, attend, check_outputs, randn, weighted_size

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    san_build.build()
    B.lib()


def _reference(q, k, v, window, sink):
    """q [l][64], k [l][64], v [L][l][64] in 64 bits -> outputs, slack and weighted sizes [L][l][64]."""
    l = q.shape[0]
    a, b = torch.arange(l)[:, None], torch.arange(l)[None, :]
    seen = (b <= a) & ((b > a - window) | (b < sink))
    z = (q @ k.T / 8.0).masked_fill(~seen, -float("inf"))
    p = torch.softmax(z, -1)
    size = p @ v.abs()
    # as in serve_helpers.attend, the largest score error of any pair
    dz = 70 * 2.0 ** -24 * float((q.abs() @ k.abs().T).max()) / 8.0
    return p @ v, size * (4 * dz + 2.0 ** -20 + 2 * l * 2.0 ** -24), size


def _run(lens, cap, H, Hk, L, window, sink, max_len=0, seed=0, spoil=None, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    n = len(lens)
    q, k = randn(gen, n, cap, H, DH, dtype=torch.bfloat16), randn(gen, n, cap, Hk, DH, dtype=torch.bfloat16)
    v = randn(gen, L, n, cap, Hk, DH, dtype=torch.bfloat16)
    q *= scale
    dq, dk, dv = (x.clone() for x in (q, k, v))
    for i, t in enumerate(lens):                                # behind the end of a sequence: NaN
        dq[i, t:], dk[i, t:] = float("nan"), float("nan")
        dv[:, i, t:] = float("nan")
    if spoil:
        spoil(dk, dv)
    dq, dk, dv = (x.to(DEV) for x in (dq, dk, dv))
    out = torch.full((L, n, cap, H, DH), -7.0, dtype=torch.bfloat16, device=DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    B.check(B.san_window_block(B.SAN_BF16, H, Hk, L, window, sink, dq, dk, dv, dl, n, cap, max_len, out))
    torch.cuda.synchronize()
    got = out.cpu()
    return q, k, v, got


def _check(q, k, v, got, lens, window, sink, skip=lambda i: ()):
    L, n, cap, H = got.shape[:4]
    r = H // k.shape[2]
    for i, t in enumerate(lens):
        assert (got[:, i, t:] == -7.0).all(), i
        rows = [a for a in range(t) if a not in set(skip(i))]
        if not rows:
            continue
        for h in range(H):
            want, slack, size = _reference(q[i, :t, h].double(), k[i, :t, h // r].double(), v[:, i, :t, h // r].double(), window, sink)
            check_outputs(got[:, i, rows, h], want[:, rows], slack[:, rows], size[:, rows], torch.bfloat16, (i, h))


@pytest.mark.parametrize("lens,cap,H,Hk,L,window,sink", [
    ([1], 1, 1, 1, 1, 1, 0),
    ([1, 2, 15, 16, 17, 63, 64, 65, 0, 80, 33], 80, 2, 2, 3, 16, 1),
    ([130, 128, 127, 1], 131, 2, 1, 2, 1, 0),                   # a window of one row
    ([200, 190], 200, 3, 3, 1, 64, 4),
    ([200, 190], 200, 4, 2, 2, 65, 5),
    ([300, 129], 300, 2, 2, 2, 1000000000, 0),                    # causal
    ([513, 400], 520, 1, 1, 5, 100, 130),                       # more sinks than a tile
    ([1000], 1000, 2, 1, 1, 257, 3),
    ([700], 700, 1, 1, 2, 33, 64),
])
def test_lengths_windows_sinks(lens, cap, H, Hk, L, window, sink):
    q, k, v, got = _run(lens, cap, H, Hk, L, window, sink, seed=cap)
    _check(q, k, v, got, lens, window, sink)


@pytest.mark.parametrize("L", [1, 5])
@pytest.mark.parametrize("window,sink", [(1, 32), (7, 3), (29, 4), (30, 4), (33, 0), (34, 0)])
def test_small_windows_of_long_sequences(window, sink, L):
    """Both sides of the size from which a window's rows no longer fit one slot."""
    lens, cap, H, Hk = [700, 1, 333], 705, 4, 2
    q, k, v, got = _run(lens, cap, H, Hk, L, window, sink, seed=window)
    _check(q, k, v, got, lens, window, sink)


@pytest.mark.parametrize("window,sink", [(100, 2 ** 31 - 1), (1, 2 ** 31 - 63), (100, 2 ** 31 - 64), (2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("lens,cap", [([100, 1, 37], 100), ([700, 128, 513, 1], 703)])
def test_sinks_and_windows_up_to_the_largest_number(lens, cap, window, sink):
    """More sinks, or a longer window, than there are rows: all of them are seen, by the tiles and below their length."""
    q, k, v, got = _run(lens, cap, 2, 1, 2, window, sink, seed=cap)
    _check(q, k, v, got, lens, window, sink)


def test_equals_the_causal_full_sequence_call():
    """A window over everything is san_full_block's causal form."""
    lens, cap, H, L = [150, 77], 150, 2, 2
    q, k, v, got = _run(lens, cap, H, H, L, cap, 0)
    dq, dk, dv = (x.to(DEV) for x in (q, k, v))
    out = torch.full_like(got, -7.0).to(DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    B.check(B.san_full_block(B.SAN_BF16, H, L, 1, dq, dk, dv, dl, 2, cap, 0, None, 0, out))
    torch.cuda.synchronize()
    a, b = got.double(), out.cpu().double()
    assert (a - b).norm() <= 2.0 ** -7 * b.norm()               # each within half a step twice


def test_host_bound_cuts_longer_sequences():
    lens, cap = [96, 50], 96
    q, k, v, got = _run(lens, cap, 2, 2, 2, 20, 2, max_len=64)
    _check(q, k, v, got, [64, 50], 20, 2)


@pytest.mark.parametrize("what", ["nan", "inf"])
def test_what_a_row_does_not_see_does_not_reach_it(what):
    """One spoilt key and value row: rows that see it come out as its values demand, the others as if it were not there."""
    bad, window, sink, lens = 70, 40, 2, [200]

    def spoil(dk, dv):
        dv[:, 0, bad] = float(what)
        if what == "nan":
            dk[0, bad] = float("nan")

    q, k, v, got = _run(lens, 200, 2, 2, 2, window, sink, spoil=spoil)
    sees = list(range(bad, bad + window))
    _check(q, k, v, got, lens, window, sink, skip=lambda i: sees)
    assert not torch.isfinite(got[:, 0, sees]).any()


@pytest.mark.parametrize("what", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("lens,H,Hk,L,window,sink,bad", [
    ([700, 300], 2, 1, 2, 100, 4, [1]),                         # a sink: every row behind it sees it
    ([700, 300], 2, 2, 3, 100, 4, [2, 290, 299]),
    ([1100], 1, 1, 1, 300, 0, [0, 129, 640, 1099]),
    ([600], 4, 2, 2, 600, 0, [255, 256]),                       # causal
    ([520], 1, 1, 1, 40, 70, [69, 70, 480]),                    # sinks that end inside a chunk
    ([100, 60], 2, 1, 3, 20, 2, [1, 50]),                       # below the tiles
])
def test_single_bad_values(what, lens, H, Hk, L, window, sink, bad):
    """One element of some value rows of the last layer: its column alone, of the rows that see it alone, is no number."""
    cap, col = max(lens), 5

    def spoil(dk, dv):
        dv[L - 1, :, bad, :, col] = float(what)
        for i, t in enumerate(lens):
            dv[:, i, t:] = float("nan")

    q, k, v, got = _run(lens, cap, H, Hk, L, window, sink, spoil=spoil)
    v[L - 1, :, bad, :, col] = 0.0
    for i, t in enumerate(lens):
        hit = [a for a in range(t) if any(b <= a and (b > a - window or b < sink) for b in bad)]
        rest = torch.ones(t, dtype=torch.bool)
        rest[hit] = False
        assert not torch.isfinite(got[L - 1, i, hit][..., col]).any() and torch.isfinite(got[L - 1, i, :t][rest][..., col]).all()
        got[L - 1, i, hit, :, col] = 0.0
        r = H // Hk
        for h in range(H):
            want, slack, size = _reference(q[i, :t, h].double(), k[i, :t, h // r].double(), v[:, i, :t, h // r].double(), window, sink)
            want[L - 1, hit, col] = 0.0
            check_outputs(got[:, i, :t, h], want, slack, size, torch.bfloat16, (i, h))


@pytest.mark.parametrize("row", [0, 3000])
def test_one_bad_value_costs_little(row):
    """A NaN in one value of a long prompt, seen by thousands of rows: some 1 ms at most (0.1 without), a hundred of them are
    allowed here."""
    n, cap, H = 1, 8192, 8
    gen = torch.Generator(device=DEV).manual_seed(3)
    mk = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(torch.bfloat16)        # noqa: E731
    q, k, v = mk(n, cap, H, DH), mk(n, cap, H, DH), mk(1, n, cap, H, DH)
    v[:, :, row, :, 9] = float("nan")
    out = torch.zeros(1, n, cap, H, DH, dtype=torch.bfloat16, device=DEV)
    dl = torch.tensor([cap], dtype=torch.int32, device=DEV)
    call = lambda: B.check(B.san_window_block(B.SAN_BF16, H, H, 1, cap, 0, q, k, v, dl, n, cap, 0, out))     # noqa: E731
    call()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    call()
    end.record()
    torch.cuda.synchronize()
    bad = torch.isnan(out)
    assert bad[:, :, row:, :, 9].all() and int(bad.sum()) == (cap - row) * H
    assert begin.elapsed_time(end) < 100


def test_inputs_full_of_nan():
    """Every row comes out as NaN, and soon: 2000 rows of a causal prompt."""
    n, cap, H = 1, 2000, 2
    x = torch.full((n, cap, H, DH), float("nan"), dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(1, n, cap, H, DH, dtype=torch.bfloat16, device=DEV)
    dl = torch.tensor([cap], dtype=torch.int32, device=DEV)
    ok = torch.randn(n, cap, H, DH, device=DEV).to(torch.bfloat16)
    for q, k, v in ((x, ok, ok), (ok, x, ok), (ok, ok, x)):
        B.check(B.san_window_block(B.SAN_BF16, H, H, 1, cap, 0, q, k, v[None].contiguous(), dl, n, cap, 0, out))
        torch.cuda.synchronize()
        assert torch.isnan(out).all()


def test_scores_that_keep_growing():
    """The running maximum moves by more than 2^8 from chunk to chunk: outputs are scaled."""
    gen = torch.Generator().manual_seed(8)
    l, H = 700, 2
    q, k, v = (randn(gen, 1, l, H, DH, dtype=torch.bfloat16) for _ in range(3))
    k *= torch.linspace(0.1, 60.0, l)[None, :, None, None].to(torch.bfloat16)
    out = torch.full((2, 1, l, H, DH), -7.0, dtype=torch.bfloat16, device=DEV)
    vv = torch.stack([v, -v])
    dq, dk, dv = q.to(DEV), k.to(DEV), vv.to(DEV)
    dl = torch.tensor([l], dtype=torch.int32, device=DEV)
    B.check(B.san_window_block(B.SAN_BF16, H, H, 2, 400, 2, dq, dk, dv, dl, 1, l, 0, out))
    torch.cuda.synchronize()
    _check(q, k, vv, out.cpu(), [l], 400, 2)


def test_scores_in_the_thousands():
    lens = [140]
    q, k, v, got = _run(lens, 140, 1, 1, 1, 50, 4, scale=512.0)
    _check(q, k, v, got, lens, 50, 4)


def test_captured_and_replayed():
    lens, cap, H = [100, 64], 100, 2
    gen = torch.Generator().manual_seed(1)
    mk = lambda *s: randn(gen, *s, dtype=torch.bfloat16)        # noqa: E731
    k, v = mk(2, cap, H, DH), mk(1, 2, cap, H, DH)
    dq, dk, dv = torch.zeros(2, cap, H, DH, dtype=torch.bfloat16, device=DEV), k.to(DEV), v.to(DEV)
    out = torch.full((1, 2, cap, H, DH), -7.0, dtype=torch.bfloat16, device=DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    call = lambda: B.check(B.san_window_block(B.SAN_BF16, H, H, 1, 30, 3, dq, dk, dv, dl, 2, cap, 0, out))     # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(2):
        q = mk(2, cap, H, DH)
        dq.copy_(q)
        g.replay()
        torch.cuda.synchronize()
        _check(q, k, v, out.cpu(), lens, 30, 3)


@pytest.mark.parametrize("window,sink", [(100, 3), (20, 2)])
def test_far_rows_of_large_arrays(window, sink):
    """Byte offsets beyond 32 bits in every array, by the tiles and by the kernel for small windows: the last sequence's last
    rows, of the last layer too."""
    n, cap, H, Hk, L = 3, 100000, 64, 32, 2             # queries and outputs 2.5 GB a layer, keys and values 1.2
    gen = torch.Generator(device=DEV).manual_seed(5)
    mk = lambda *s: torch.randn(*s, generator=gen, device=DEV, dtype=torch.bfloat16)        # noqa: E731
    q, k, v = mk(n, cap, H, DH), mk(n, cap, Hk, DH), mk(L, n, cap, Hk, DH)
    out = torch.full((L, n, cap, H, DH), -7.0, dtype=torch.bfloat16, device=DEV)
    lens = [1, 0, cap]
    B.check(B.san_window_block(B.SAN_BF16, H, Hk, L, window, sink, q, k, v, torch.tensor(lens, dtype=torch.int32, device=DEV), n, cap, 0, out))
    torch.cuda.synchronize()
    assert (out[:, 1] == -7.0).all() and (out[:, 0, 1:] == -7.0).all()
    begin = cap - window - 200                          # rows whose windows are within the copied part
    part = torch.cat([torch.arange(sink), torch.arange(begin, cap)])
    kk, vv = k[2, part].cpu().double(), v[:, 2, part].cpu().double()
    for a in (cap - 1, cap - 2, cap - 64, cap - 200):
        for h in (0, 31, 63):
            pos = [i for i in range(len(part)) if part[i] <= a and (part[i] > a - window or part[i] < sink)]
            assert len(pos) == window + sink
            qq = q[2, a, h].cpu().double()
            want, slack = attend(qq, kk[pos, h // 2], vv[:, pos, h // 2])
            check_outputs(out[:, 2, a, h].cpu(), want, slack, weighted_size(qq, kk[pos, h // 2], vv[:, pos, h // 2]), torch.bfloat16, (a, h))


def test_on_another_stream_behind_its_inputs():
    lens, cap, H, window, sink = [300, 41], 300, 2, 90, 2
    gen = torch.Generator().manual_seed(6)
    q, k, v = (randn(gen, *s, cap, H, DH, dtype=torch.bfloat16) for s in ((2,), (2,), (1, 2)))
    side = torch.cuda.Stream()
    dq, dk, dv = (x.to(DEV) for x in (q, k, v))
    out = torch.full((1, 2, cap, H, DH), -7.0, dtype=torch.bfloat16, device=DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                       # the current stream is the one that is taken
        B.check(B.san_window_block(B.SAN_BF16, H, H, 1, window, sink, dq, dk, dv, dl, 2, cap, 0, out))
    side.synchronize()
    _check(q, k, v, out.cpu(), lens, window, sink)
