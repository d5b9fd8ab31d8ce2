"""Step attention over sliding windows (san_window_attn) and behind shared prefixes (san_prefix_attn) against the
rows that are seen, one after the other, in 64 bits."""
import numpy as np
import pytest
import torch

from paper_1906_11024_b200 import binding as B
from paper_1906_11024_b200 import build as san_build
from tests.serve_helpers import DH, attend, check_outputs, dtype_of, randn, to_planes, weighted_size

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    san_build.build()
    B.lib()


class Rows:
    """Query rows and own cached rows; what lies behind a sequence's end is NaN."""

    def __init__(self, dtype, lens, H, Hk, L, cap, seed=0, spare=2):
        self.dt, self.code = dtype_of(dtype)
        gen = torch.Generator().manual_seed(seed)
        n = len(lens)
        self.lens, self.H, self.Hk, self.L, self.cap = list(lens), H, Hk, L, cap
        self.q = randn(gen, n, H, DH, dtype=self.dt)
        self.ids = torch.randperm(n + spare, generator=gen)[:n].to(torch.int32)
        self.k = randn(gen, n + spare, Hk, cap, DH, dtype=self.dt)
        self.v = randn(gen, L, n + spare, Hk, cap, DH, dtype=self.dt)
        pk, pv = to_planes(self.k), to_planes(self.v)
        self.hidden = torch.ones(n + spare, cap, dtype=torch.bool)
        for i, t in enumerate(lens):
            self.hidden[self.ids[i], :max(0, min(t, cap))] = False
        pk.masked_fill_(self.hidden[:, None, :, None], float("nan"))
        pv.masked_fill_(self.hidden[None, :, None, :, None], float("nan"))
        self.d = [x.to(DEV) for x in (self.q, pk, pv, self.ids, torch.tensor(self.lens, dtype=torch.int32))]
        self.out = torch.full((L, n, H, DH), -7.0, dtype=self.dt, device=DEV)
        self.status = torch.zeros(8, dtype=torch.int32, device=DEV)

    def args(self, max_len=0, **kw):
        q, k, v, ids, lens = self.d
        return B.cached_rows(**(dict(dtype=self.code, n_heads=self.H, n_kv_heads=self.Hk, n_layers=self.L, d_q=q, d_k=k, d_v=v,
                                     v_stride=v[0].numel(), max_ids=k.shape[0], cap_len=self.cap, d_ids=ids, d_lens=lens,
                                     n_items=q.shape[0], max_len=max_len, d_out=self.out, d_status=self.status) | kw))

    def check(self, seen, extra=None, skip=()):
        """seen(i): own positions that row i sees; extra(i, hk): keys and values [L] in front of them."""
        got = self.out.cpu()
        for i in range(len(self.lens)):
            if i in skip:
                assert (got[:, i] == -7.0).all(), i
                continue
            pos = torch.as_tensor(seen(i), dtype=torch.long)
            for h in range(self.H):
                hk = h // (self.H // self.Hk)
                k, v = self.k[self.ids[i], hk, pos].double(), self.v[:, self.ids[i], hk, pos].double()
                if extra is not None:
                    ek, ev = extra(i, hk)
                    k, v = torch.cat([ek, k]), torch.cat([ev, v], 1)
                q = self.q[i, h].double()
                want, slack = attend(q, k, v)
                check_outputs(got[:, i, h], want, slack, weighted_size(q, k, v), self.dt, (i, h))
        if not skip:
            assert int(self.status[0]) == 0


def _window(rows, window, sink, max_len=0, stream=None):
    a = rows.args(max_len)
    rc, n = B.san_window_attn_bytes(a, window, sink)
    B.check(rc)
    ws = torch.full((max(n, 1),), 0xFF, dtype=torch.uint8, device=DEV)     # NaN patterns: the contents are of no importance
    B.check(B.san_window_attn(a, window, sink, ws, n, stream))
    torch.cuda.synchronize()


def _sees(lens, window, sink):
    return lambda i: [j for j in range(lens[i]) if j >= lens[i] - window or j < sink]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,cap,window,sink,H,Hk,L", [
    ([1], 1, 1, 0, 1, 1, 1),
    ([0, 1, 2, 31, 32, 33, 64, 65, 5, 0], 70, 16, 1, 2, 2, 3),      # around the 32-row slot; empty rows
    ([200, 77, 1, 129, 200], 200, 50, 5, 3, 3, 4),                    # windows that begin inside a slot, sinks before them
    ([90, 40, 7], 96, 1, 0, 4, 4, 1),                                  # a window of one
    ([90, 40, 7], 96, 1000000000, 64, 4, 4, 1),                          # everything is seen
    ([300, 299, 8, 64], 301, 100, 37, 8, 2, 2),                         # query heads in groups of four
    ([61, 13], 64, 33, 4, 20, 1, 5),                                    # more query heads per key head than a unit's rows; two layer groups
    ([1500, 1024], 1500, 1400, 3, 2, 1, 1),                             # one row over several units
    ([257], 300, 300, 0, 1, 1, 9),                                      # three layer groups
])
def test_window_lengths_heads_layers(dtype, lens, cap, window, sink, H, Hk, L):
    r = Rows(dtype, lens, H, Hk, L, cap, seed=len(lens) + cap)
    _window(r, window, sink)
    r.check(_sees(lens, window, sink))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_seen_does_not_matter(dtype):
    """Infinities and NaN between the sinks and the window, and a host bound below the capacity."""
    lens = [150, 88, 41]
    r = Rows(dtype, lens, 4, 2, 2, 160, seed=5)
    k, v = r.d[1], r.d[2]
    for i, t in enumerate(lens):
        gone = slice(3, t - 20)
        k[r.ids[i], :, gone] = float("inf")
        v[:, r.ids[i], :, gone] = float("nan")
    _window(r, 20, 3, max_len=150)
    r.check(_sees(lens, 20, 3))


def test_a_row_whose_scores_are_all_alike_or_huge():
    """Zero queries give the mean of the values; scores in the thousands give the largest one's values."""
    lens = [70, 70]
    r = Rows("bf16", lens, 2, 2, 2, 70, seed=9)
    r.q[0] = 0
    r.q[1] *= 1000
    r.d[0].copy_(r.q)
    _window(r, 64, 4)
    r.check(_sees(lens, 64, 4))


def test_the_same_sequence_twice_and_bad_items():
    lens = [20, 30, 25, 10]
    r = Rows("bf16", lens, 2, 2, 1, 40)
    r.ids[2] = r.ids[1]                                        # the same index twice: read-only, both answered
    r.lens[2] = lens[2] = 30
    r.d[3].copy_(r.ids)
    r.d[4][2] = 30
    r.d[3][0] = 99                                             # an id that there is not
    r.d[4][3] = 41                                             # longer than the bound
    _window(r, 8, 2)
    r.check(_sees(lens, 8, 2), skip=(0, 3))
    st = r.status.cpu().tolist()
    assert st[0] == B.SAN_ERR_DEVICE_CHECK and st[1] == 9 and (st[2], st[3]) in ((0, 99), (3, 41))


def _prefixes(r, plens, groups, pcap, seed=1):
    gen = torch.Generator().manual_seed(seed)
    pk, pv = randn(gen, len(plens), pcap, r.Hk, DH, dtype=r.dt), randn(gen, r.L, len(plens), pcap, r.Hk, DH, dtype=r.dt)
    dk, dv = pk.clone(), pv.clone()
    for g, n in enumerate(plens):
        dk[g, max(0, n):] = float("nan")
        dv[:, g, max(0, n):] = float("nan")
    first = torch.tensor(groups, dtype=torch.int32)
    dev = [x.to(DEV) for x in (dk, dv, torch.tensor(plens, dtype=torch.int32), first)]
    return pk, pv, dev


def _prefix(r, plens, groups, pcap, max_len=0, max_prefix=0, max_group=0, skip=(), stream=None):
    pk, pv, dev = _prefixes(r, plens, groups, pcap)
    a = r.args(max_len)
    x = B.shared_prefix(d_k=dev[0], d_v=dev[1], v_stride=dev[1][0].numel(), n_prefix=len(plens), cap_len=pcap, d_lens=dev[2],
                        max_len=max_prefix, d_first=dev[3], max_group=max_group)
    rc, n = B.san_prefix_attn_bytes(a, x)
    B.check(rc)
    ws = torch.full((max(n, 1),), 0xFF, dtype=torch.uint8, device=DEV)
    B.check(B.san_prefix_attn(a, x, ws, n, stream))
    torch.cuda.synchronize()

    def extra(i, hk):
        for g in range(len(plens)):
            if groups[g] <= i < groups[g + 1]:
                return pk[g, :plens[g], hk].double(), pv[:, g, :plens[g], hk].double()
        return torch.zeros(0, DH, dtype=torch.float64), torch.zeros(r.L, 0, DH, dtype=torch.float64)

    r.check(lambda i: range(r.lens[i]), extra, skip)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,cap,plens,groups,pcap,H,Hk,L", [
    ([0], 1, [1], [0, 1], 1, 1, 1, 1),                                     # nothing of its own
    ([9, 3, 1, 7], 10, [33], [0, 4], 40, 2, 2, 1),                         # one beam behind one prompt
    ([5, 0, 12, 40, 40, 3, 0], 40, [65, 0, 31], [0, 2, 5, 7], 70, 2, 2, 3),    # an empty prefix
    ([0, 3, 0], 4, [0, 9], [0, 2, 3], 9, 2, 1, 2),                         # a row that sees nothing at all
    ([5, 6, 7, 8, 9], 10, [64, 10], [1, 1, 4], 64, 3, 3, 2),               # a prefix without rows; rows without a prefix
    ([4] * 37, 6, [130], [0, 37], 130, 2, 1, 2),                           # more query rows than a unit holds
    ([4] * 70, 4, [100, 90], [0, 50, 70], 100, 4, 4, 1),
    ([4] * 130, 4, [300], [0, 130], 300, 1, 1, 1),
    ([3] * 100, 4, [257, 511], [0, 71, 100], 512, 2, 1, 2),                # 142 and 58 query rows, odd prefixes
    ([2] * 300, 4, [9, 4000, 3999], [0, 3, 3, 300], 4000, 2, 2, 1),        # tensor-core tiles: three rows, none, two tiles and 41 rows
    ([2] * 257, 4, [2500], [0, 257], 2500, 4, 2, 3),                       # the same, query heads in pairs, two layer groups
    ([17, 2], 20, [2000], [0, 2], 2000, 2, 2, 5),                          # one prefix over several units
])
def test_prefix_lengths_groups_heads(dtype, lens, cap, plens, groups, pcap, H, Hk, L):
    r = Rows(dtype, lens, H, Hk, L, cap, seed=len(lens))
    _prefix(r, plens, groups, pcap)


def test_tensor_core_tiles_with_scores_that_keep_growing():
    """Scores that rise along the prefix by more than 2^8 between chunks: the running maximum moves, outputs are scaled."""
    n, P = 600, 6000
    r = Rows("bf16", [1] * n, 2, 2, 2, 2, seed=3)
    gen = torch.Generator().manual_seed(2)
    pk, pv = randn(gen, 1, P, 2, DH, dtype=r.dt), randn(gen, 2, 1, P, 2, DH, dtype=r.dt)
    pk *= torch.linspace(0.1, 40.0, P)[None, :, None, None].to(r.dt)
    dev = [x.to(DEV) for x in (pk, pv, torch.tensor([P], dtype=torch.int32), torch.tensor([0, n], dtype=torch.int32))]
    a = r.args()
    x = B.shared_prefix(d_k=dev[0], d_v=dev[1], v_stride=dev[1][0].numel(), n_prefix=1, cap_len=P, d_lens=dev[2], d_first=dev[3])
    rc, nb = B.san_prefix_attn_bytes(a, x)
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    B.check(B.san_prefix_attn(a, x, ws, nb))
    torch.cuda.synchronize()
    r.check(lambda i: range(1), lambda i, hk: (pk[0, :, hk].double(), pv[:, 0, :, hk].double()))


def test_prefix_bounds_from_the_host_and_a_stream():
    r = Rows("bf16", [4, 9, 2, 2, 7], 4, 2, 2, 32)
    torch.cuda.synchronize()
    _prefix(r, [70, 50], [0, 3, 5], 90, max_len=9, max_prefix=70, max_group=3, stream=torch.cuda.Stream())


@pytest.mark.parametrize("plens,groups,skip,tag", [
    ([20, 21], [0, 2, 4], (2, 3), 10),          # longer than the bound
    ([20, -1], [0, 2, 4], (2, 3), 10),
    ([20, 20], [0, 1, 4], (1, 2, 3), 10),       # more items than the bound
    ([20, 20], [0, 2, 6], (2, 3), 10),          # past the last item
])
def test_a_bad_prefix_leaves_its_rows_alone(plens, groups, skip, tag):
    r = Rows("bf16", [4, 9, 2, 3], 2, 2, 1, 10)
    _prefix(r, plens, groups, 24, max_prefix=20, max_group=2, skip=skip)
    st = r.status.cpu().tolist()
    assert st[:3] == [B.SAN_ERR_DEVICE_CHECK, tag, 1]


def test_captured_twice_in_a_row_with_one_workspace():
    """Two captured calls in order share a workspace; replays see new queries."""
    r = Rows("bf16", [40, 33, 20, 1], 2, 2, 2, 64)
    pk, pv, dev = _prefixes(r, [100], [0, 4], 100)
    a = r.args()
    x = B.shared_prefix(d_k=dev[0], d_v=dev[1], v_stride=dev[1][0].numel(), n_prefix=1, cap_len=100, d_lens=dev[2], d_first=dev[3])
    n = max(B.san_prefix_attn_bytes(a, x)[1], B.san_window_attn_bytes(a, 16, 2)[1])
    ws = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)
    out2 = torch.zeros_like(r.out)
    b = r.args(d_out=out2)
    B.check(B.san_prefix_attn(a, x, ws, n))
    B.check(B.san_window_attn(b, 16, 2, ws, n))
    torch.cuda.synchronize()
    graphs = []
    for call in (lambda: B.san_prefix_attn(a, x, ws, n), lambda: B.san_window_attn(b, 16, 2, ws, n)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.check(call())
        graphs.append(g)
    for seed in (3, 4):
        r.q = randn(torch.Generator().manual_seed(seed), *r.q.shape, dtype=r.dt)
        r.d[0].copy_(r.q)
        r.out.fill_(-7)
        out2.fill_(-7)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        r.check(lambda i: range(r.lens[i]), lambda i, hk: (pk[0, :, hk].double(), pv[:, 0, :, hk].double()))
        first, r.out = r.out, out2
        r.check(_sees(r.lens, 16, 2))
        r.out = first


def test_tensor_core_tiles_captured_and_replayed():
    """Tiles, own rows beside them and the join, replayed back to back with new queries and lengths."""
    n, P = 600, 8100
    r = Rows("bf16", [3] * n, 2, 2, 1, 6, seed=21)
    gen = torch.Generator().manual_seed(12)
    pk, pv = randn(gen, 1, P, 2, DH, dtype=r.dt), randn(gen, 1, 1, P, 2, DH, dtype=r.dt)
    dev = [x.to(DEV) for x in (pk, pv, torch.tensor([P], dtype=torch.int32), torch.tensor([0, n], dtype=torch.int32))]
    a = r.args()
    x = B.shared_prefix(d_k=dev[0], d_v=dev[1], v_stride=dev[1][0].numel(), n_prefix=1, cap_len=P, d_lens=dev[2], d_first=dev[3])
    rc, nb = B.san_prefix_attn_bytes(a, x)
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    B.check(B.san_prefix_attn(a, x, ws, nb))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(3):                                      # the same workspace, call after call
            B.check(B.san_prefix_attn(a, x, ws, nb))
    for seed, p in ((5, P), (6, 65)):
        r.q = randn(torch.Generator().manual_seed(seed), *r.q.shape, dtype=r.dt)
        r.d[0].copy_(r.q)
        dev[2].fill_(p)
        r.out.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        r.check(lambda i: range(3), lambda i, hk: (pk[0, :p, hk].double(), pv[:, 0, :p, hk].double()))


def test_far_rows_of_a_large_plane():
    """Byte offsets beyond 32 bits inside one key plane: the rows that are read are the last ones."""
    H, cap, n = 2, 70000, 260                       # 260 * 2 * 70000 * 128 B = 4.66 GB a plane
    k = torch.zeros(n, H, cap, DH, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros(1, n, H, cap, DH, dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator().manual_seed(7)
    small = randn(gen, H, cap % 8 + 40, DH, dtype=torch.bfloat16)
    t = small.shape[1]
    last = cap - t
    full_k = torch.zeros(H, t, DH, dtype=torch.bfloat16)
    full_k.copy_(small)
    # permuted by the absolute position: `last` is a multiple of 8
    assert last % 8 == 0
    k[n - 1, :, last:] = to_planes(full_k).to(DEV)
    v[0, n - 1, :, last:] = to_planes(full_k).to(DEV)
    q = randn(gen, 1, H, DH, dtype=torch.bfloat16)
    out = torch.zeros(1, 1, H, DH, dtype=torch.bfloat16, device=DEV)
    qd = q.to(DEV)
    ids, lens = (torch.tensor([x], dtype=torch.int32, device=DEV) for x in (n - 1, cap))
    a = B.cached_rows(dtype=B.SAN_BF16, n_heads=H, n_kv_heads=H, n_layers=1, d_q=qd, d_k=k, d_v=v, v_stride=k.numel(), max_ids=n,
                      cap_len=cap, d_ids=ids, d_lens=lens, n_items=1, d_out=out)
    rc, nb = B.san_window_attn_bytes(a, t, 0)
    ws = torch.empty(max(nb, 1), dtype=torch.uint8, device=DEV)
    B.check(B.san_window_attn(a, t, 0, ws, nb))
    torch.cuda.synchronize()
    got = out.cpu()
    for h in range(H):
        kk = small[h].double()
        want, slack = attend(q[0, h].double(), kk, kk[None])
        check_outputs(got[:, 0, h], want, slack, weighted_size(q[0, h].double(), kk, kk[None]), torch.bfloat16, h)


def _least(r, room, call):
    """`call` with a workspace of exactly `room` bytes; what lies behind it stays as it was."""
    ws = torch.full((room + 512,), 0x5A, dtype=torch.uint8, device=DEV)
    ws[:room] = 0xFF
    r.out.fill_(-7)
    B.check(call(ws, room))
    torch.cuda.synchronize()
    assert (ws[room:] == 0x5A).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_window_with_the_workspace_of_a_larger_batch(dtype):
    """Rows that are cut into several runs, into as many as find room, and into one."""
    window, sink, H, L = 900, 3, 2, 2
    lens = [1500, 1024, 7, 0, 1499]
    r = Rows(dtype, lens, H, 1, L, 1500, seed=2)
    a = r.args()
    full = B.san_window_attn_bytes(a, window, sink)[1]
    one = (len(lens) * H * 8 + 255) // 256 * 256 + len(lens) * H * L * DH * 4
    assert full > 3 * one
    for room in (full, 4 * one + 300, 2 * one + 5, 2 * one - 300, 5, 0):
        _least(r, room, lambda ws, n: B.san_window_attn(a, window, sink, ws, n))
        r.check(_sees(lens, window, sink))
    B.check(B.san_window_attn(a, window, sink, None, 0))
    # the batch shrinks, the workspace is that of its beginning
    for n in range(len(lens), 0, -1):
        b = r.args(n_items=n)
        out = torch.full_like(r.out, -7.0)
        ws = torch.empty(max(full, 1), dtype=torch.uint8, device=DEV)
        b.d_out = out.data_ptr()
        B.check(B.san_window_attn(b, window, sink, ws, full))
        torch.cuda.synchronize()
        got = out.flatten()[:L * n * H * DH].view(L, n, H, DH)
        keep, r.out = r.out, torch.full_like(r.out, -7.0)
        r.out[:, :n] = got
        r.check(_sees(lens, window, sink), skip=range(n, len(lens)))
        r.out = keep


@pytest.mark.parametrize("dtype,n,P,H,Hk,L", [
    ("bf16", 3, 4000, 2, 2, 2),           # one long prefix in many runs
    ("f32", 3, 900, 2, 1, 2),
    ("bf16", 257, 2500, 2, 2, 3),         # tensor-core tiles
])
def test_prefix_with_the_least_workspace(dtype, n, P, H, Hk, L):
    """Two partial results a row are enough; less than that is refused."""
    own = 300
    lens = [own if i == 1 else 2 + i % 3 for i in range(n)]
    r = Rows(dtype, lens, H, Hk, L, own, seed=n)
    pk, pv, dev = _prefixes(r, [P], [0, n], P)
    a = r.args()
    x = B.shared_prefix(d_k=dev[0], d_v=dev[1], v_stride=dev[1][0].numel(), n_prefix=1, cap_len=P, d_lens=dev[2], d_first=dev[3])
    full = B.san_prefix_attn_bytes(a, x)[1]
    need = lambda k: (k * n * H * 8 + 255) // 256 * 256 + k * n * H * L * DH * 4          # noqa: E731
    assert full > need(2)
    for room in sorted({need(2), need(3), need(4) + 100, full - 1}):
        _least(r, room, lambda ws, b: B.san_prefix_attn(a, x, ws, b))
        r.check(lambda i: range(lens[i]), lambda i, hk: (pk[0, :, hk].double(), pv[:, 0, :, hk].double()))
    ws = torch.empty(full, dtype=torch.uint8, device=DEV)
    assert B.san_prefix_attn(a, x, ws, need(2) - 1) == B.SAN_ERR_CAPACITY
    assert B.san_prefix_attn(a, x, None, 0) == B.SAN_ERR_NULL


def test_many_small_prefixes_without_a_bound_on_groups():
    """max_group left at 0: any prefix may have all items, by the host's knowledge; their kernel is the tiles' then."""
    G, own = 24, 5
    groups = [0]
    for g in range(G):
        groups.append(groups[-1] + (g * 5) % 9)                # 0 to 8 items each
    lens = [(i * 3) % (own + 1) for i in range(groups[-1])]
    plens = [(g * 37) % 65 for g in range(G)]
    for bound in (0, 8):
        r = Rows("bf16", lens, 2, 2, 2, own, seed=bound)
        _prefix(r, plens, groups, 64, max_group=bound)


@pytest.mark.parametrize("n,P,H,Hk,L", [(100, 2500, 16, 1, 2), (400, 3000, 8, 2, 1), (130, 2100, 12, 3, 3)])
def test_tensor_core_tiles_with_grouped_heads(n, P, H, Hk, L):
    """4 and 16 query heads a key head: 256 rows of a tile pair are several items' heads."""
    r = Rows("bf16", [i % 4 for i in range(n)], H, Hk, L, 4, seed=n)
    _prefix(r, [P], [0, n], P)


@pytest.mark.parametrize("what", ["inf", "-inf", "nan"])
@pytest.mark.parametrize("n", [3, 300])
def test_bad_values_in_a_prefix(what, n):
    """One element of one value row of a prefix, by the streams and by the tiles: its column is no number for the rows behind
    that prefix, all other outputs are as they are without it."""
    P, L, col, bad = 2500, 2, 11, 1777
    r = Rows("bf16", [2] * (n + 2), 2, 2, L, 4, seed=n)
    pk, pv, dev = _prefixes(r, [P, 30], [0, n, n + 2], P)
    pv[1, 0, bad, :, col] = 0.0
    dev[1][1, 0, bad, :, col] = float(what)
    a = r.args()
    x = B.shared_prefix(d_k=dev[0], d_v=dev[1], v_stride=dev[1][0].numel(), n_prefix=2, cap_len=P, d_lens=dev[2], d_first=dev[3])
    size = B.san_prefix_attn_bytes(a, x)[1]
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    B.check(B.san_prefix_attn(a, x, ws, size))
    torch.cuda.synchronize()
    assert not torch.isfinite(r.out[1, :n, :, col]).any()
    r.out[1, :n, :, col] = 0.0
    got = r.out.cpu()
    assert torch.isfinite(got).all()
    for i in list(range(0, n, max(1, n // 20))) + [n, n + 1]:
        g, plen = (0, P) if i < n else (1, 30)
        for h in range(2):
            q = r.q[i, h].double()
            k = torch.cat([pk[g, :plen, h].double(), r.k[r.ids[i], h, :2].double()])
            v = torch.cat([pv[:, g, :plen, h].double(), r.v[:, r.ids[i], h, :2].double()], 1)
            want, slack = attend(q, k, v)
            if i < n:
                want[1, col] = 0.0
            check_outputs(got[:, i, h], want, slack, weighted_size(q, k, v), r.dt, (i, h))


@pytest.mark.parametrize("n,own", [(2, 3), (200, 3)])
def test_far_rows_of_large_prefixes(n, own):
    """Byte offsets beyond 32 bits in the arrays of a prefix, by the streams and by the tiles."""
    P, H, G = 70000, 64, 4                                          # 2.3 GB of keys, and of values
    r = Rows("bf16", [own] * n, H, H, 1, 4, seed=n)
    gen = torch.Generator(device=DEV).manual_seed(9)
    pk, pv = (torch.randn(*s, G, P, H, DH, generator=gen, device=DEV, dtype=torch.bfloat16) for s in ((), (1,)))
    plens, first = [5, 0, 9, P], [0, 0, 0, 1, n]                    # item 0 behind the third prefix, the others behind the last
    dev = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (plens, first)]
    a = r.args()
    x = B.shared_prefix(d_k=pk, d_v=pv, v_stride=pv.numel(), n_prefix=G, cap_len=P, d_lens=dev[0], d_first=dev[1], max_group=max(1, n - 1))
    size = B.san_prefix_attn_bytes(a, x)[1]
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    B.check(B.san_prefix_attn(a, x, ws, size))
    torch.cuda.synchronize()
    assert int(r.status[0]) == 0
    for i, h in ((0, 63), (1, 0), (1, 63), (n - 1, 31)):
        g = 2 if i == 0 else 3
        q = r.q[i, h].double()
        k = torch.cat([pk[g, :plens[g], h].cpu().double(), r.k[r.ids[i], h, :own].double()])
        v = torch.cat([pv[:, g, :plens[g], h].cpu().double(), r.v[:, r.ids[i], h, :own].double()], 1)
        want, slack = attend(q, k, v)
        check_outputs(r.out[:, i, h].cpu(), want, slack, weighted_size(q, k, v), r.dt, (i, h))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_streams_at_once_behind_their_inputs(dtype):
    """Two calls that may overlap, a workspace each, both behind what wrote their inputs."""
    r = Rows(dtype, [1500, 1024, 700], 2, 1, 2, 1500, seed=3)
    pk, pv, dev = _prefixes(r, [900], [0, 3], 900)
    other = torch.full_like(r.out, -7.0)
    a, b = r.args(), r.args(d_out=other)
    x = B.shared_prefix(d_k=dev[0], d_v=dev[1], v_stride=dev[1][0].numel(), n_prefix=1, cap_len=900, d_lens=dev[2], d_first=dev[3])
    na, nb = B.san_prefix_attn_bytes(a, x)[1], B.san_window_attn_bytes(b, 1200, 2)[1]
    wa, wb = (torch.full((max(s, 1),), 0xFF, dtype=torch.uint8, device=DEV) for s in (na, nb))
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (one, two):
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        B.check(B.san_prefix_attn(a, x, wa, na, one))
        B.check(B.san_window_attn(b, 1200, 2, wb, nb, two))
    torch.cuda.synchronize()
    r.check(lambda i: range(r.lens[i]), lambda i, hk: (pk[0, :, hk].double(), pv[:, 0, :, hk].double()))
    r.out = other
    r.check(_sees(r.lens, 1200, 2))
