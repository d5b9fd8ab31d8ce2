"""san_packed_block against attention of each sequence in 64 bits: lengths, groups, layers, strides, values that are not seen."""
import math

import pytest
import torch

from paper_1906_11024_b200 import binding as B
from paper_1906_11024_b200 import build as san_build
from tests.keep_helpers import DH, packed

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    san_build.build()


def make(lens, H, Hk, L, seed=0, gap=0, ld=None):
    """Inputs for sequences of these lengths, `gap` tokens of none in front of the first and behind the last."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    N = sum(lens) + 2 * gap
    r = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(BF)                       # noqa: E731
    first = [gap]
    for t in lens:
        first.append(first[-1] + t)
    x = dict(lens=lens, H=H, Hk=Hk, L=L, N=N, first=torch.tensor(first, dtype=torch.int32, device=DEV))
    if ld == "fused":
        qkv = r(L, N, H + 2 * Hk, DH)
        x.update(q=qkv[0, :, :H], k=qkv[0, :, H:H + Hk], v=qkv[:, :, H + Hk:])
    elif ld == "apart":                                     # three distances between tokens
        x.update(q=r(N, H + 1, DH)[:, :H], k=r(N, Hk + 2, DH)[:, 1:1 + Hk], v=r(L, N, 2 * Hk + 3, DH)[:, :, Hk:2 * Hk])
    else:
        x.update(q=r(N, H, DH), k=r(N, Hk, DH), v=r(L, N, Hk, DH))
    x["out"] = torch.full((L, N, H, DH), -7.0, dtype=BF, device=DEV)
    x["status"] = torch.zeros(8, dtype=torch.int32, device=DEV)
    return x


def args(x, **kw):
    a = dict(dtype=B.SAN_BF16, n_heads=x["H"], n_kv_heads=x["Hk"], n_layers=x["L"], d_q=x["q"], ld_q=x["q"].stride(0), d_k=x["k"],
             ld_k=x["k"].stride(0), d_v=x["v"], ld_v=x["v"].stride(1), v_stride=x["v"].stride(0), d_first=x["first"], n_seq=len(x["lens"]),
             n_tokens=x["N"], max_len=max(x["lens"]), d_out=x["out"], d_status=x["status"])
    return B.packed_args(**(a | kw))


def room(a):
    rc, n = B.san_packed_block_bytes(a)
    B.check(rc)
    return torch.full((max(n, 256),), 0xAB, dtype=torch.uint8, device=DEV), n


def call(x, stream=None, **kw):
    a = args(x, **kw)
    ws, n = room(a)
    B.check(B.san_packed_block(a, ws, n, stream))
    torch.cuda.synchronize()


def check(x, out=None, lens=None):
    out = x["out"] if out is None else out
    first = x["first"].tolist()
    seen = torch.zeros(x["N"], dtype=torch.bool, device=DEV)
    for s, t in enumerate(lens or x["lens"]):
        a = first[s]
        if t == 0:
            continue
        want, bound = packed(x["q"][a:a + t], x["k"][a:a + t], x["v"][:, a:a + t], BF)
        off = (out[:, a:a + t].double() - want).abs()
        bad = ~(off <= bound)
        assert not bool(bad.any()), (s, t, int(bad.sum()), float((off / bound).max()))
        seen[a:a + t] = True
    assert bool((out[:, ~seen] == -7.0).all())              # tokens of no sequence


SHAPES = [
    ([37], 8, 8, 1), ([1], 3, 1, 2), ([1, 1, 1, 0, 2], 2, 2, 1), ([31, 32, 33, 64, 65, 127], 4, 2, 3), ([16] * 40, 4, 1, 5), ([0, 5, 0, 0, 9, 0], 6, 3, 4),
    ([128], 2, 2, 1), ([127, 128, 129, 1, 255, 256, 257, 0, 383, 600], 4, 2, 2), ([700], 3, 1, 3), ([1, 2000, 3, 40], 4, 4, 1), ([300] * 12, 6, 2, 5),
    ([2049, 0, 511], 12, 4, 2),
]


@pytest.mark.parametrize("lens,H,Hk,L", SHAPES)
@pytest.mark.parametrize("ld", [None, "fused", "apart"])
def test_packed(lens, H, Hk, L, ld):
    x = make(lens, H, Hk, L, seed=len(lens) + H, gap=3 if ld else 0, ld=ld)
    call(x)
    check(x)
    assert int(x["status"][0]) == 0


@pytest.mark.parametrize("bound", [0, 150, 1000])
def test_bound_on_lengths_does_not_matter(bound):
    x = make([40, 100, 7, 150], 4, 2, 2)
    N = x["N"]
    call(x, max_len=min(bound, N))
    check(x)


def test_many_sequences():
    x = make([(i * 37) % 90 for i in range(1500)] + [400], 2, 1, 1, seed=5)
    call(x)
    check(x)


def test_long_sequence():
    x = make([9000, 1, 5000], 2, 1, 2, seed=6)
    call(x)
    check(x)


@pytest.mark.parametrize("t", [60, 700])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_what_is_not_seen_does_not_matter(t, value):
    """Keys and values of later tokens, of other sequences, of no sequence."""
    x = make([t, 90, t], 4, 2, 2, seed=7, gap=5)
    wants = [(s, packed(x["q"][s:s + n], x["k"][s:s + n], x["v"][:, s:s + n], BF)) for s, n in ((5, t), (5 + t, 90), (95 + t, t))]
    a = 5 + t // 3
    for y in (x["k"], x["v"][0], x["v"][1]):
        y[a, 0, 3] = value                                  # token a of the first sequence, key head 0
        y[:5] = value
        y[-5:] = value
    x["out"].fill_(-7.0)
    call(x)
    out = x["out"]
    spoiled = torch.zeros_like(out, dtype=torch.bool)
    spoiled[:, a:5 + t, :2] = True                          # rows that see it, heads of that key head
    # the others are what they are without it (rows may be computed another way next to such values: no bits are compared)
    for s, (want, bound) in wants:
        off = (out[:, s:s + want.shape[1]].double() - want).abs()
        assert bool(((off <= bound) | spoiled[:, s:s + want.shape[1]]).all())
    assert bool((out[:, :5] == -7.0).all()) and bool((out[:, -5:] == -7.0).all())
    if math.isnan(value):
        assert bool(out[:, a:5 + t, :2].isnan().all())
    else:
        # a score of +inf makes its row NaN (one of -inf is a weight of zero)
        up = x["q"][a:5 + t, :2, 3].float() * value > 0
        assert bool(out[:, a:5 + t, :2].isnan().all(-1)[:, up].all()) and bool(up.any())


@pytest.mark.parametrize("lens", [[700, 90], [60, 100]])
@pytest.mark.parametrize("shape", ["rising", "falling", "steps", "one", "far"])
def test_scores_that_move_along_a_sequence(lens, shape):
    """Maxima that a row meets late, early, at some tokens alone, and scores too far apart for one scale."""
    x = make(lens, 4, 2, 2, seed=16)
    N = x["N"]
    at = torch.arange(N, device=DEV).float()
    up = {"rising": at / 40, "falling": (N - at) / 40, "steps": (at // 64 % 3) * 9, "one": (at % 97 == 13) * 40.0, "far": (at // 50) * 60}[shape]
    x["q"][..., 0] = 8.0                                    # a score of its own for every token: q.k / 8 = up + the rest
    x["k"][..., 0] = up[:, None].bfloat16()
    call(x)
    check(x)
    assert int(x["status"][0]) == 0


@pytest.mark.parametrize("t", [50, 300])
def test_scores_of_minus_infinity_give_zeros(t):
    x = make([t, 20], 2, 2, 1, seed=8)
    x["q"][:t] = 0
    x["q"][:t, :, 0] = 1.0
    x["k"][:t] = 0
    x["k"][:t, :, 0] = -math.inf
    call(x)
    assert bool((x["out"][:, :t] == 0).all())
    first = x["first"].tolist()
    want, bound = packed(x["q"][t:], x["k"][t:], x["v"][:, t:], BF)
    assert first[1] == t and bool(((x["out"][:, t:].double() - want).abs() <= bound).all())


@pytest.mark.parametrize("lens", [[50, 60, 70], [200, 300, 100]])
def test_bad_sequences_are_skipped_and_reported(lens):
    for first, item, bad in [([0, lens[0], lens[0] + lens[1] + 10 ** 6, sum(lens)], 1, [1, 2]), ([lens[2], lens[2] + lens[0], 0, lens[2]], 1, [1]),
                             ([-4, lens[0], lens[0] + lens[1], sum(lens)], 0, [0])]:
        x = make(lens, 2, 1, 1, seed=9)
        x["first"] = torch.tensor(first, dtype=torch.int32, device=DEV)
        call(x, max_len=max(lens) + 20)
        st = x["status"].tolist()
        assert st[0] == B.SAN_ERR_DEVICE_CHECK and st[1] == 12 and st[2] in bad
        for s in range(3):
            if s in bad:
                continue
            a, b = first[s], first[s + 1]
            want, bound = packed(x["q"][a:b], x["k"][a:b], x["v"][:, a:b], BF)
            assert not bool(((x["out"][:, a:b].double() - want).abs() > bound).any()), (first, s)
    x = make(lens, 2, 1, 1, seed=9)                         # longer than the bound
    call(x, max_len=max(lens) - 1)
    s = lens.index(max(lens))
    assert x["status"].tolist()[:5] == [B.SAN_ERR_DEVICE_CHECK, 12, s, max(lens), max(lens) - 1]
    check(x, lens=[0 if i == s else t for i, t in enumerate(lens)])


def test_sequences_that_overlap_stay_in_bounds():
    """More tiles than the tokens have room for: what does not fit the list is skipped and reported."""
    x = make([600], 1, 1, 1, seed=10)
    n = 41
    x["first"] = torch.tensor([0, 600] * n, dtype=torch.int32, device=DEV)
    x["lens"] = [600] * (2 * n - 1)
    a = args(x, n_tokens=600, max_len=600)
    ws, b = room(a)
    guard = torch.full((b + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    B.check(B.san_packed_block(a, guard, b))
    torch.cuda.synchronize()
    assert bool((guard[b:] == 0x5A).all()) and int(x["status"][0]) == B.SAN_ERR_DEVICE_CHECK


@pytest.mark.parametrize("lens", [[30, 60], [500, 40, 300]])
def test_captured_and_replayed_on_other_inputs_and_lengths(lens):
    x, y = make(lens, 4, 2, 2, seed=11), make(lens[::-1], 4, 2, 2, seed=12)
    a = args(x)
    ws, n = room(a)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        B.check(B.san_packed_block(a, ws, n))
    for z in (x, y):
        for name in ("q", "k", "v", "first"):
            x[name].copy_(z[name])
        x["out"].fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        check(x, lens=z["lens"])


def test_two_streams_with_workspaces_of_their_own():
    xs = [make([400, 30, 900], 4, 2, 2, seed=13), make([70, 800, 0, 129], 4, 1, 1, seed=14)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    plans = [(args(x), *room(args(x))) for x in xs]
    torch.cuda.synchronize()
    for _ in range(20):
        for (a, ws, n), s in zip(plans, streams):
            B.check(B.san_packed_block(a, ws, n, s))
    torch.cuda.synchronize()
    for x in xs:
        check(x)


def test_offsets_past_32_bits():
    """Tokens so far apart that their addresses pass 4 GB."""
    H, t = 2, 300
    x = make([t, t], H, H, 1, seed=15)
    ld = 1 << 23                                            # elements: 600 tokens are 10 GB of bf16
    big = torch.zeros(2 * t * ld, dtype=BF, device=DEV)
    wide = lambda off: torch.as_strided(big, (2 * t, H, DH), (ld, DH, 1), off)             # noqa: E731
    q, k, v = wide(0), wide(H * DH), wide(2 * H * DH)
    q.copy_(x["q"]); k.copy_(x["k"]); v.copy_(x["v"][0])
    for short in (False, True):
        x["out"].fill_(-7.0)
        if short:
            x["first"] = torch.tensor([0, 100, 100], dtype=torch.int32, device=DEV)
            x["first"] += 450
            x["lens"] = [100, 0]
        x.update(q=q, k=k, v=v[None])
        call(x, v_stride=8, max_len=max(x["lens"]))
        check(x)


@pytest.mark.parametrize("lens", [[700, 90, 1000], [60, 100]])
@pytest.mark.parametrize("layout", [None, "fused", "apart", "wide keys", "wide values"])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_seen_at_all_distances(lens, layout, value):
    """Rows that are computed again beside a bad value read keys and values each at their own distance."""
    H, Hk, L = 4, 2, 3
    x = make(lens, H, Hk, L, seed=17, ld=layout if layout in ("fused", "apart") else None)
    N = x["N"]
    if layout in ("wide keys", "wide values"):              # (with room behind the other, so that a wrong distance stays in its buffer)
        wide, tight = ("k", "v") if layout == "wide keys" else ("v", "k")
        room_for = torch.zeros(L * N * (Hk + 20) * DH, dtype=BF, device=DEV)
        room_for.normal_()
        x[tight] = room_for[:x[tight].numel()].view(x[tight].shape).copy_(x[tight])
        far = torch.randn(*x[wide].shape[:-2], Hk + 20, DH, device=DEV).to(BF)
        far[..., 7:7 + Hk, :] = x[wide]
        x[wide] = far[..., 7:7 + Hk, :]
    first = x["first"].tolist()
    wants = [packed(x["q"][a:a + t], x["k"][a:a + t], x["v"][:, a:a + t], BF) for a, t in zip(first, lens)]
    bad = [(s, b) for s, t in enumerate(lens) for b in (1, t // 3, t - 1)]
    for s, b in bad:                                        # one dim of key head 0, in one layer
        x["v"][1, first[s] + b, 0, 3] = value
    call(x)
    assert int(x["status"][0]) == 0
    for s, (a, t) in enumerate(zip(first, lens)):
        out, (want, bound) = x["out"][:, a:a + t], wants[s]
        sees = torch.zeros_like(out, dtype=torch.bool)
        sees[1, 1:, :H // Hk, 3] = True
        assert bool((((out.double() - want).abs() <= bound) | sees).all()), s
        assert not bool(out[sees].isfinite().any())


def test_rows_computed_again_may_take_longer_than_a_wait():
    """A bad value at the end of a sequence so long that the rows before it, computed again, take a second and more."""
    N, L = 1_300_000, 2
    x = make([N], 1, 1, L, seed=18)
    x["q"] *= 3                                             # few keys have most of a row's weight
    x["v"][1, N - 1, 0, 3] = math.nan
    call(x)
    assert int(x["status"][0]) == 0
    out = x["out"][:, :, 0]
    rows = list(range(N - 129, N - 1, 9)) + [0, 1, 127, 128, 255, N // 3, N // 2 + 1]
    for a in rows:
        q, k, v = x["q"][a, 0].double(), x["k"][:a + 1, 0].double(), x["v"][:, :a + 1, 0].double()
        p = torch.softmax(k @ q / 8.0, 0)
        want, size = p @ v, p @ v.abs()
        # as in keep_helpers.packed, but that sums are made of products of 16 keys at once, added up one after the other
        dz = 70 * 2.0 ** -23 * float((k.abs() @ q.abs()).max()) / 8.0
        bound = size * (4 * dz + 2.0 ** -20 + 2 * (a / 8 + 16) * 2.0 ** -23 + 2 * 2.0 ** -8) + 2.0 ** -8 * want.abs() + 1e-30
        assert bool(((out[:, a].double() - want).abs() <= bound).all()), a
    assert bool(out[:, :N - 1].isfinite().all()) and bool((out[:, ::997] != -7.0).any(-1).all())
    assert bool(out[0, N - 1].isfinite().all()) and bool(out[1, N - 1, 3].isnan())
