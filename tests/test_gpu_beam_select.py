"""Beam selection (san_beam_select) against a 64-bit choice over all candidates: whole numbers equal, scores within
float32 rounding."""
import numpy as np
import pytest
import torch

from paper_1906_11024_b200 import binding as B
from paper_1906_11024_b200 import build as san_build
from tests.serve_helpers import dtype_of, select

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    san_build.build()
    B.lib()


def _state(rng, S, beam, V, steps, cap, done_share=0.2, dead_share=0.0):
    rows = S * beam
    done = (rng.random(rows) < done_share).astype(np.int32)
    score = (-(0.3 + rng.random(rows)) * steps).astype(np.float32)
    score[rng.random(rows) < dead_share] = -np.inf
    length = np.where(done == 1, rng.integers(1, steps + 1, rows), steps).astype(np.int32)
    return dict(score=score, len=length, done=done, tokens=rng.integers(0, V, (rows, cap)).astype(np.int32))


def _call(logits, ld, V, st, S, beam, eos, alpha, in_place=False, history=True, stream=None, offset=0, status=None):
    """Returns the outputs as numpy arrays (histories behind the new length hold -7)."""
    rows = S * beam
    buf = torch.full((rows * ld + offset,), float("nan"), dtype=logits.dtype, device=DEV)
    view = buf[offset:].view(rows, ld)
    view[:, :V] = logits.to(DEV)
    d = {k: torch.from_numpy(np.array(v)).to(DEV) for k, v in st.items()}
    o = d if in_place else {k: torch.full_like(v, -7) for k, v in d.items()}
    parent, nxt = torch.full_like(d["len"], -9), torch.full_like(d["len"], -9)
    rc, n = B.san_beam_select_bytes(S, beam, V)
    B.check(rc)
    ws = torch.full((n + 1,), 0xA5, dtype=torch.uint8, device=DEV)          # the contents are of no importance
    a = B.select_args(dtype=B.SAN_BF16 if logits.dtype == torch.bfloat16 else B.SAN_F32, n_sent=S, beam=beam, vocab=V,
                      d_logits=buf.data_ptr() + offset * buf.element_size(), ld_logits=ld, eos=eos, alpha=alpha,
                      d_score=d["score"], d_len=d["len"], d_done=d["done"], d_tokens=d["tokens"] if history else None,
                      ld_tokens=d["tokens"].shape[1] if history else 0, d_score_out=o["score"], d_len_out=o["len"],
                      d_done_out=o["done"], d_tokens_out=o["tokens"] if history else None, d_parent=parent, d_next=nxt,
                      d_workspace=ws, workspace_bytes=n, d_status=status)
    B.check(B.san_beam_select(a, stream))
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in o.items()} | {"parent": parent.cpu().numpy(), "next": nxt.cpu().numpy()}


def _compare(got, want, st, history=True, in_place=False):
    for k in ("parent", "next", "len", "done"):
        assert np.array_equal(got[k], want[k]), k
    live = np.isfinite(want["score"])
    assert np.array_equal(np.isfinite(got["score"]), live) and (got["score"][~live] == -np.inf).all()
    # float32 terms of the sum of exponentials within 2^-21, rounded to float32 once
    assert (np.abs(got["score"][live] - want["score"][live]) <= 2.0 ** -20 + 2.0 ** -23 * np.abs(want["score"][live])).all()
    if history:
        for r, tok in enumerate(want["tokens"]):
            assert list(got["tokens"][r][:len(tok)]) == [int(t) for t in tok], r
            behind = got["tokens"][r][len(tok):]
            assert np.array_equal(behind, st["tokens"][r][len(tok):]) if in_place else (behind == -7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,beam,V,pad,alpha", [
    (1, 1, 1, 0, 0.0),            # one token
    (1, 4, 7, 1, 0.6),            # fewer tokens than a thread's share
    (3, 4, 2048, 0, 0.0),         # a chunk exactly
    (2, 5, 2049, 7, 1.0),         # one token in the last chunk
    (5, 8, 8191, 1, 0.6),
    (40, 4, 16385, 7, 0.6),       # chunks of 8192, rows on 16-byte boundaries
    (3, 9, 700, 4, 0.0),          # more than eight wanted: the merged bound
    (30, 20, 8200, 3, 1.0),       # rows off 16-byte boundaries
    (2, 32, 40, 0, 0.6),          # barely more tokens than slots
    (2, 32, 33000, 8, 0.0),
])
def test_against_all_candidates(dtype, S, beam, V, pad, alpha):
    rng = np.random.default_rng([S, beam, V])
    dt, _ = dtype_of(dtype)
    st = _state(rng, S, beam, V, steps=6, cap=9)
    logits = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32) * 2).to(dt)
    eos = min(2, V - 1)
    want = select(logits, st["score"], st["len"], st["done"], st["tokens"], eos, float(np.float32(alpha)), beam)
    assert want["gap"] > 1e-6 or want["gap"] == 0.0         # the choice is not within float32 rounding of another
    _compare(_call(logits, V + pad, V, st, S, beam, eos, alpha), want, st)
    if pad == 7:                                            # a base address off its boundary too
        _compare(_call(logits, V + pad, V, st, S, beam, eos, alpha, offset=3), want, st)


@pytest.mark.parametrize("beam", [4, 12, 32])
def test_ties_go_to_the_lowest_slot_and_token(beam):
    """Equal hypotheses with equal logits, all logits alike, and the type's lowest value everywhere."""
    S, V = 2, 5000
    st = dict(score=np.full(S * beam, -1.5, np.float32), len=np.full(S * beam, 3, np.int32), done=np.zeros(S * beam, np.int32),
              tokens=np.arange(S * beam * 5).reshape(S * beam, 5).astype(np.int32))
    rng = np.random.default_rng(0)
    one = torch.from_numpy(np.repeat(rng.integers(-2, 3, (1, V)), S * beam, 0).astype(np.float32))
    for x in (one, torch.zeros(S * beam, V), torch.full((S * beam, V), torch.finfo(torch.float32).min)):
        for ld in (V, V + 1):
            want = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, 0.0, beam)
            _compare(_call(x, ld, V, st, S, beam, 2, 0.0), want, st)


@pytest.mark.parametrize("beam,V", [(12, 1500), (15, 300), (16, 40), (5, 12000)])
def test_ties_among_a_few_hundred_candidates(beam, V):
    """More candidates than are ordered at once, all of the same rank, or of two."""
    st = dict(score=np.full(beam, -1.5, np.float32), len=np.full(beam, 3, np.int32), done=np.zeros(beam, np.int32),
              tokens=np.arange(beam * 5).reshape(beam, 5).astype(np.int32))
    two = torch.zeros(beam, V)
    two[:, 1::7] = 1.0
    for x in (torch.zeros(beam, V), two):
        want = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, 0.6, beam)
        _compare(_call(x, V, V, st, 1, beam, 2, 0.6), want, st)


def test_rising_logits_one_thread_holds_the_best():
    """The best candidates sit next to one another (all in one thread's share), and in the last chunk."""
    for beam in (4, 8, 32):
        V = 20000
        x = torch.arange(V, dtype=torch.float32).repeat(beam, 1) * 1e-3
        x[:, 4000:4032] += 30.0
        st = _state(np.random.default_rng(beam), 1, beam, V, 4, 6, done_share=0.0)
        want = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, 0.0, beam)
        _compare(_call(x, V, V, st, 1, beam, 2, 0.0), want, st)


def test_many_candidates_above_the_bound():
    """Beam 32 over many chunks where a few hypotheses hold all of the best candidates: more of them pass the
    merge's bound than its list holds."""
    S, beam, V = 1, 32, 400000
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.standard_normal((beam, V), dtype=np.float32))
    st = _state(rng, S, beam, V, 4, 6, done_share=0.0)
    st["score"][:] = -1000.0 - np.arange(beam)
    st["score"][:3] = [-1.0, -1.1, -1.2]
    want = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, 0.0, beam)
    _compare(_call(x, V, V, st, S, beam, 2, 0.0), want, st)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ties", [False, True])
def test_all_winners_in_one_part(dtype, ties):
    """Every winner of the first sentence is the best, second best, ... of the same part of one row, down to its last
    place; the merge, which takes the parts' best ones first, must not stop before."""
    S, beam, V = 2, 32, 50257
    rng = np.random.default_rng(6)
    x = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32))
    x[7, 30001:30041] = 20.0 if ties else torch.arange(40, dtype=torch.float32) / 4 + 20.0
    x = x.to(dtype_of(dtype)[0])
    st = _state(rng, S, beam, V, 4, 6, done_share=0.0)
    st["score"][:beam] -= 40.0
    st["score"][7] = -1.0
    for ld in (V, V + 7):
        want = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, 0.0, beam)
        assert (want["parent"][:beam] == 7).all()
        _compare(_call(x, ld, V, st, S, beam, 2, 0.0), want, st)


def test_long_histories_in_place():
    """Histories of several windows of the merge's shared memory, taking the old ones' place."""
    S, beam, V, cap = 2, 32, 70, 420
    rng = np.random.default_rng(13)
    st = _state(rng, S, beam, V, 400, cap, done_share=0.3)
    x = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32) * 3)
    want = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, 0.6, beam)
    _compare(_call(x, V, V, st, S, beam, 2, 0.6, in_place=True), want, st, in_place=True)


def test_first_step_masks_and_too_few_candidates():
    """One live slot; masked tokens of every kind; rows with fewer candidates than slots, or none."""
    beam, V, S = 4, 300, 5
    inf, low = float("inf"), torch.finfo(torch.float32).min
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32))
    st = _state(rng, S, beam, V, 1, 4, done_share=0.0)
    st["score"][np.arange(S * beam) % beam > 0] = -np.inf
    x[0, ::2] = -inf                       # sentence 0: half of the tokens masked
    x[0, 1::4] = float("nan")              # and a quarter holds NaN
    x[4, 2:] = -inf                        # sentence 1: two tokens for four slots
    x[8] = -inf                            # sentence 2: none
    x[12, :] = low; x[12, 7] = 0.0         # sentence 3: the type's lowest value as a mask
    x[16, 5] = inf; x[16, 9] = inf         # sentence 4: two infinities share the row
    for h in (True, False):
        want = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, 0.6, beam)
        got = _call(x, V, V, st, S, beam, 2, 0.6, history=h)
        _compare(got, want, st, history=h)
    assert (want["next"][8:12] == 2).all() and (want["done"][8:12] == 1).all()
    assert list(want["next"][16:18]) == [5, 9]


def test_finished_hypotheses_and_no_eos():
    """All finished: nothing moves but the order.  Without eos nothing finishes."""
    S, beam, V = 3, 4, 500
    rng = np.random.default_rng(8)
    x = torch.full((S * beam, V), float("nan"))            # logits of finished hypotheses are not used
    st = _state(rng, S, beam, V, 5, 5, done_share=1.1)
    want = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, 1.0, beam)
    _compare(_call(x, V, V, st, S, beam, 2, 1.0), want, st)
    x = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32))
    st = _state(rng, S, beam, V, 5, 8, done_share=0.3)
    want = select(x, st["score"], st["len"], st["done"], st["tokens"], -1, 1.0, beam)
    _compare(_call(x, V, V, st, S, beam, -1, 1.0), want, st)


def test_in_place_over_several_steps_and_another_stream():
    """The state's own buffers as outputs, step after step, on a stream of its own."""
    S, beam, V, cap = 6, 5, 900, 700
    rng = np.random.default_rng(11)
    st = _state(rng, S, beam, V, 300, cap, done_share=0.1)
    stream = torch.cuda.Stream()
    for step in range(3):
        x = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32) * 3)
        want = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, 0.6, beam)
        torch.cuda.synchronize()
        got = _call(x, V, V, st, S, beam, 2, 0.6, in_place=True, stream=stream)
        _compare(got, want, st, in_place=True)
        st = {k: got[k] for k in st}


def test_captured_and_replayed_with_new_inputs():
    S, beam, V = 4, 4, 5000
    rng = np.random.default_rng(21)
    st = _state(rng, S, beam, V, 6, 9)
    d = {k: torch.from_numpy(np.array(v)).to(DEV) for k, v in st.items()}
    o = {k: torch.full_like(v, -7) for k, v in d.items()}
    x = torch.zeros(S * beam, V, device=DEV)
    parent, nxt = torch.zeros_like(d["len"]), torch.zeros_like(d["len"])
    rc, n = B.san_beam_select_bytes(S, beam, V)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    a = B.select_args(dtype=B.SAN_F32, n_sent=S, beam=beam, vocab=V, d_logits=x, ld_logits=V, eos=2, alpha=0.6, d_score=d["score"],
                      d_len=d["len"], d_done=d["done"], d_tokens=d["tokens"], ld_tokens=9, d_score_out=o["score"], d_len_out=o["len"],
                      d_done_out=o["done"], d_tokens_out=o["tokens"], d_parent=parent, d_next=nxt, d_workspace=ws, workspace_bytes=n)
    B.check(B.san_beam_select(a))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.check(B.san_beam_select(a))
    for _ in range(2):
        y = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32))
        x.copy_(y)
        for v in o.values():
            v.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        got = {k: v.cpu().numpy() for k, v in o.items()} | {"parent": parent.cpu().numpy(), "next": nxt.cpu().numpy()}
        _compare(got, select(y, st["score"], st["len"], st["done"], st["tokens"], 2, float(np.float32(0.6)), beam), st)


def test_a_bad_length_skips_its_sentence_and_is_reported():
    S, beam, V, cap = 3, 4, 600, 8
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32))
    for bad in (-1, cap + 1, cap):                          # the last: no room for a token
        st = _state(rng, S, beam, V, 5, cap, done_share=0.0)
        good = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, 0.6, beam)
        st["len"][beam + 2] = bad
        status = torch.zeros(8, dtype=torch.int32, device=DEV)
        got = _call(x, V, V, st, S, beam, 2, 0.6, status=status)
        assert status.cpu().tolist()[:4] == [B.SAN_ERR_DEVICE_CHECK, 8, beam + 2, bad]
        rows = np.r_[0:beam, 2 * beam:3 * beam]
        for k in ("parent", "next", "len", "done"):
            assert np.array_equal(got[k][rows], good[k][rows]), k
            assert (got[k][beam:2 * beam] == (-9 if k in ("parent", "next") else -7)).all()
        assert (got["tokens"][beam:2 * beam] == -7).all()


@pytest.mark.parametrize("alpha", [32.0, -32.0, 130.0, -130.0])
def test_large_length_exponents(alpha):
    """Ranks far from 1 (down to (405 / 6)^-130 = 10^-238): the choice and the scores are those of the definition."""
    S, beam, V = 2, 4, 50
    rng = np.random.default_rng(31)
    st = _state(rng, S, beam, V, 400, 410, done_share=0.3)
    x = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32) * 2)
    want = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, alpha, beam)
    _compare(_call(x, V, V, st, S, beam, 2, alpha), want, st)


@pytest.mark.parametrize("alpha", [300.0, -300.0, 1e38])
def test_an_exponent_beyond_the_range_of_ranks_is_reported(alpha):
    """(405 / 6)^300 is no number of 64 bits: the sentence is skipped; one of length 0 (5 / 6, 6 / 6) is answered at 300."""
    S, beam, V, cap = 2, 4, 50, 410
    rng = np.random.default_rng(32)
    st = _state(rng, S, beam, V, 400, cap, done_share=0.0)
    st["len"][beam:] = 0
    x = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32))
    want = select(x, st["score"], st["len"] * 0, st["done"], st["tokens"], 2, 1.0, beam)
    status = torch.zeros(8, dtype=torch.int32, device=DEV)
    got = _call(x, V, V, st, S, beam, 2, alpha, status=status)
    found = status.cpu().tolist()
    assert found[:2] == [B.SAN_ERR_DEVICE_CHECK, 8] and 0 <= found[2] < beam and found[3] == 400
    for k in ("parent", "next", "len", "done"):
        assert (got[k][:beam] == (-9 if k in ("parent", "next") else -7)).all(), k
        assert np.array_equal(got[k][beam:], want[k][beam:]), k        # ((5 + 1) / 6)^alpha = 1 for every alpha
    live = np.abs(got["score"][beam:] - want["score"][beam:])
    assert (live <= 2.0 ** -20 + 2.0 ** -23 * np.abs(want["score"][beam:])).all()


def test_a_batch_that_shrinks_in_the_workspace_of_its_beginning():
    beam, V, S = 4, 9000, 60
    rng = np.random.default_rng(41)
    x = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32) * 2)
    st = _state(rng, S, beam, V, 5, 8)
    dx, d = x.to(DEV), {k: torch.from_numpy(np.array(v)).to(DEV) for k, v in st.items()}
    rc, size = B.san_beam_select_bytes(S, beam, V)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    for n in (60, 37, 9, 1):
        o = {k: torch.full_like(v, -7) for k, v in d.items()}
        parent, nxt = torch.full_like(d["len"], -9), torch.full_like(d["len"], -9)
        a = B.select_args(dtype=B.SAN_F32, n_sent=n, beam=beam, vocab=V, d_logits=dx, ld_logits=V, eos=2, alpha=0.6, d_score=d["score"],
                          d_len=d["len"], d_done=d["done"], d_tokens=d["tokens"], ld_tokens=8, d_score_out=o["score"],
                          d_len_out=o["len"], d_done_out=o["done"], d_tokens_out=o["tokens"], d_parent=parent, d_next=nxt,
                          d_workspace=ws, workspace_bytes=size)
        B.check(B.san_beam_select(a))
        torch.cuda.synchronize()
        rows = n * beam
        part = {k: v[:rows] for k, v in st.items()}
        want = select(x[:rows], part["score"], part["len"], part["done"], part["tokens"], 2, float(np.float32(0.6)), beam)
        got = {k: v.cpu().numpy()[:rows] for k, v in o.items()} | {"parent": parent.cpu().numpy()[:rows], "next": nxt.cpu().numpy()[:rows]}
        _compare(got, want, part)
        assert (parent[rows:] == -9).all() and (o["tokens"][rows:] == -7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,V", [(512, 128000), (592, 1 << 20)])
def test_sums_of_long_rows_do_not_drift(dtype, S, V):
    """One long part a row, with terms that are all alike: what each addition rounds off has the same sign.  Beam 1, so that the
    scores are the sums."""
    dt, code = dtype_of(dtype)
    val = (-0.05 - torch.arange(S, device=DEV) % 512 * 0.0137).to(dt)
    x = val[:, None].repeat(1, V)
    x[:, :8192] = 0.0                                       # every thread's maximum
    i32 = lambda n: torch.full((S,), n, dtype=torch.int32, device=DEV)       # noqa: E731
    d = dict(d_score=torch.full((S,), -1.0, device=DEV), d_len=i32(3), d_done=i32(0))
    o = dict(d_score_out=torch.zeros(S, device=DEV), d_len_out=i32(-7), d_done_out=i32(-7), d_parent=i32(-9), d_next=i32(-9))
    rc, n = B.san_beam_select_bytes(S, 1, V)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    B.check(B.san_beam_select(B.select_args(dtype=code, n_sent=S, beam=1, vocab=V, d_logits=x, ld_logits=V, eos=-1, alpha=0.0,
                                            d_workspace=ws, workspace_bytes=n, **d, **o)))
    torch.cuda.synchronize()
    z = val.double()
    want = -1.0 - (8192 + (V - 8192) * z.exp()).log()
    # a term: the exponential within 2^-22, its argument z log2(e) rounded by half a step (|z| 2^-24 of the term); up to nine
    # additions within a step; the sum's relative error is the logarithm's absolute one; the score is rounded once
    bound = 2.0 ** -22 + z.abs() * 2.0 ** -24 + 9 * 2.0 ** -24 + 2.0 ** -24 * want.abs()
    assert (o["d_next"] == 0).all()
    assert ((o["d_score_out"].double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sums_of_rising_rows(dtype):
    """The maximum moves with every step, by little: sums are not rescaled each time."""
    beam, V, rows = 1, 128000, 3
    x = torch.stack([torch.arange(V) * s for s in (1e-5, 1e-4, 1e-3)]).to(dtype_of(dtype)[0])
    st = dict(score=np.full(rows, -1.0, np.float32), len=np.full(rows, 3, np.int32), done=np.zeros(rows, np.int32),
              tokens=np.zeros((rows, 5), np.int32))
    want = select(x, st["score"], st["len"], st["done"], st["tokens"], -1, 0.0, beam)
    _compare(_call(x, V, V, st, rows, beam, -1, 0.0), want, st)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_token_alone_has_all_of_the_probability(dtype):
    """Rows with one token, or one that is not masked, offer it at the hypothesis' own score: they tie with one another and with
    finished hypotheses, whatever the logit."""
    S, beam = 40, 16
    rng = np.random.default_rng(51)
    for V in (1, 3000):
        x = torch.full((S * beam, V), -float("inf"))
        at = torch.from_numpy(rng.integers(0, V, S * beam))
        x[torch.arange(S * beam), at] = torch.from_numpy(rng.standard_normal(S * beam, dtype=np.float32) * 10)
        x = x.to(dtype_of(dtype)[0])
        st = _state(rng, S, beam, V, 6, 9, done_share=0.3)
        st["score"][:] = -1.5
        st["len"][st["done"] == 0] = 5
        want = select(x, st["score"], st["len"], st["done"], st["tokens"], -1, 0.0, beam)
        got = _call(x, V, V, st, S, beam, -1, 0.0)
        _compare(got, want, st)
        assert (got["score"] == -1.5).all() and np.array_equal(got["parent"], np.tile(np.arange(beam), S))


def test_on_another_stream_behind_its_inputs():
    """As test_in_place_over_several_steps_and_another_stream, the side stream waiting for what fills the buffers."""
    S, beam, V = 6, 5, 900
    rng = np.random.default_rng(61)
    st = _state(rng, S, beam, V, 30, 40, done_share=0.1)
    x = torch.from_numpy(rng.standard_normal((S * beam, V), dtype=np.float32) * 3)
    want = select(x, st["score"], st["len"], st["done"], st["tokens"], 2, float(np.float32(0.6)), beam)
    side = torch.cuda.Stream()
    dx, d = torch.empty(S * beam, V, device=DEV), {k: torch.from_numpy(np.array(v)).to(DEV) for k, v in st.items()}
    dx.copy_(x)
    o = {k: torch.full_like(v, -7) for k, v in d.items()}
    parent, nxt = torch.full_like(d["len"], -9), torch.full_like(d["len"], -9)
    rc, n = B.san_beam_select_bytes(S, beam, V)
    ws = torch.full((n,), 0xA5, dtype=torch.uint8, device=DEV)
    a = B.select_args(dtype=B.SAN_F32, n_sent=S, beam=beam, vocab=V, d_logits=dx, ld_logits=V, eos=2, alpha=0.6, d_score=d["score"],
                      d_len=d["len"], d_done=d["done"], d_tokens=d["tokens"], ld_tokens=40, d_score_out=o["score"], d_len_out=o["len"],
                      d_done_out=o["done"], d_tokens_out=o["tokens"], d_parent=parent, d_next=nxt, d_workspace=ws, workspace_bytes=n)
    side.wait_stream(torch.cuda.current_stream())
    B.check(B.san_beam_select(a, side))
    side.synchronize()
    got = {k: v.cpu().numpy() for k, v in o.items()} | {"parent": parent.cpu().numpy(), "next": nxt.cpu().numpy()}
    _compare(got, want, st)
