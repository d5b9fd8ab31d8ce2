"""Refusals and sizes of the calls around the decode step that need no GPU: every call below fails its host checks
(or has nothing to do) before a device is touched."""
import pytest

from paper_1906_11024_b200 import binding as B
from paper_1906_11024_b200 import build as san_build

FAKE = 0x10000          # an aligned address that is never dereferenced


@pytest.fixture(scope="module", autouse=True)
def _built():
    san_build.build()
    B.lib()


def _select(**kw):
    a = dict(dtype=B.SAN_F32, n_sent=2, beam=4, vocab=100, d_logits=FAKE, ld_logits=100, eos=2, alpha=0.6, d_score=FAKE, d_len=FAKE,
             d_done=FAKE, d_tokens=FAKE, ld_tokens=10, d_score_out=FAKE, d_len_out=FAKE, d_done_out=FAKE, d_tokens_out=FAKE,
             d_parent=FAKE, d_next=FAKE, d_workspace=FAKE, workspace_bytes=1 << 20)
    return B.san_beam_select(B.select_args(**(a | kw)), stream=0)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), B.SAN_ERR_DTYPE), (dict(n_sent=-1), B.SAN_ERR_SHAPE), (dict(beam=0), B.SAN_ERR_SHAPE),
    (dict(beam=B.SAN_MAX_BEAM + 1), B.SAN_ERR_SHAPE), (dict(vocab=0), B.SAN_ERR_SHAPE), (dict(ld_logits=99), B.SAN_ERR_SHAPE),
    (dict(eos=100), B.SAN_ERR_SHAPE), (dict(eos=-2), B.SAN_ERR_SHAPE), (dict(alpha=float("nan")), B.SAN_ERR_SHAPE),
    (dict(alpha=float("inf")), B.SAN_ERR_SHAPE), (dict(d_logits=None), B.SAN_ERR_NULL), (dict(d_logits=FAKE + 2), B.SAN_ERR_SHAPE),
    (dict(d_score=None), B.SAN_ERR_NULL), (dict(d_next=None), B.SAN_ERR_NULL), (dict(d_tokens=None), B.SAN_ERR_NULL),
    (dict(d_tokens_out=None), B.SAN_ERR_NULL), (dict(ld_tokens=0), B.SAN_ERR_SHAPE), (dict(d_workspace=None), B.SAN_ERR_NULL),
    (dict(d_workspace=FAKE + 16), B.SAN_ERR_SHAPE), (dict(workspace_bytes=16), B.SAN_ERR_CAPACITY),
    (dict(n_sent=1 << 23, beam=32), B.SAN_ERR_SHAPE), (dict(n_sent=0, d_logits=None), B.SAN_OK),
])
def test_select_refusals(kw, status):
    assert _select(**kw) == status


def test_select_refuses_histories_past_its_indices():
    assert _select(ld_tokens=0x7fff0001) == B.SAN_ERR_SHAPE and _select(ld_tokens=0x7ffffffe) == B.SAN_ERR_SHAPE
    assert _select(ld_tokens=0x7fff0000, workspace_bytes=16) == B.SAN_ERR_CAPACITY      # taken, and refused for the next reason


def test_select_workspace():
    rc, n = B.san_beam_select_bytes(64, 4, 32000)
    assert rc == B.SAN_OK and n % (256 * (16 + 8 * 4)) == 0      # whole parts of rows: a maximum, a sum and four keys each
    rc, n = B.san_beam_select_bytes(1, 4, 32000)
    assert rc == B.SAN_OK and n % (4 * (16 + 8 * 4)) == 0 and n > 4 * (16 + 8 * 4)      # few rows: several parts each
    assert B.san_beam_select_bytes(1, 0, 10)[0] == B.SAN_ERR_SHAPE
    assert B.lib().san_beam_select_bytes(1, 1, 10, None) == B.SAN_ERR_NULL
    assert B.lib().san_beam_select(None, None) == B.SAN_ERR_NULL


def _rows(**kw):
    a = dict(dtype=B.SAN_BF16, n_heads=8, n_kv_heads=2, n_layers=2, d_q=FAKE, d_k=FAKE, d_v=FAKE, v_stride=64 * 100, max_ids=4, cap_len=100,
             d_ids=FAKE, d_lens=FAKE, n_items=4, max_len=0, d_out=FAKE)
    return B.cached_rows(**(a | kw))


def _pre(**kw):
    a = dict(d_k=FAKE, d_v=FAKE, v_stride=6400, n_prefix=2, cap_len=50, d_lens=FAKE, max_len=0, d_first=FAKE, max_group=0)
    return B.shared_prefix(**(a | kw))


BAD_ROWS = [
    (dict(dtype=5), B.SAN_ERR_DTYPE), (dict(n_heads=0), B.SAN_ERR_SHAPE), (dict(n_kv_heads=3), B.SAN_ERR_SHAPE),
    (dict(n_kv_heads=0), B.SAN_ERR_SHAPE), (dict(n_layers=0), B.SAN_ERR_SHAPE), (dict(n_layers=65), B.SAN_ERR_SHAPE),
    (dict(max_ids=0), B.SAN_ERR_SHAPE), (dict(cap_len=0), B.SAN_ERR_SHAPE), (dict(n_items=-1), B.SAN_ERR_SHAPE),
    (dict(max_len=101), B.SAN_ERR_SHAPE), (dict(v_stride=0), B.SAN_ERR_SHAPE), (dict(v_stride=6401), B.SAN_ERR_SHAPE),
    (dict(d_q=None), B.SAN_ERR_NULL), (dict(d_lens=None), B.SAN_ERR_NULL), (dict(d_out=FAKE + 8), B.SAN_ERR_SHAPE),
    (dict(d_k=FAKE + 2), B.SAN_ERR_SHAPE), (dict(n_items=0, d_q=None), B.SAN_OK),
]


@pytest.mark.parametrize("kw,status", BAD_ROWS)
def test_step_attention_refusals(kw, status):
    r = _rows(**kw)
    big = 1 << 40
    assert B.san_window_attn(r, 16, 1, FAKE, big, stream=0) == status
    x = _pre(max_group=0)
    assert B.san_prefix_attn(r, x, FAKE, big, stream=0) == status


def test_window_prefix_and_workspace_refusals():
    r, big = _rows(), 1 << 40
    assert B.san_window_attn(r, 0, 1, FAKE, big, stream=0) == B.SAN_ERR_SHAPE
    assert B.san_window_attn(r, 1, -1, FAKE, big, stream=0) == B.SAN_ERR_SHAPE
    assert B.lib().san_window_attn(None, 1, 0, FAKE, big, None) == B.SAN_ERR_NULL
    for kw, status in [(dict(n_prefix=-1), B.SAN_ERR_SHAPE), (dict(cap_len=0), B.SAN_ERR_SHAPE), (dict(max_len=51), B.SAN_ERR_SHAPE),
                       (dict(max_group=5), B.SAN_ERR_SHAPE), (dict(v_stride=63), B.SAN_ERR_SHAPE), (dict(d_k=None), B.SAN_ERR_NULL),
                       (dict(d_first=None), B.SAN_ERR_NULL), (dict(d_v=FAKE + 8), B.SAN_ERR_SHAPE)]:
        assert B.san_prefix_attn(r, _pre(**kw), FAKE, big, stream=0) == status, kw
    rc, n = B.san_prefix_attn_bytes(r, _pre())
    assert rc == B.SAN_OK and n > 0
    assert B.san_prefix_attn(r, _pre(), None, n, stream=0) == B.SAN_ERR_NULL
    assert B.san_prefix_attn(r, _pre(), FAKE + 16, n, stream=0) == B.SAN_ERR_SHAPE
    assert B.san_prefix_attn(r, _pre(), FAKE, n - 1, stream=0) == B.SAN_ERR_CAPACITY
    # a short window is one unit per row and key head: no partial results, no workspace
    assert B.san_window_attn_bytes(r, 16, 1) == (B.SAN_OK, 0)


def test_window_block_refusals():
    def f(dtype=B.SAN_BF16, H=4, Hk=2, L=1, window=8, sink=1, q=FAKE, k=FAKE, v=FAKE, lens=FAKE, n=1, cap=10, m=0, out=FAKE):
        return B.san_window_block(dtype, H, Hk, L, window, sink, q, k, v, lens, n, cap, m, out, stream=0)

    for kw, status in [(dict(dtype=B.SAN_F32), B.SAN_ERR_UNSUPPORTED), (dict(dtype=9), B.SAN_ERR_DTYPE), (dict(H=0), B.SAN_ERR_SHAPE),
                       (dict(Hk=3), B.SAN_ERR_SHAPE), (dict(L=0), B.SAN_ERR_SHAPE), (dict(window=0), B.SAN_ERR_SHAPE),
                       (dict(sink=-1), B.SAN_ERR_SHAPE), (dict(n=-1), B.SAN_ERR_SHAPE), (dict(cap=0), B.SAN_ERR_SHAPE),
                       (dict(m=11), B.SAN_ERR_SHAPE), (dict(q=None), B.SAN_ERR_NULL), (dict(lens=None), B.SAN_ERR_NULL),
                       (dict(k=FAKE + 2), B.SAN_ERR_SHAPE), (dict(n=70000, L=2), B.SAN_ERR_SHAPE), (dict(n=0, q=None), B.SAN_OK)]:
        assert f(**kw) == status, kw


def test_select_workspace_holds_for_everything_smaller():
    """A decoder's batch shrinks while its workspace stays."""
    for beam in (1, 4, 20, 32):
        for vocab in (1, 2048, 2049, 32000, 50257, 128000, 1 << 22):
            sizes = [B.san_beam_select_bytes(n, beam, vocab)[1] for n in range(0, 300)]
            assert sizes == sorted(sizes)
    for n in (1, 64, 129):
        sizes = [B.san_beam_select_bytes(n, beam, 32000)[1] for beam in range(1, 33)]
        assert sizes == sorted(sizes)
        sizes = [B.san_beam_select_bytes(n, 4, v)[1] for v in range(1, 140000, 777)]
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("dtype", [B.SAN_F32, B.SAN_BF16])
@pytest.mark.parametrize("H,Hk,L", [(8, 8, 4), (16, 4, 1), (20, 1, 9)])
def test_window_workspace_holds_for_everything_smaller(dtype, H, Hk, L):
    def size(n, cap, window, sink):
        rc, b = B.san_window_attn_bytes(_rows(dtype=dtype, n_heads=H, n_kv_heads=Hk, n_layers=L, n_items=n, cap_len=cap, v_stride=64 * cap), window, sink)
        assert rc == B.SAN_OK
        return b

    for window, sink in ((16, 1), (512, 4), (16384, 5), (1 << 30, 0)):
        for cap in (100, 4096, 131072):
            sizes = [size(n, cap, window, sink) for n in list(range(0, 200)) + [256, 500, 1000, 5000]]
            assert sizes == sorted(sizes)
        sizes = [size(64, cap, window, sink) for cap in range(1, 70000, 331)]
        assert sizes == sorted(sizes)


def test_cache_planes_needs_a_context():
    assert B.san_cache_planes(None, B.SAN_SELF, 0)[0] == B.SAN_ERR_NULL
