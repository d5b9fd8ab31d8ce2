"""Refusals and sizes of the calls for long prompts and small caches that need no GPU: every call below fails its host checks
(or has nothing to do) before a device is touched."""
import pytest

from paper_1906_11024_b200 import binding as B
from paper_1906_11024_b200 import build as san_build

FAKE = 0x10000          # an aligned address that is never dereferenced
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def _built():
    san_build.build()
    B.lib()


def _packed(**kw):
    a = dict(dtype=B.SAN_BF16, n_heads=8, n_kv_heads=2, n_layers=2, d_q=FAKE, ld_q=512, d_k=FAKE, ld_k=128, d_v=FAKE, ld_v=128, v_stride=128000,
             d_first=FAKE, n_seq=3, n_tokens=1000, max_len=0, d_out=FAKE)
    return B.packed_args(**(a | kw))


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=B.SAN_F32), B.SAN_ERR_UNSUPPORTED), (dict(dtype=B.SAN_Q4), B.SAN_ERR_DTYPE), (dict(n_heads=0), B.SAN_ERR_SHAPE),
    (dict(n_kv_heads=3), B.SAN_ERR_SHAPE), (dict(n_kv_heads=0), B.SAN_ERR_SHAPE), (dict(n_layers=0), B.SAN_ERR_SHAPE),
    (dict(n_layers=65), B.SAN_ERR_SHAPE), (dict(n_seq=-1), B.SAN_ERR_SHAPE), (dict(n_tokens=-1), B.SAN_ERR_SHAPE),
    (dict(max_len=1001), B.SAN_ERR_SHAPE), (dict(max_len=-1), B.SAN_ERR_SHAPE), (dict(ld_q=504), B.SAN_ERR_SHAPE), (dict(ld_q=516), B.SAN_ERR_SHAPE),
    (dict(ld_k=120), B.SAN_ERR_SHAPE), (dict(ld_v=132), B.SAN_ERR_SHAPE), (dict(v_stride=0), B.SAN_ERR_SHAPE), (dict(v_stride=4), B.SAN_ERR_SHAPE),
    (dict(d_q=None), B.SAN_ERR_NULL), (dict(d_first=None), B.SAN_ERR_NULL), (dict(d_out=None), B.SAN_ERR_NULL), (dict(d_k=FAKE + 8), B.SAN_ERR_SHAPE),
    (dict(n_seq=0, d_q=None), B.SAN_OK), (dict(n_tokens=0, d_q=None), B.SAN_OK), (dict(n_tokens=1 << 29), B.SAN_ERR_SHAPE),
    (dict(max_len=100, n_seq=70000), B.SAN_ERR_SHAPE),
])
def test_packed_refusals(kw, status):
    assert B.san_packed_block(_packed(**kw), FAKE, BIG, stream=0) == status


def test_packed_workspace():
    rc, n = B.san_packed_block_bytes(_packed())
    assert rc == B.SAN_OK and n > 0
    assert B.san_packed_block(_packed(), None, n, stream=0) == B.SAN_ERR_NULL
    assert B.san_packed_block(_packed(), FAKE + 16, n, stream=0) == B.SAN_ERR_SHAPE
    assert B.san_packed_block(_packed(), FAKE, n - 1, stream=0) == B.SAN_ERR_CAPACITY
    assert B.san_packed_block_bytes(_packed(n_seq=1)) == (B.SAN_OK, 0)         # nothing to sort
    assert B.san_packed_block_bytes(_packed(max_len=100)) == (B.SAN_OK, 0)
    assert B.lib().san_packed_block(None, None, 0, None) == B.SAN_ERR_NULL
    assert B.lib().san_packed_block_bytes(None, None) == B.SAN_ERR_NULL
    for kw in (dict(n_seq=4), dict(n_tokens=4000)):                            # a larger batch's workspace serves smaller ones
        assert B.san_packed_block_bytes(_packed(**kw))[1] >= n


def _planes(**kw):
    a = dict(dtype=B.SAN_Q4, n_kv_heads=2, n_layers=2, d_k=FAKE, d_v=FAKE, v_stride=64 * 800, d_k_scale=FAKE, d_v_scale=FAKE, max_ids=4, cap_len=100)
    return B.planes(**(a | kw))


BAD_PLANES = [(dict(dtype=7), B.SAN_ERR_DTYPE), (dict(n_kv_heads=0), B.SAN_ERR_SHAPE), (dict(n_layers=0), B.SAN_ERR_SHAPE),
              (dict(n_layers=65), B.SAN_ERR_SHAPE), (dict(max_ids=0), B.SAN_ERR_SHAPE), (dict(cap_len=0), B.SAN_ERR_SHAPE),
              (dict(v_stride=0), B.SAN_ERR_SHAPE), (dict(v_stride=100), B.SAN_ERR_SHAPE), (dict(d_k=None), B.SAN_ERR_NULL),
              (dict(d_v=FAKE + 8), B.SAN_ERR_SHAPE), (dict(d_k_scale=None), B.SAN_ERR_NULL), (dict(d_v_scale=FAKE + 2), B.SAN_ERR_SHAPE)]


def _rows(call, planes=None, dtype=B.SAN_BF16, k=FAKE, v=FAKE, ids=FAKE, n=3, rows=5):
    return call(planes or _planes(), dtype, k, v, ids, None, None, n, rows, None, stream=0)


@pytest.mark.parametrize("call", [B.san_quant_append, B.san_quant_read])
def test_quant_rows_refusals(call):
    for kw, status in BAD_PLANES + [(dict(dtype=B.SAN_BF16), B.SAN_ERR_DTYPE)]:
        assert _rows(call, _planes(**kw)) == status, kw
    for kw, status in [(dict(dtype=B.SAN_Q4), B.SAN_ERR_DTYPE), (dict(n=-1), B.SAN_ERR_SHAPE), (dict(rows=0), B.SAN_ERR_SHAPE),
                       (dict(rows=101), B.SAN_ERR_SHAPE), (dict(k=None), B.SAN_ERR_NULL), (dict(v=None), B.SAN_ERR_NULL),
                       (dict(ids=None), B.SAN_ERR_NULL), (dict(k=FAKE + 4), B.SAN_ERR_SHAPE), (dict(n=0, k=None), B.SAN_OK),
                       (dict(n=0x7fffffff, rows=100), B.SAN_ERR_SHAPE)]:
        assert _rows(call, **kw) == status, kw


def test_quant_rows_wider_than_the_cache():
    """With counts of their own the items' rows may lie further apart than the cache is long."""
    for call in (B.san_quant_append, B.san_quant_read):
        got = call(_planes(), B.SAN_BF16, FAKE, FAKE, FAKE, None, FAKE, 0, 101, None, stream=0)
        assert got == B.SAN_OK
        assert call(_planes(), B.SAN_BF16, None, FAKE, FAKE, None, FAKE, 3, 101, None, stream=0) == B.SAN_ERR_NULL
        assert call(_planes(), B.SAN_BF16, FAKE, FAKE, FAKE, None, FAKE, 3, 0x7fffffff, None, stream=0) == B.SAN_ERR_SHAPE


def _step(**kw):
    a = dict(dtype=B.SAN_BF16, n_heads=8, d_q=FAKE, d_ids=FAKE, d_lens=FAKE, n_items=4, max_len=0, d_out=FAKE)
    return B.step_rows(**(a | kw))


def test_quant_attention_refusals():
    for kw, status in BAD_PLANES + [(dict(dtype=B.SAN_F32), B.SAN_ERR_DTYPE)]:
        assert B.san_quant_attn(_planes(**kw), _step(), FAKE, BIG, stream=0) == status, kw
    for kw, status in [(dict(dtype=B.SAN_Q4), B.SAN_ERR_DTYPE), (dict(n_heads=0), B.SAN_ERR_SHAPE), (dict(n_heads=7), B.SAN_ERR_SHAPE),
                       (dict(n_items=-1), B.SAN_ERR_SHAPE), (dict(max_len=101), B.SAN_ERR_SHAPE), (dict(d_q=None), B.SAN_ERR_NULL),
                       (dict(d_lens=None), B.SAN_ERR_NULL), (dict(d_out=FAKE + 8), B.SAN_ERR_SHAPE), (dict(d_S=FAKE, ld_s=99), B.SAN_ERR_SHAPE),
                       (dict(d_S=FAKE + 2, ld_s=100), B.SAN_ERR_SHAPE), (dict(n_items=0, d_q=None), B.SAN_OK)]:
        assert B.san_quant_attn(_planes(), _step(**kw), FAKE, BIG, stream=0) == status, kw
    rows = _step(d_S=FAKE, ld_s=100)
    rc, n = B.san_quant_attn_bytes(_planes(), rows)
    assert rc == B.SAN_OK and n > 0                                            # (max, sum) of every row for the weights
    assert B.san_quant_attn(_planes(), rows, None, n, stream=0) == B.SAN_ERR_NULL
    assert B.san_quant_attn(_planes(), rows, FAKE + 64, n, stream=0) == B.SAN_ERR_SHAPE
    assert B.san_quant_attn(_planes(), rows, FAKE, n - 1, stream=0) == B.SAN_ERR_CAPACITY
    assert B.lib().san_quant_attn(None, None, None, 0, None) == B.SAN_ERR_NULL
    assert B.lib().san_quant_attn_bytes(_planes(), None, None) == B.SAN_ERR_NULL


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("H,Hk,L", [(8, 8, 4), (16, 4, 1), (20, 1, 9)])
def test_quant_attention_workspace_holds_for_everything_smaller(H, Hk, L, weights):
    """A decoder's batch shrinks while its workspace stays."""
    def size(n, cap):
        kw = dict(d_S=FAKE, ld_s=cap) if weights else {}
        rc, b = B.san_quant_attn_bytes(_planes(n_kv_heads=Hk, n_layers=L, cap_len=cap), _step(n_heads=H, n_items=n, **kw))
        assert rc == B.SAN_OK
        return b

    for cap in (100, 4096, 131072):
        sizes = [size(n, cap) for n in list(range(0, 200)) + [256, 500, 1000, 5000]]
        assert sizes == sorted(sizes)
    sizes = [size(64, cap) for cap in range(1, 70000, 331)]
    assert sizes == sorted(sizes)


def _mass(**kw):
    a = dict(n_heads=8, n_kv_heads=2, d_S=FAKE, item_stride=800, row_stride=0, head_stride=100, n_rows=1, d_ids=FAKE, d_lens=FAKE, n_items=4,
             max_len=100, decay=0.9, d_mass=FAKE, ld_mass=100, max_ids=4)
    return B.mass_args(**(a | kw))


@pytest.mark.parametrize("kw,status", [
    (dict(n_heads=0), B.SAN_ERR_SHAPE), (dict(n_kv_heads=3), B.SAN_ERR_SHAPE), (dict(n_rows=-1), B.SAN_ERR_SHAPE), (dict(n_items=-1), B.SAN_ERR_SHAPE),
    (dict(n_items=65536), B.SAN_ERR_SHAPE), (dict(max_len=-1), B.SAN_ERR_SHAPE), (dict(max_len=101), B.SAN_ERR_SHAPE), (dict(max_ids=0), B.SAN_ERR_SHAPE),
    (dict(decay=float("nan")), B.SAN_ERR_SHAPE), (dict(decay=float("inf")), B.SAN_ERR_SHAPE), (dict(d_S=None), B.SAN_ERR_NULL),
    (dict(d_ids=None), B.SAN_ERR_NULL), (dict(d_mass=None), B.SAN_ERR_NULL), (dict(d_mass=FAKE + 2), B.SAN_ERR_SHAPE), (dict(n_items=0, d_S=None), B.SAN_OK),
])
def test_mass_refusals(kw, status):
    assert B.san_weight_mass(_mass(**kw), stream=0) == status
    assert B.lib().san_weight_mass(None, None) == B.SAN_ERR_NULL


def _evict(**kw):
    a = dict(d_ids=FAKE, d_lens=FAKE, n_items=4, max_len=0, n_keep=50, n_sink=4, n_recent=10, d_mass=FAKE, ld_mass=100, d_lens_out=FAKE)
    return B.evict_args(**(a | kw))


def test_evict_refusals():
    for kw, status in BAD_PLANES:
        assert B.san_cache_evict(_planes(**kw), _evict(), FAKE, BIG, stream=0) == status, kw
    for dtype in (B.SAN_F32, B.SAN_BF16):                                      # rows that have no scales
        assert B.san_cache_evict(_planes(dtype=dtype, d_k_scale=None, d_v_scale=None), _evict(), None, BIG, stream=0) == B.SAN_ERR_NULL
        assert B.san_cache_evict(_planes(dtype=dtype, d_k_scale=None, d_v_scale=None), _evict(n_items=0), None, 0, stream=0) == B.SAN_OK
    for kw, status in [(dict(n_items=-1), B.SAN_ERR_SHAPE), (dict(n_items=65536), B.SAN_ERR_SHAPE), (dict(max_len=101), B.SAN_ERR_SHAPE),
                       (dict(n_keep=0), B.SAN_ERR_SHAPE), (dict(n_keep=13), B.SAN_ERR_SHAPE), (dict(n_sink=-1), B.SAN_ERR_SHAPE),
                       (dict(n_recent=-1), B.SAN_ERR_SHAPE), (dict(n_recent=0x7fffffff), B.SAN_ERR_SHAPE), (dict(ld_mass=99), B.SAN_ERR_SHAPE),
                       (dict(d_kept=FAKE, ld_kept=49), B.SAN_ERR_SHAPE), (dict(d_ids=None), B.SAN_ERR_NULL), (dict(d_mass=None), B.SAN_ERR_NULL),
                       (dict(d_lens_out=None), B.SAN_ERR_NULL), (dict(n_keep=1 << 27), B.SAN_ERR_SHAPE), (dict(n_items=0, d_ids=None), B.SAN_OK)]:
        assert B.san_cache_evict(_planes(), _evict(**kw), FAKE, BIG, stream=0) == status, kw
    rc, n = B.san_cache_evict_bytes(_planes(), _evict())
    assert rc == B.SAN_OK and n >= 4 * 2 * 50 * 4
    assert B.san_cache_evict(_planes(), _evict(), None, n, stream=0) == B.SAN_ERR_NULL
    assert B.san_cache_evict(_planes(), _evict(), FAKE + 4, n, stream=0) == B.SAN_ERR_SHAPE
    assert B.san_cache_evict(_planes(), _evict(), FAKE, n - 1, stream=0) == B.SAN_ERR_CAPACITY
    assert B.lib().san_cache_evict(None, None, None, 0, None) == B.SAN_ERR_NULL
    assert B.lib().san_cache_evict_bytes(_planes(), _evict(), None) == B.SAN_ERR_NULL


def test_mass_bound_of_zero_is_the_mass_itself():
    """As in the other calls: no bound given is the bound of the buffer, not "no rows"."""
    assert B.san_weight_mass(_mass(max_len=0, d_S=None), stream=0) == B.SAN_ERR_NULL
    assert B.san_weight_mass(_mass(max_len=0, ld_mass=(1 << 28) + 1), stream=0) == B.SAN_ERR_SHAPE
    assert B.san_weight_mass(_mass(max_len=0, ld_mass=0, d_S=None), stream=0) == B.SAN_OK         # a mass of no rows
    assert B.san_weight_mass(_mass(max_len=0, ld_mass=-1), stream=0) == B.SAN_ERR_SHAPE


def test_packed_more_sequences_than_are_counted():
    """Counts of tiles are 31 bits: n_tokens / 256 + n_seq was formed in as many and came out negative."""
    for n_seq, n_tokens in (((1 << 28) + 1, 1000), (0x7fffffff, 1000), (0x7fffffff, 1 << 28)):
        a = _packed(n_seq=n_seq, n_tokens=n_tokens, n_heads=1, n_kv_heads=1, n_layers=1)
        assert B.san_packed_block_bytes(a)[0] == B.SAN_ERR_SHAPE
        assert B.san_packed_block(a, FAKE, BIG, stream=0) == B.SAN_ERR_SHAPE
    rc, n = B.san_packed_block_bytes(_packed(n_seq=1 << 28, n_tokens=1 << 28))
    assert rc == B.SAN_OK and n == 16 * (1 + (1 << 20) + (1 << 28))
