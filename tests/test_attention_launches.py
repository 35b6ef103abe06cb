"""The largest calls of the attention layers past the fixed windows, through the C
ABI with the runtime's launch calls recorded: every grid fits, and the launches
together cover the call."""
import pytest

from tests.test_launch_limits import NONE, i32, i64, launches, mem  # noqa: F401  (a fixture)

F32 = lambda v: [["float", v]]  # noqa: E731


def forward(batch, n_q, n_k, heads, kv, hd, stride):
    return (i64(batch, n_q, n_k) + i32(heads, kv, hd, 1) + F32(0.125) + [NONE]
            + [mem(0)] + i64(stride) + [mem(1)] + i64(kv * hd) + [mem(2)] + i64(kv * hd)
            + [mem(3), mem(4)])


@pytest.mark.parametrize("batch,n,heads,kv,hd", [((1 << 24) + 5, 1, 1, 1, 64), (1, 1 << 20, 1024, 8, 64),
                                                 (1 << 16, 129, 128, 1, 64), (3, 1 << 20, 300, 300, 128)])
def test_grouped_forward(launches, batch, n, heads, kv, hd):  # noqa: F811
    ls = launches("hcmix_grouped_attention_forward",
                  forward(batch, n, n, heads, kv, hd, heads * hd) + [NONE])
    per, done = -(-n // 128) * heads, 0
    for (x, y, z), _, q0 in ls:
        assert (y, z) == (1, 1) and x % per == 0
        assert q0 == mem(0)[1] + done * n * heads * hd * 2     # starts where the last one ended
        done += x // per
    assert done == batch


@pytest.mark.parametrize("batch,n,heads,kv,hd", [((1 << 24) + 5, 1, 1, 1, 64), (1, 1 << 20, 256, 8, 64),
                                                 (1 << 16, 129, 128, 1, 64), (2, 4096, 8, 8, 128),
                                                 ((1 << 20) + 5, 1, 8, 8, 128), (1 << 16, 129, 64, 64, 128),
                                                 ((1 << 20) + 5, 1, 8, 8, 64)])
def test_grouped_backward(launches, batch, n, heads, kv, hd):  # noqa: F811
    w, kw = heads * hd, kv * hd
    ls = launches("hcmix_grouped_attention_backward",
                  forward(batch, n, n, heads, kv, hd, w) + [mem(5), mem(6)] + i64(w) + [mem(7)]
                  + i64(kw) + [mem(8)] + i64(kw) + [mem(9), ["size_t", 1 << 39], NONE])
    q = sum(x for (x, _, _), _, _ in ls[0::2])
    keys = sum(x for (x, _, _), _, _ in ls[1::2])
    assert q == batch * -(-n // 128) * heads
    assert keys == batch * -(-n // 128) * kv


def test_key_tiles_that_are_shared(launches):  # noqa: F811
    """Blocks of 64 rows; 32 tiles of keys and 512 steps over the queries: 8 blocks to
    each, and their join."""
    ls = launches("hcmix_grouped_attention_backward",
                  forward(1, 4096, 1024, 8, 2, 64, 512) + [mem(5), mem(6)] + i64(512) + [mem(7)]
                  + i64(128) + [mem(8)] + i64(128) + [mem(9), ["size_t", 1 << 39], NONE])
    assert [x for (x, _, _), _, _ in ls] == [64 * 8, 32 * 8, 1024 * 128 // 8 // 256]
    assert ls[2][0][1] == 2


@pytest.mark.parametrize("rows,heads,hd", [(1 << 30, 1, 2), (1 << 20, 1024, 128), (1, 1, 512)])
def test_rotary(launches, rows, heads, hd):  # noqa: F811
    ls = launches("hcmix_rotary", i64(rows) + i32(heads, hd, hd, 0, 0, 1) + [mem(0)]
                  + i64(heads * hd) + [NONE] + i64(4096) + [mem(1)] + F32(1.0) + [mem(2)]
                  + i64(heads * hd) + [NONE])
    assert len(ls) == 1 and ls[0][0][0] <= 1 << 20


@pytest.mark.parametrize("batch,capacity,kv,tokens", [(65535, 64, 16, 1), (1, 1 << 24, 8, 65536),
                                                      (2, 1 << 20, 1024, 65536)])
def test_cache(launches, batch, capacity, kv, tokens):  # noqa: F811
    size, ptr = ["size_t", 1 << 40], mem
    dims = i64(batch, capacity) + i32(kv, 64) + i64(tokens)
    (x, y, z), _, _ = launches("hcmix_kv_cache_append", dims + [ptr(0)] + i64(kv * 64) + [ptr(1)]
                               + i64(kv * 64) + [ptr(2), NONE, ptr(3), size, NONE])[0]
    if tokens == 1:       # a wave to a head
        assert 4 * x >= kv > 4 * (x - 1) and (y, z) == (batch, 1)
    else:                 # blocks from the last token of one on
        assert (y, z) == (kv, batch) and 64 * x >= tokens + 63 > 64 * (x - 1)
    (x, y, z), _, _ = launches("hcmix_kv_cache_read", dims + [ptr(0), ptr(1), ptr(3), size, ptr(4),
                                                              ptr(5), NONE])[0]
    assert (y, z) == (kv, batch) and 64 * x >= tokens
    ls = launches("hcmix_kv_cache_attention", i64(batch, capacity) + i32(4 * kv if kv < 256 else kv, kv, 64)
                  + i64(min(tokens, 5)) + F32(0.125) + [ptr(0)] + i64((4 * kv if kv < 256 else kv) * 64)
                  + [ptr(1)] + i64(capacity) + [ptr(3), size, ptr(6), ptr(7), ["size_t", 1 << 39], NONE])
    assert ls[0][0][1:] == [kv, batch] and len(ls) <= 2
