"""The 8-bit key/value cache: what it holds equals the oracle's cache number by
number; attention over it lies within the oracle's bounds for those numbers."""
import numpy as np
import pytest
import torch

from oracle import grouped
from paper_2609_18145_amd import hcmix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hcmix.load()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Both:
    """The library's cache and the oracle's, one per sequence."""

    def __init__(self, batch, capacity, kv, hd, fill=0xff):
        self.dims = (batch, capacity, kv, hd)
        self.cache = hcmix.alloc_kv_cache(batch, capacity, kv, hd, "cuda").fill_(fill)   # NaN bytes
        self.ref = [[grouped.Cache(capacity, kv, hd) for _ in range(batch)] for _ in range(2)]

    def append(self, k, v, pos, counts=None):
        hcmix.kv_cache_append(k, v, ints(pos), self.cache, self.dims[1],
                              None if counts is None else ints(counts))
        for t, ref in zip((k, v), self.ref):
            for b, c in enumerate(ref):
                n = t.shape[1] if counts is None else min(max(counts[b], 0), t.shape[1])
                if n:
                    c.append(t[b, :n].double().cpu().numpy(), pos[b])

    def check(self, lengths):
        batch, capacity, kv, hd = self.dims
        got = hcmix.kv_cache_read(self.cache, capacity, kv, hd, ints([0] * batch), ints(lengths),
                                  capacity + 3)
        for name, t, ref in zip("kv", got, self.ref):
            t = t.double().cpu().numpy()
            for b, n in enumerate(lengths):
                n = min(max(n, 0), capacity)
                np.testing.assert_array_equal(t[b, :n], ref[b].held[:n], err_msg=f"{name} {b}")
                assert (t[b, n:] == 0).all()


def tokens(batch, n, kv, hd, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((batch, n, kv, hd), generator=g)
    x *= torch.exp2(torch.randint(-9, 9, (batch, n, 1, 1), generator=g)) * size
    return x.to(torch.bfloat16).cuda()


@pytest.mark.parametrize("batch,capacity,kv,hd,chunks", [
    (2, 1, 1, 64, [1]), (2, 64, 2, 64, [1] * 64), (1, 200, 3, 128, [1] * 5 + [63, 64, 68]),
    (3, 130, 1, 128, [130]), (2, 129, 8, 64, [100, 1, 1, 20, 7]), (1, 1000, 1, 64, [65, 1, 700, 234]),
    (1, 70, 2, 64, [60, 30])])                                   # past the capacity
def test_what_is_held(batch, capacity, kv, hd, chunks):
    print(f"case: append {batch} {capacity} {kv} {hd} {chunks}", flush=True)
    c, pos = Both(batch, capacity, kv, hd), 0
    for i, n in enumerate(chunks):
        c.append(tokens(batch, n, kv, hd, i), tokens(batch, n, kv, hd, 100 + i), [pos] * batch)
        pos += n
        if n > 1 or i % 16 == 0:
            c.check([pos] * batch)
    c.check([pos] * batch)


def test_ragged_positions_counts_and_sequences_left_out():
    c = Both(6, 150, 2, 64)
    c.append(tokens(6, 100, 2, 64, 1), tokens(6, 100, 2, 64, 2), [0] * 6, [100, 64, 0, 1, 63, 999])
    lengths = [100, 64, 0, 1, 63, 100]
    c.check(lengths)
    before = c.cache.clone()
    c.append(tokens(6, 3, 2, 64, 3), tokens(6, 3, 2, 64, 4), [150, -1, 4000, -64, 150, 151])
    c.append(tokens(6, 3, 2, 64, 3), tokens(6, 3, 2, 64, 4), [0] * 6, [0, -5, 0, 0, 0, 0])
    assert torch.equal(before, c.cache)
    c.append(tokens(6, 70, 2, 64, 5), tokens(6, 70, 2, 64, 6), lengths, [70, 1, 70, 64, 2, 50])
    c.check([150, 65, 70, 65, 65, 150])


def test_drafted_tokens_are_taken_back():
    """Appending at an earlier position: what was behind it is dropped, the
    block's scale stays at what its tokens have needed."""
    c = Both(1, 256, 1, 128)
    c.append(tokens(1, 100, 1, 128, 1), tokens(1, 100, 1, 128, 2), [0])
    c.append(tokens(1, 8, 1, 128, 3, size=64.0), tokens(1, 8, 1, 128, 4, size=64.0), [100])
    c.append(tokens(1, 2, 1, 128, 5), tokens(1, 2, 1, 128, 6), [102])
    c.check([104])
    c.append(tokens(1, 3, 1, 128, 7), tokens(1, 3, 1, 128, 8), [64])      # a whole block anew
    c.check([67])


def test_extremes():
    """Zeros, the smallest and largest numbers, infinities (held as 448 times
    2^120, where bf16's largest lies below 2^128) and NaN."""
    x = torch.zeros((1, 192, 1, 64), dtype=torch.bfloat16, device="cuda")
    x[0, 64, 0, 0], x[0, 65, 0, 1], x[0, 70, 0, 2] = 1e-38, -3e-39, 9.2e-41
    x[0, 128, 0, 0], x[0, 129, 0, 1] = 3e38, -1e36
    c = Both(1, 192, 1, 64)
    c.append(x, -x, [0])
    c.check([192])
    x[0, 0, 0, 0] = float("nan")
    x[0, 64, 0, 0] = float("inf")
    c = hcmix.alloc_kv_cache(1, 192, 1, 64, "cuda")
    hcmix.kv_cache_append(x, x, ints([0]), c, 192)
    for t in hcmix.kv_cache_read(c, 192, 1, 64, ints([0]), ints([192]), 192):
        assert t[0, 0, 0, 0].isnan() and t[0, :, 0, :].isnan().sum() == 1
        assert t[0, 64, 0, 0] == float("inf")      # 448 2^120 is past bf16's largest


def test_read_a_range():
    c = Both(3, 200, 2, 128)
    k, v = tokens(3, 200, 2, 128, 1), tokens(3, 200, 2, 128, 2)
    c.append(k, v, [0] * 3)
    first, lengths = [0, 77, -5], [200, 120, 10]
    got = hcmix.kv_cache_read(c.cache, 200, 2, 128, ints(first), ints(lengths), 90)
    for t, ref in zip(got, c.ref):
        t = t.double().cpu().numpy()
        for b in range(3):
            for i in range(90):
                p = first[b] + i
                want = ref[b].held[p] if 0 <= p < lengths[b] else np.zeros((2, 128))
                np.testing.assert_array_equal(t[b, i], want)


# batch, capacity, query heads, key/value heads, head_dim, tokens, lengths, max_length
ATTENTION = [
    (1, 1, 1, 1, 64, 1, [1], None), (2, 256, 8, 8, 64, 1, [1, 256], None),
    (3, 300, 8, 2, 64, 5, [300, 5, 64], None), (2, 129, 4, 1, 128, 1, [129, 0], None),
    (4, 500, 6, 2, 128, 3, [2, 0, 1, 499], None), (1, 5000, 8, 1, 64, 1, [4999], None),
    (2, 3000, 16, 2, 128, 1, [3000, 63], 64), (1, 700, 40, 1, 64, 1, [700], None),
    (1, 700, 12, 4, 128, 30, [650], None), (2, 200, 3, 3, 64, 130, [200, 131], None),
    (2, 90, 4, 2, 64, 2, [-7, 1000], None), (1, 2100, 32, 1, 128, 1, [2050], 2100),
    (1, 2100, 64, 1, 128, 2, [2050], 2100),
    # blocks of 16 and of 8 waves that have a sequence each; 18 ranges
    (5, 777, 4, 2, 64, 1, [777, 0, 300, 1, 700], None), (2, 700, 20, 1, 128, 1, [700, 10], None),
    (64, 1000, 8, 4, 64, 2, [1000 - 9 * i for i in range(64)], None), (1, 9000, 4, 1, 64, 1, [8800], None),
    (3, 700, 20, 1, 64, 1, [64, 700, 449], 700),
]


@pytest.mark.parametrize("case", ATTENTION, ids=lambda c: "x".join(map(str, c[:6])))
def test_attention_matches_the_oracle(case):
    print(f"case: cache attention {case}", flush=True)
    batch, capacity, heads, kv, hd, n, lengths, longest = case
    c = Both(batch, capacity, kv, hd)
    held = [min(max(x, 0), capacity) for x in lengths]
    g = torch.Generator().manual_seed(capacity)
    if max(held):
        k, v = (torch.randn((batch, max(held), kv, hd), generator=g).to(torch.bfloat16).cuda()
                for _ in range(2))
        c.append(k, v, [0] * batch, held)
    q = torch.randn((batch, n, heads, hd), generator=g).to(torch.bfloat16).cuda()
    out = hcmix.kv_cache_attention(q, ints(lengths), c.cache, capacity, kv, max_length=longest)
    again = hcmix.kv_cache_attention(q, ints(lengths), c.cache, capacity, kv, max_length=longest)
    assert torch.equal(out, again)
    out = out.double().cpu().numpy()
    for b, m in enumerate(held):
        if not m:
            assert (out[b] == 0).all()
            continue
        r, _, bound = grouped.forward(q[b:b + 1].double().cpu().numpy(), c.ref[0][b].held[None, :m],
                                      c.ref[1][b].held[None, :m])
        err = np.abs(out[b] - r[0])
        print(f"  sequence {b}: {err.max():.2e}, of its bound {np.nanmax(err / np.maximum(bound[0], 1e-30)):.2f}",
              flush=True)
        assert (err <= bound[0]).all()


def test_packed_queries_other_scale_and_graph():
    """One token appended and attended in a captured graph, replayed at later
    positions: as the same calls outside."""
    batch, capacity, heads, kv, hd = 3, 150, 4, 2, 64
    caches = [hcmix.alloc_kv_cache(batch, capacity, kv, hd, "cuda") for _ in range(2)]
    packed = torch.zeros((batch, 1, heads + 2 * kv, hd), dtype=torch.bfloat16, device="cuda")
    q, k, v = packed.split([heads, kv, kv], 2)
    pos, lengths = ints([0] * batch), ints([1] * batch)

    def step(cache):
        hcmix.kv_cache_append(k, v, pos, cache, capacity)
        return hcmix.kv_cache_attention(q, lengths, cache, capacity, kv, scale=0.2)
    step(caches[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(caches[0])
    for p in range(140):
        g = torch.Generator().manual_seed(p)
        packed.copy_(torch.randn(packed.shape, generator=g))
        pos.fill_(p)
        lengths.fill_(p + 1)
        graph.replay()
        want = step(caches[1])
        torch.cuda.synchronize()
        assert torch.equal(out, want), p


def test_calls_on_two_streams_at_once():
    """Two batches decoded on streams of their own, each with its cache: as one
    after the other."""
    def decode(seed):
        g = torch.Generator().manual_seed(seed)
        cache = hcmix.alloc_kv_cache(4, 700, 2, 64, "cuda")
        outs = []
        k, v = (torch.randn((4, 600, 2, 64), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        hcmix.kv_cache_append(k, v, ints([0] * 4), cache, 700)
        for p in range(600, 620):
            q = torch.randn((4, 1, 8, 64), generator=g).to(torch.bfloat16).cuda()
            hcmix.kv_cache_append(q[:, :, :2], q[:, :, 2:4], ints([p] * 4), cache, 700)
            outs.append(hcmix.kv_cache_attention(q, ints([p + 1] * 4), cache, 700, 2))
        return torch.stack(outs)
    want = [decode(s) for s in (1, 2)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for i, st in enumerate(streams):
        with torch.cuda.stream(st):
            got.append(decode(i + 1))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("chunks", [[70], [1] * 4, [3, 1, 66]])
def test_the_largest_finite_numbers_stay_finite(chunks):
    """From 248 2^120 on a quotient at the largest scale would round to 2^128."""
    top = torch.finfo(torch.bfloat16).max
    n = sum(chunks)
    x = torch.zeros((1, n, 1, 64), dtype=torch.bfloat16, device="cuda")
    for t, v in enumerate((top, -top, 3.31e38, 3.29e38, -3.2e38, 1e30, float("inf"))[:n]):
        x[0, t, 0, 5 * t] = v
    c, pos = Both(1, n, 1, 64), 0
    for m in chunks:
        c.append(x[:, pos:pos + m].contiguous(), -x[:, pos:pos + m].contiguous(), [pos])
        pos += m
    got = hcmix.kv_cache_read(c.cache, n, 1, 64, ints([0]), ints([n]), n)
    for t, ref, sign in zip(got, c.ref, (1, -1)):
        assert torch.equal(t.isinf(), x.isinf())
        want = np.where(x.isinf().cpu().numpy()[0], sign * np.inf, ref[0].held)
        np.testing.assert_array_equal(t[0].double().cpu().numpy(), want)
    # one token alone: its value back
    out = hcmix.kv_cache_attention(torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16, device="cuda"),
                                   ints([1]), c.cache, n, 1)
    assert torch.equal(out, got[1][:, :1]) and out.isfinite().all()
