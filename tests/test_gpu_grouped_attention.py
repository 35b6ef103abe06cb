"""Attention over windows of any length against the oracle, element by element
within the oracle's bounds (what the roundings that the library names can make).
lse is held in 32 bits: off by 2^-14 of the largest score's size (a score is a
sum of at most 128 products, a sum of exponentials off by 2^-18)."""
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


def draw(batch, n_q, n_k, heads, kv, hd, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g).to(torch.bfloat16).cuda()
    q, k = normal(batch, n_q, heads, hd) * size, normal(batch, n_k, kv, hd)
    return q, k, normal(batch, n_k, kv, hd), normal(batch, n_q, heads, hd)


def host(t):
    return t.detach().double().cpu().numpy()


def within(name, got, ref, bound):
    err = np.abs(host(got) - ref)
    with np.errstate(invalid="ignore", divide="ignore"):
        print(f"  {name}: largest error {err.max():.2e}, of its bound {np.nanmax(err / bound):.2f}",
              flush=True)
    assert (err <= bound).all(), name


def check(q, k, v, do, causal, lengths, scale=None, grads=True):
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out, lse = hcmix.grouped_attention_forward(q, k, v, causal, ln, scale)
    hq, hk, hv, hdo = (host(t) for t in (q, k, v, do))
    r_out, r_lse, bound = grouped.forward(hq, hk, hv, causal, lengths, scale)
    within("out", out, r_out, bound)
    empty = np.isneginf(r_lse)
    assert np.array_equal(np.isneginf(host(lse)), empty)
    top = max(1.0, np.abs(r_lse[~empty]).max(initial=0.0))
    assert np.abs(host(lse)[~empty] - r_lse[~empty]).max(initial=0.0) <= 2.0 ** -14 * top
    if not grads:
        return out, lse
    g = hcmix.grouped_attention_backward(q, k, v, out, lse, do, causal, ln, scale)
    again = hcmix.grouped_attention_backward(q, k, v, out, lse, do, causal, ln, scale)
    ref, bounds = grouped.backward(hq, hk, hv, hdo, causal, lengths, scale)
    for i, name in enumerate(("dq", "dk", "dv")):
        within(name, g[i], ref[i], bounds[i])
        assert torch.equal(g[i], again[i])
    return g


# batch, n_q, n_k, heads, kv_heads, head_dim, causal, lengths, size of the queries
CASES = [
    (1, 1, 1, 1, 1, 64, True, None, 1.0), (2, 1, 300, 4, 2, 128, True, None, 1.0),
    (2, 31, 31, 2, 2, 64, True, None, 1.0), (1, 32, 33, 3, 1, 128, False, None, 1.0),
    (2, 64, 64, 2, 1, 64, False, None, 1.0), (1, 65, 129, 4, 4, 64, True, None, 1.0),
    (2, 127, 257, 6, 2, 128, True, [257, 1], 1.0), (3, 128, 128, 2, 2, 64, True, [0, 5, 128], 1.0),
    (1, 129, 65, 2, 1, 64, True, None, 1.0),      # the first 64 rows see nothing
    (2, 200, 40, 2, 2, 128, True, [40, 7], 1.0), (3, 100, 100, 4, 1, 128, False, [0, 33, 100], 1.0),
    (1, 513, 513, 2, 1, 64, True, None, 3.0), (1, 300, 700, 8, 1, 64, False, [650], 3.0),
    (2, 1000, 1000, 2, 1, 128, True, [1000, 511], 1.0), (1, 4096, 40, 1, 1, 64, False, None, 1.0),
    (1, 40, 4096, 1, 1, 128, True, None, 1.0), (2, 7, 7, 4, 4, 64, True, [-3, 99], 1.0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:6])))
def test_matches_the_oracle(case):
    print(f"case: grouped attention {case}", flush=True)
    batch, n_q, n_k, heads, kv, hd, causal, lengths, size = case
    check(*draw(batch, n_q, n_k, heads, kv, hd, seed=n_q + n_k, size=size), causal, lengths)


@pytest.mark.parametrize("case", [(1, 4, 4, 2, 2, 64, True), (15, 4, 4, 2, 2, 64, True), (2, 32, 32, 4, 1, 128, True),
                                  (1, 100, 100, 2, 1, 64, True), (1, 7, 128, 2, 2, 128, False)],
                         ids=lambda c: "x".join(map(str, c[:6])))
def test_few_scores_are_as_near_as_their_own_rounding(case):
    """P and dS taken as two bf16 numbers are off by 2^-17, which adds less than a
    twentieth to what the rounding of the results themselves, 2^-9.2 in the mean, is off in norm."""
    batch, n_q, n_k, heads, kv, hd, causal = case
    for seed in range(4):
        q, k, v, do = draw(batch, n_q, n_k, heads, kv, hd, seed=seed)
        out, lse = hcmix.grouped_attention_forward(q, k, v, causal)
        got = (out, *hcmix.grouped_attention_backward(q, k, v, out, lse, do, causal))
        hq, hk, hv, hdo = (host(t) for t in (q, k, v, do))
        ref = (grouped.forward(hq, hk, hv, causal)[0], *grouped.backward(hq, hk, hv, hdo, causal)[0])
        for name, g, r in zip(("out", "dq", "dk", "dv"), got, ref):
            own = np.linalg.norm(host(torch.from_numpy(r).to(torch.bfloat16)) - r)
            err = np.linalg.norm(host(g) - r)
            print(f"  {name}: {err / own:.3f} of its own rounding", flush=True)
            assert err <= 1.05 * own, name


def spread(batch, n):
    """Lengths from 0 past n, none of them round."""
    return [0, n, n + 5] + [1 + (37 * i) % n for i in range(3, batch)]


# more blocks of 128 rows and of 128 keys than the GPU has CUs: blocks of four waves
MANY = [
    (70, 130, 260, 4, 2, 64, True, spread(70, 260), 1.0), (70, 260, 130, 4, 2, 128, False, spread(70, 130), 1.0),
    (66, 290, 300, 4, 2, 64, True, spread(66, 300), 2.0), (66, 300, 300, 4, 2, 128, True, None, 1.0),
    # few queries of many keys, more such blocks than the GPU has CUs
    (70, 3, 1030, 4, 2, 64, True, spread(70, 1030), 1.0), (70, 40, 1030, 4, 4, 128, False, None, 1.0),
]


@pytest.mark.parametrize("case", MANY, ids=lambda c: "x".join(map(str, c[:6])))
def test_many_blocks_match_the_oracle(case):
    print(f"case: grouped attention {case[:7]}", flush=True)
    batch, n_q, n_k, heads, kv, hd, causal, lengths, size = case
    check(*draw(batch, n_q, n_k, heads, kv, hd, seed=n_q + n_k, size=size), causal, lengths)


def test_long_window_sampled():
    """A sequence of 4096; the last head of the last group checked whole."""
    q, k, v, do = draw(1, 4096, 4096, 4, 2, 64, seed=9)
    out, lse = hcmix.grouped_attention_forward(q, k, v)
    g = hcmix.grouped_attention_backward(q, k, v, out, lse, do)
    s = [host(t) for t in (q[:, :, 2:], k[:, :, 1:], v[:, :, 1:], do[:, :, 2:])]
    r_out, _, bound = grouped.forward(*s[:3])
    within("out", out[:, :, 2:], r_out, bound)
    ref, bounds = grouped.backward(*s)
    for i, name in enumerate(("dq", "dk", "dv")):
        within(name, g[i][:, :, 2 if i == 0 else 1:], ref[i], bounds[i])


@pytest.mark.parametrize("batch,n_q,n_k,heads,kv,hd,causal", [
    (40, 100, 100, 8, 4, 64, True), (40, 70, 200, 8, 8, 128, False), (3, 1500, 1500, 16, 2, 64, True),
    (44, 129, 257, 6, 3, 128, True)])
def test_more_blocks_than_compute_units_sampled(batch, n_q, n_k, heads, kv, hd, causal):
    """Ragged batches that fill the chip several times; three (sequence, group) pairs."""
    print(f"case: {batch} {n_q} {n_k} {heads} {kv} {hd} {causal}", flush=True)
    q, k, v, do = draw(batch, n_q, n_k, heads, kv, hd, seed=batch)
    lengths = [(7 * b + 1) % (n_k + 1) for b in range(batch)]
    lengths[-1] = n_k
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out, lse = hcmix.grouped_attention_forward(q, k, v, causal, ln)
    g = hcmix.grouped_attention_backward(q, k, v, out, lse, do, causal, ln)
    per = heads // kv
    for b, c in ((0, 0), (batch // 2, kv - 1), (batch - 1, kv // 2)):
        hq, ck = slice(c * per, c * per + per), slice(c, c + 1)
        s = [host(t[b:b + 1, :, h]) for t, h in ((q, hq), (k, ck), (v, ck), (do, hq))]
        r_out, r_lse, bound = grouped.forward(*s[:3], causal, lengths[b:b + 1])
        within("out", out[b:b + 1, :, hq], r_out, bound)
        seen = ~np.isneginf(r_lse)
        got = host(lse[b:b + 1, hq])
        assert np.array_equal(~np.isneginf(got), seen)
        assert np.abs(got[seen] - r_lse[seen]).max(initial=0.0) <= 2.0 ** -14 * 10
        ref, bounds = grouped.backward(*s, causal, lengths[b:b + 1])
        for i, (name, h) in enumerate((("dq", hq), ("dk", ck), ("dv", ck))):
            within(name, g[i][b:b + 1, :, h], ref[i], bounds[i])


@pytest.mark.parametrize("heads,kv,hd", [(4, 2, 64), (2, 2, 128)])
def test_packed_projection_in_and_out(heads, kv, hd):
    """Slices of one packed buffer in and one packed gradient out: as apart."""
    n = 70
    g = torch.Generator().manual_seed(1)
    packed = torch.randn((2, n, heads + 2 * kv, hd), generator=g).to(torch.bfloat16).cuda()
    do = torch.randn((2, n, heads, hd), generator=g).to(torch.bfloat16).cuda()
    q, k, v = packed.split([heads, kv, kv], 2)
    out, lse = hcmix.grouped_attention_forward(q, k, v)
    a = hcmix.grouped_attention_forward(q.contiguous(), k.contiguous(), v.contiguous())
    assert torch.equal(out, a[0]) and torch.equal(lse, a[1])
    dpacked = torch.full_like(packed, 3)
    hcmix.grouped_attention_backward(q, k, v, out, lse, do,
                                     **dict(zip(("dq", "dk", "dv"),
                                                dpacked.split([heads, kv, kv], 2))))
    b = hcmix.grouped_attention_backward(q.contiguous(), k.contiguous(), v.contiguous(), out, lse,
                                         do)
    assert torch.equal(dpacked, torch.cat(b, 2))


@pytest.mark.parametrize("fill", [float("nan"), float("inf"), torch.finfo(torch.bfloat16).min])
def test_what_lies_behind_the_lengths_is_not_taken(fill):
    q, k, v, do = draw(2, 90, 90, 2, 1, 64, seed=3)
    ln = torch.tensor([37, 64], dtype=torch.int32, device="cuda")
    res = []
    for put in (0.0, fill):
        for b, n in enumerate((37, 64)):
            k[b, n:], v[b, n:] = put, put
        out, lse = hcmix.grouped_attention_forward(q, k, v, True, ln)
        res.append((out, lse, *hcmix.grouped_attention_backward(q, k, v, out, lse, do, True, ln)))
    for a, b in zip(*res):
        assert torch.equal(a, b)
    assert (res[1][3][0, 37:] == 0).all() and (res[1][4][1, 64:] == 0).all()


@pytest.mark.parametrize("batch,hd,size", [(1, 128, 1.0), (1, 64, 1.0), (1, 64, 6.0), (50, 64, 6.0), (50, 128, 6.0)])
def test_rows_do_not_see_ahead(batch, hd, size):
    """Bit for bit, also where later rows of a wave rescale their sums (large scores)."""
    q, k, v, _ = draw(batch, 300, 300, 2, 1, hd, seed=4, size=size)
    a, la = hcmix.grouped_attention_forward(q, k, v)
    for i in (0, 1, 17, 63, 64, 200, 280):
        k2, v2 = k.clone(), v.clone()
        k2[:, i + 1:], v2[:, i + 1:] = 5.0, -3.0
        b, lb = hcmix.grouped_attention_forward(q, k2, v2)
        assert torch.equal(a[:, :i + 1], b[:, :i + 1])
        assert torch.equal(la[:, :, :i + 1], lb[:, :, :i + 1])


def test_other_scale_and_autograd():
    q, k, v, do = draw(2, 50, 50, 4, 2, 64, seed=5)
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
    out = hcmix.GroupedAttention.apply(*leaves, True, None, 0.25)
    out.backward(do)
    ref, bounds = grouped.backward(*(host(t) for t in (q, k, v, do)), scale=0.25)
    for i, t in enumerate(leaves):
        within(f"grad {i}", t.grad, ref[i], bounds[i])


def test_on_another_stream_and_captured():
    q, k, v, do = draw(2, 130, 130, 4, 2, 64, seed=6)
    out, lse = hcmix.grouped_attention_forward(q, k, v)
    want = (out, lse, *hcmix.grouped_attention_backward(q, k, v, out, lse, do))

    def step():
        o, l = hcmix.grouped_attention_forward(q, k, v)
        return (o, l, *hcmix.grouped_attention_backward(q, k, v, o, l, do))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_autograd_captured_whole():
    """Rotary and attention with their gradients in one captured graph, replayed on
    other inputs between eager runs of the same: as those."""
    g = torch.Generator().manual_seed(7)
    freqs, _ = hcmix.rotary_frequencies(64)

    def step(q, k, v, do):
        q, k, v = (t.detach().requires_grad_(True) for t in (q, k, v))
        out = hcmix.GroupedAttention.apply(hcmix.Rotary.apply(q, freqs), hcmix.Rotary.apply(k, freqs), v)
        return (out.detach(), *torch.autograd.grad(out, (q, k, v), do))
    sets = [[torch.randn((2, 90, h, 64), generator=g).to(torch.bfloat16).cuda() for h in (4, 2, 2, 4)]
            for _ in range(3)]
    ops = [t.clone() for t in sets[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*ops)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*ops)
    for other in sets:
        for a, b in zip(ops, other):
            a.copy_(b)
        graph.replay()
        want = step(*other)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("case", [(40, 256, 257, 4, 2, 64, 1.0), (40, 256, 257, 4, 2, 128, 1.0), (70, 256, 129, 4, 2, 64, 1.0),
                                  (40, 256, 300, 4, 2, 64, 3.0), (4, 256, 300, 4, 2, 128, 3.0), (4, 256, 257, 4, 2, 64, 1.0)],
                         ids=lambda c: "x".join(map(str, c[:6])))
def test_rows_of_few_keys_beside_rows_of_many(case):
    """A row that sees at most 128 keys takes D from P itself, whatever the other rows of
    its block see: the rounding of out is not in its bounds.  In norm dS's rounding then
    adds as much as dq's own (its terms meet independent keys): sqrt(2) of it together."""
    print(f"case: grouped attention {case}", flush=True)
    batch, n_q, n_k, heads, kv, hd, size = case
    q, k, v, do = draw(batch, n_q, n_k, heads, kv, hd, seed=n_k, size=size)
    out, lse = hcmix.grouped_attention_forward(q, k, v)
    got = hcmix.grouped_attention_backward(q, k, v, out, lse, do)
    ref, bounds = grouped.backward(*(host(t) for t in (q, k, v, do)), exact=128)
    for i, name in enumerate(("dq", "dk", "dv")):
        within(name, got[i], ref[i], bounds[i])
    seen = np.clip(np.arange(n_q) + 1 + n_k - n_q, 0, n_k)
    for lo, hi in ((2, 4), (5, 16), (17, 64), (65, 128)):
        rows = (seen >= lo) & (seen <= hi)
        if not rows.any():
            continue
        r = ref[0][:, rows]
        own = np.linalg.norm(host(torch.from_numpy(r).to(torch.bfloat16)) - r)
        err = np.linalg.norm(host(got[0])[:, rows] - r)
        print(f"  dq of rows of {lo} to {hi} keys: {err / own:.3f} of its own rounding", flush=True)
        assert err <= 1.6 * own, (lo, hi)


@pytest.mark.parametrize("case", [(1, 16, 512, 4, 4, 64, False), (1, 16, 512, 4, 4, 128, False), (1, 100, 300, 2, 1, 64, True),
                                  (1, 100, 300, 2, 1, 128, True), (1, 1, 4000, 8, 2, 128, True), (1, 6, 2900, 3, 1, 64, True)],
                         ids=lambda c: "x".join(map(str, c[:6])))
def test_few_scores_of_many_keys_are_as_near(case):
    """As the calls of few scores above, also past 128 keys and with weights that few
    keys share (queries of size 3)."""
    batch, n_q, n_k, heads, kv, hd, causal = case
    for seed in range(3):
        q, k, v, do = draw(batch, n_q, n_k, heads, kv, hd, seed=seed, size=3.0)
        lengths = None if seed else [n_k - 150] * batch
        ln = None if seed else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        out, lse = hcmix.grouped_attention_forward(q, k, v, causal, ln)
        got = (out, *hcmix.grouped_attention_backward(q, k, v, out, lse, do, causal, ln))
        hq, hk, hv, hdo = (host(t) for t in (q, k, v, do))
        ref = (grouped.forward(hq, hk, hv, causal, lengths)[0],
               *grouped.backward(hq, hk, hv, hdo, causal, lengths)[0])
        for name, g, r in zip(("out", "dq", "dk", "dv"), got, ref):
            own = np.linalg.norm(host(torch.from_numpy(r).to(torch.bfloat16)) - r)
            err = np.linalg.norm(host(g) - r)
            print(f"  {name}: {err / own:.3f} of its own rounding", flush=True)
            assert err <= 1.05 * own, name


@pytest.mark.parametrize("hd", [64, 128])
def test_few_scores_over_more_key_tiles_than_compute_units(hd):
    """One query of 40000 keys: 313 tiles of keys, and all gradients as near as of fewer."""
    q, k, v, do = draw(1, 1, 40000, 1, 1, hd, seed=1, size=3.0)
    out, lse = hcmix.grouped_attention_forward(q, k, v)
    got = (out, *hcmix.grouped_attention_backward(q, k, v, out, lse, do))
    hq, hk, hv, hdo = (host(t) for t in (q, k, v, do))
    ref = (grouped.forward(hq, hk, hv)[0], *grouped.backward(hq, hk, hv, hdo)[0])
    for name, g, r in zip(("out", "dq", "dk", "dv"), got, ref):
        own = np.linalg.norm(host(torch.from_numpy(r).to(torch.bfloat16)) - r)
        err = np.linalg.norm(host(g) - r)
        print(f"  {name}: {err / own:.3f} of its own rounding", flush=True)
        assert err <= 1.05 * own, name


@pytest.mark.parametrize("case", [(1, 200, 150, 2, 1, 64, None), (1, 200, 150, 2, 1, 128, None), (2, 100, 160, 2, 2, 64, [131, 0]),
                                  (2, 100, 160, 2, 1, 128, [160, 140]), (40, 260, 200, 4, 2, 64, None),
                                  (40, 260, 200, 4, 4, 128, None)], ids=lambda c: "x".join(map(str, c[:6])))
def test_blocks_of_empty_short_and_long_rows(case):
    """Rows that see nothing, at most 128 keys and more beside each other, in calls of few
    scores and of many."""
    print(f"case: grouped attention {case}", flush=True)
    batch, n_q, n_k, heads, kv, hd, lengths = case
    q, k, v, do = draw(batch, n_q, n_k, heads, kv, hd, seed=n_q, size=3.0)
    check(q, k, v, do, True, lengths)
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out, lse = hcmix.grouped_attention_forward(q, k, v, True, ln)
    dq, dk, _ = hcmix.grouped_attention_backward(q, k, v, out, lse, do, True, ln)
    ref, bounds = grouped.backward(*(host(t) for t in (q, k, v, do)), True, lengths, exact=128)
    within("dq", dq, ref[0], bounds[0])
    within("dk", dk, ref[1], bounds[1])
