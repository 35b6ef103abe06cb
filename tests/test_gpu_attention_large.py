"""The attention layers past the fixed windows on tensors of more than 2^31 elements
and a cache of more than 2^32 bytes: the last rows against the oracle."""
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
    yield
    torch.cuda.empty_cache()


def host(t):
    return t.detach().double().cpu().numpy()


def test_a_million_queries_of_33_heads():
    n, n_k, heads, hd = 1 << 20, 70, 33, 64
    g = torch.Generator("cuda").manual_seed(1)
    q, do = (torch.randn((1, n, heads, hd), generator=g, device="cuda", dtype=torch.bfloat16)
             for _ in range(2))
    assert q.numel() > 1 << 31
    k, v = (torch.randn((1, n_k, heads, hd), generator=g, device="cuda", dtype=torch.bfloat16)
            for _ in range(2))
    out, lse = hcmix.grouped_attention_forward(q, k, v, causal=False)
    dq, dk, dv = hcmix.grouped_attention_backward(q, k, v, out, lse, do, causal=False)
    s = slice(n - 50, n)
    r, r_lse, bound = grouped.forward(host(q[:, s]), host(k), host(v), causal=False)
    assert (np.abs(host(out[:, s]) - r) <= bound).all()
    assert np.abs(host(lse[:, :, s]) - r_lse).max() <= 2.0 ** -14 * 10
    ref, bounds = grouped.backward(host(q[:, s]), host(k), host(v), host(do[:, s]), causal=False)
    assert (np.abs(host(dq[:, s]) - ref[0]) <= bounds[0]).all()
    # the key gradients are sums over every query: the last 50 alone move them by what the
    # oracle says (a sum of 2^20 terms of bf16 P and dS, so a share of its own rounding)
    do2 = do.clone()
    do2[:, s] = 0
    _, _, dv2 = hcmix.grouped_attention_backward(q, k, v, out, lse, do2, causal=False)
    size = host(dv).std()
    assert np.abs(host(dv) - host(dv2) - ref[2]).max() <= 2.0 ** -7 * 6 * size + np.abs(bounds[2]).max()
    del do, do2, dq, out
    freqs, _ = hcmix.rotary_frequencies(hd)
    before = host(q[:, s])
    hcmix.rotary(q, freqs, out=q)
    ref = grouped.rotary(before, np.arange(n - 50, n)[None], freqs.cpu().numpy(), True)
    assert np.abs(host(q[:, s]) - ref).max() <= 2.0 ** -8 * np.abs(ref).max() + 2.0 ** -20 * 16


def test_a_cache_of_eight_gigabytes():
    """Four million tokens held as zeros, then some at the end: the zeros' scores
    are 0, their values nothing."""
    capacity, kv, hd, heads = (1 << 22) - 5, 8, 128, 16
    cache = hcmix.alloc_kv_cache(1, capacity, kv, hd, "cuda").zero_()
    assert cache.numel() > 1 << 33
    at = torch.tensor([capacity - 131], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((1, 131, kv, hd), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    hcmix.kv_cache_append(k, v, at, cache, capacity)
    end = torch.tensor([capacity], dtype=torch.int32, device="cuda")
    got = hcmix.kv_cache_read(cache, capacity, kv, hd, at, end, 140)
    held = []
    for t, x in zip(got, (k, v)):
        ref = grouped.Cache(131 + 64, kv, hd)
        first = (capacity - 131) % 64
        ref.append(np.zeros((first, kv, hd)), 0)
        ref.append(host(x)[0], first)
        np.testing.assert_array_equal(host(t)[0, :131], ref.held[first:first + 131])
        assert (host(t)[0, 131:] == 0).all()
        held.append(ref.held[first:first + 131])
    # scores large enough that the last tokens matter among four million
    q = (3 * torch.randn((1, 1, heads, hd), generator=g)).to(torch.bfloat16).cuda()
    out = host(hcmix.kv_cache_attention(q, end, cache, capacity, kv))[0, 0]
    for h in range(heads):
        s = host(q)[0, 0, h] @ held[0][:, h // 2].T / np.sqrt(hd)
        p = np.exp(s) / (np.exp(s).sum() + capacity - 131)
        want, size = p @ held[1][:, h // 2], p @ np.abs(held[1][:, h // 2])
        # as the oracle's bounds; the sum of four million ones in 32 bits is off by 2^-12 at most
        assert (np.abs(out[h] - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -11) * size).all()


def test_a_million_sequences_of_one_position():
    """More blocks than a launch takes: a position that sees itself alone gets its value
    back, and gives its output's gradient to it.  P is 1 to 2^-20, so 1 in bf16; dP - D is
    off by four roundings of a sum of at most 128 products of numbers below 6."""
    batch, heads, hd = (1 << 20) + 5, 8, 128
    g = torch.Generator("cuda").manual_seed(2)
    q, k, v, do = (torch.randn((batch, 1, heads, hd), generator=g, device="cuda", dtype=torch.bfloat16)
                   .clamp_(-6, 6) for _ in range(4))
    out, lse = hcmix.grouped_attention_forward(q, k, v)
    assert torch.equal(out, v)
    dq, dk, dv = hcmix.grouped_attention_backward(q, k, v, out, lse, do)
    assert torch.equal(dv, do)
    limit = 4 * 2.0 ** -24 * 128 * 6 * 6 * 6 * hd ** -0.5
    assert max(dq.abs().max().item(), dk.abs().max().item()) <= limit


@pytest.mark.parametrize("n_k", [70, 300])
def test_key_gradients_of_the_last_of_a_million_queries(n_k):
    """The key gradients where only the last 50 queries' outputs have a gradient (all
    others add zeros): those queries' own, element by element, from rows past 2^31
    elements."""
    n, heads, hd = 1 << 20, 33, 64
    g = torch.Generator("cuda").manual_seed(3)
    q = torch.randn((1, n, heads, hd), generator=g, device="cuda", dtype=torch.bfloat16)
    assert q.numel() > 1 << 31
    k, v = (torch.randn((1, n_k, heads, hd), generator=g, device="cuda", dtype=torch.bfloat16)
            for _ in range(2))
    do = torch.zeros_like(q)
    s = slice(n - 50, n)
    do[:, s] = torch.randn((1, 50, heads, hd), generator=g, device="cuda", dtype=torch.bfloat16)
    out, lse = hcmix.grouped_attention_forward(q, k, v, causal=False)
    got = hcmix.grouped_attention_backward(q, k, v, out, lse, do, causal=False)
    assert not got[0][:, :n - 50].any()
    ref, bounds = grouped.backward(host(q[:, s]), host(k), host(v), host(do[:, s]), causal=False)
    for name, t, r, b in zip(("dq", "dk", "dv"), (got[0][:, s], *got[1:]), ref, bounds):
        err = np.abs(host(t) - r)
        print(f"  {name}: largest error {err.max():.2e}, of its bound {(err / b).max():.2f}", flush=True)
        assert (err <= b).all(), name
