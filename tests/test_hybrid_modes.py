"""Which attention a hybrid stack's attention layers run, on the CPU: the library's
calls are replaced by ones that note what they are asked for."""
import pytest
import torch

from paper_2609_18145_amd import hcmix
from paper_2609_18145_amd.hybrid import HybridStack


@pytest.fixture()
def calls(monkeypatch):
    seen = []

    def linear(x, w, out=None):
        return (x.float() @ w.float().T).to(x.dtype)

    def linear_backward(x, w, dy):
        return (dy.float() @ w.float()).to(x.dtype), dy.float().T @ x.float()

    def fixed(qkv):
        seen.append(("fixed", True))
        return torch.zeros_like(qkv[:, :, 0]), torch.zeros(qkv.shape[0], qkv.shape[3], qkv.shape[1])

    def fixed_backward(qkv, out, lse, dout):
        seen.append(("fixed", True))
        return torch.zeros_like(qkv)

    def grouped(q, k, v, causal=True, lengths=None, scale=None, out=None, lse=None):
        seen.append(("grouped", causal))
        return torch.zeros(q.shape, dtype=q.dtype), torch.zeros(q.shape[0], q.shape[2], q.shape[1])

    def grouped_backward(q, k, v, out, lse, dout, causal=True, lengths=None, scale=None, dq=None,
                         dk=None, dv=None, workspace=None):
        seen.append(("grouped", causal))
        for t in (dq, dk, dv):
            t.zero_()
        return dq, dk, dv
    for name, f in (("linear_forward", linear), ("linear_backward", linear_backward),
                    ("attention_forward", fixed), ("attention_backward", fixed_backward),
                    ("grouped_attention_forward", grouped),
                    ("grouped_attention_backward", grouped_backward)):
        monkeypatch.setattr(hcmix, name, f)
    return seen


@pytest.mark.parametrize("n,kv,causal,want", [
    (64, 2, True, ("fixed", True)),          # the fixed core, which is causal
    (64, 2, False, ("grouped", False)), (40, 2, False, ("grouped", False)),
    (64, 1, False, ("grouped", False)), (40, 2, True, ("grouped", True)),
    (64, 1, True, ("grouped", True))])
def test_attention_layers_take_the_stacks_direction(calls, n, kv, causal, want):
    heads, hd, width = 2, 64, 64
    g = torch.Generator().manual_seed(n)
    wqkv = torch.randn(((heads + 2 * kv) * hd, width), generator=g).to(torch.bfloat16)
    wout = torch.randn((width, heads * hd), generator=g).to(torch.bfloat16)
    h = HybridStack(["attn"], [], [], [(wqkv, wout)], heads, causal=causal, kv_heads=kv)
    x = torch.randn((2, n, width), generator=g).to(torch.bfloat16)
    y = h.forward_segment(0, x)
    h._dw_in, h.dw_attn = [], [None]
    h.backward_segment(0, torch.ones_like(y))
    assert calls == [want, want]


def test_a_stack_of_attention_layers_alone_has_a_backward(calls):
    g = torch.Generator().manual_seed(1)
    attn = [(torch.randn((6 * 64, 64), generator=g).to(torch.bfloat16),
             torch.randn((64, 128), generator=g).to(torch.bfloat16)) for _ in range(2)]
    h = HybridStack(["attn", "attn"], [], [], attn, 2)
    x = torch.randn((2, 32, 64), generator=g).to(torch.bfloat16)
    dx = h.backward(torch.ones_like(h.forward(x)))
    assert dx.shape == x.shape and h.dw_self == [] and h.dw_off == []
    assert [[w.shape for w in p] for p in h.dw_attn] == [[(384, 64), (64, 128)]] * 2


@pytest.mark.parametrize("batch", [2, 3])
def test_a_decoder_takes_its_own_batch(batch):
    """An odd batch is copied into rows of the decoder's own: one row of x is not given
    to every window, nor another type converted."""
    attn = (torch.zeros((6 * 64, 64), dtype=torch.bfloat16), torch.zeros((64, 128), dtype=torch.bfloat16))
    d = HybridStack(["attn"], [], [], [attn], 2).decoder(batch, 16, "cpu")
    bf = torch.bfloat16
    for x, match in ((torch.zeros((1, 64), dtype=bf), "shape"), (torch.zeros(64, dtype=bf), "shape"),
                     (torch.zeros((batch, 1), dtype=bf), "shape"),
                     (torch.zeros((batch, 64)), "dtype"), (torch.zeros((batch, 64), dtype=bf), "GPU")):
        with pytest.raises(ValueError, match=match):
            d.step(x, 0)
