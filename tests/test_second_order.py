"""Gradients of gradients through the attention layers' autograd functions, on the CPU:
the library's calls are replaced by untracked ones of the same results."""
import pytest
import torch

from paper_2609_18145_amd import hcmix

f64 = torch.float64


def rotary(x, freqs, positions=None, layout="half", inverse=False, scale=1.0, out=None):
    """hcmix.rotary from its definition, untracked as a library call is."""
    with torch.no_grad():
        b, n, _, _ = x.shape
        pos = torch.arange(n).expand(b, n) if positions is None else positions
        t = pos.to(f64)[:, :, None, None] * freqs * (-1 if inverse else 1)
        rot = 2 * len(freqs)
        ia = torch.arange(rot // 2) if layout == "half" else torch.arange(0, rot, 2)
        ib = ia + (rot // 2 if layout == "half" else 1)
        y, a, c = x.clone(), x[..., ia], x[..., ib]
        y[..., ia] = scale * (a * t.cos() - c * t.sin())
        y[..., ib] = scale * (c * t.cos() + a * t.sin())
        return y


@pytest.mark.parametrize("layout,scale,positions", [("half", 1.0, None), ("pairs", 0.7, [[5, 900, 2], [0, 1, 7]])])
def test_rotary_has_gradients_of_gradients(monkeypatch, layout, scale, positions):
    monkeypatch.setattr(hcmix, "rotary", rotary)
    freqs = hcmix.rotary_frequencies(4, device="cpu")[0]
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32)
    g = torch.Generator().manual_seed(1)
    x = torch.randn((2, 3, 2, 6), generator=g, dtype=f64).requires_grad_(True)

    def turned(x):
        return hcmix.Rotary.apply(x, freqs, pos, layout, scale)
    assert torch.autograd.gradcheck(turned, (x,))
    assert torch.autograd.gradgradcheck(turned, (x,))
    # a path around the gradient as well: what was lost with no error
    y = turned(x)
    dx, = torch.autograd.grad((y ** 3).sum(), x, create_graph=True)
    got, = torch.autograd.grad((dx * x).sum(), x)
    u = rotary(x.detach(), freqs, pos, layout, scale=scale)
    want = 9 * rotary(u ** 2, freqs, pos, layout, inverse=True, scale=scale)
    # d/dx sum(x . R^T 3 (R x)^2) = d/dx 3 sum((R x)^3)
    torch.testing.assert_close(got, want)


def attention(q, k, v, causal=True, lengths=None, scale=None, out=None, lse=None):
    """hcmix.grouped_attention_forward of one key/value head per query head, untracked."""
    with torch.no_grad():
        s = q.shape[3] ** -0.5 * torch.matmul(q.transpose(1, 2), k.permute(0, 2, 3, 1))
        if causal:
            i, j = torch.arange(s.shape[2])[:, None], torch.arange(s.shape[3])
            s = s.masked_fill(j > i + s.shape[3] - s.shape[2], float("-inf"))
        return (s.softmax(3) @ v.transpose(1, 2)).transpose(1, 2).contiguous(), s.logsumexp(3)


def attention_backward(q, k, v, out, lse, dout, causal=True, lengths=None, scale=None, **kw):
    with torch.enable_grad():
        leaves = [t.detach().requires_grad_(True) for t in (q, k, v)]
        s = q.shape[3] ** -0.5 * torch.matmul(leaves[0].transpose(1, 2), leaves[1].permute(0, 2, 3, 1))
        if causal:
            i, j = torch.arange(s.shape[2])[:, None], torch.arange(s.shape[3])
            s = s.masked_fill(j > i + s.shape[3] - s.shape[2], float("-inf"))
        out = (s.softmax(3) @ leaves[2].transpose(1, 2)).transpose(1, 2)
        return torch.autograd.grad(out, leaves, dout.detach())


def test_attention_refuses_gradients_of_gradients(monkeypatch):
    """The first order is right also with a graph of it; the second says that there is none."""
    monkeypatch.setattr(hcmix, "grouped_attention_forward", attention)
    monkeypatch.setattr(hcmix, "grouped_attention_backward", attention_backward)
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn((1, 3, 2, 4), generator=g, dtype=f64).requires_grad_(True) for _ in range(3))
    assert torch.autograd.gradcheck(hcmix.GroupedAttention.apply, (q, k, v))
    y = hcmix.GroupedAttention.apply(q, k, v)
    dq, = torch.autograd.grad((y ** 2).sum(), q, create_graph=True)
    want, = torch.autograd.grad((hcmix.GroupedAttention.apply(q, k, v) ** 2).sum(), q)
    assert torch.equal(dq, want)
    with pytest.raises(RuntimeError, match="differentiate twice"):
        (dq * q).sum().backward()


def test_fixed_attention_refuses_gradients_of_gradients(monkeypatch):
    def forward(qkv):
        out, lse = attention(*qkv.unbind(2))
        return out, lse

    def backward(qkv, out, lse, dout):
        return torch.stack(attention_backward(*qkv.unbind(2), out, lse, dout), 2)
    monkeypatch.setattr(hcmix, "attention_forward", forward)
    monkeypatch.setattr(hcmix, "attention_backward", backward)
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((1, 3, 3, 2, 4), generator=g, dtype=f64).requires_grad_(True)
    assert torch.autograd.gradcheck(hcmix.Attention.apply, (qkv,))
    dqkv, = torch.autograd.grad((hcmix.Attention.apply(qkv) ** 2).sum(), qkv, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiate twice"):
        (dqkv * qkv).sum().backward()


def test_stack_refuses_gradients_of_gradients(monkeypatch):
    """(A stack of one map, x W' for the library's layers.)"""
    def forward(x, w_selfs, w_offs, layers, causal):
        with torch.no_grad():
            return [x, x @ w_selfs[0].T]

    def backward(xs, w_selfs, w_offs, layers, dy, causal):
        with torch.no_grad():
            dw = dy.reshape(-1, dy.shape[-1]).T @ xs[0].reshape(-1, xs[0].shape[-1])
            return dy @ w_selfs[0], [dw], [torch.zeros_like(w_offs[0])]
    monkeypatch.setattr(hcmix, "stack_forward", forward)
    monkeypatch.setattr(hcmix, "stack_backward", backward)
    g = torch.Generator().manual_seed(4)
    x, ws, wo = (torch.randn(s, generator=g, dtype=f64).requires_grad_(True)
                 for s in ((2, 3, 4), (4, 4), (4, 4)))
    assert torch.autograd.gradcheck(lambda *t: hcmix.Stack.apply(t[0], [0], True, *t[1:]), (x, ws, wo))
    y = hcmix.Stack.apply(x, [0], True, ws, wo)
    dx, = torch.autograd.grad((y ** 3).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiate twice"):
        (dx * x).sum().backward()
