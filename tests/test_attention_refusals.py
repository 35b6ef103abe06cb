"""What the attention layers past the fixed windows refuse, on the CPU: the C ABI
before anything is enqueued, the binding before the library is reached."""
import ctypes

import pytest
import torch

from paper_2609_18145_amd import hcmix
from paper_2609_18145_amd.hybrid import HybridStack

OK, INVALID, UNSUPPORTED = hcmix.HCMIX_OK, hcmix.HCMIX_ERR_INVALID_VALUE, hcmix.HCMIX_ERR_UNSUPPORTED
# addresses that are never dereferenced, 256 MiB apart
P = [0x10000000 * (k + 1) for k in range(16)]
NAN, INF = float("nan"), float("inf")


def call(name, args, changes):
    args = dict(args)
    assert set(changes) <= set(args), changes
    args.update(changes)
    return getattr(hcmix.load(), name)(*args.values())


ROTARY = dict(rows=10, heads=4, head_dim=64, rot=64, layout=0, inverse=0, dtype=1, x=P[0], xs=256,
              positions=P[1], period=0, freqs=P[2], scale=1.0, y=P[3], ys=256, stream=None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), INVALID), (dict(freqs=None), INVALID), (dict(y=None), INVALID),
    (dict(rows=0), INVALID), (dict(rows=(1 << 30) + 1), INVALID), (dict(heads=0), INVALID),
    (dict(heads=1025, xs=1 << 20, ys=1 << 20), INVALID), (dict(head_dim=0), INVALID),
    (dict(head_dim=514, xs=4096, ys=4096), INVALID), (dict(rot=0), INVALID), (dict(rot=66), INVALID),
    (dict(layout=2), INVALID), (dict(dtype=2), INVALID), (dict(scale=NAN), INVALID),
    (dict(scale=INF), INVALID), (dict(xs=255), INVALID), (dict(ys=128), INVALID),
    (dict(positions=None), INVALID),                       # and no period
    (dict(y=P[0] + 512 * 9), INVALID),                     # overlaps x's last row
    (dict(y=P[0], ys=512), INVALID),                       # in place with another stride
    (dict(y=P[2] - 64), INVALID), (dict(y=P[1] - 5120 + 4), INVALID),
    (dict(xs=600, ys=600, y=P[0] + 2 * 255), INVALID),     # rows between rows that touch
    (dict(rot=63), UNSUPPORTED), (dict(head_dim=63, rot=62), UNSUPPORTED),
    (dict(x=P[0] + 1), UNSUPPORTED), (dict(dtype=0, y=P[3] + 2), UNSUPPORTED),
    (dict(freqs=P[2] + 4), UNSUPPORTED), (dict(positions=P[1] + 2), UNSUPPORTED),
])
def test_rotary_rejects(kw, code):
    assert call("hcmix_rotary", ROTARY, kw) == code


FWD = dict(batch=2, n_q=10, n_k=12, heads=4, kv=2, hd=64, causal=1, scale=0.125, lengths=P[0], q=P[1],
           qs=256, k=P[2], ks=128, v=P[3], vs=128, out=P[4], lse=P[5], stream=None)
SHARED = [
    (dict(batch=0), INVALID), (dict(n_q=0), INVALID), (dict(n_k=-1), INVALID),
    (dict(n_q=(1 << 20) + 1), INVALID), (dict(n_k=(1 << 20) + 1), INVALID),
    (dict(batch=1 << 28), INVALID), (dict(heads=5), INVALID), (dict(kv=0), INVALID),
    (dict(heads=0), INVALID), (dict(heads=2048, qs=1 << 20), INVALID), (dict(causal=2), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=NAN), INVALID),
    (dict(scale=INF), INVALID), (dict(scale=2.0 ** -25), INVALID), (dict(scale=2.0 ** 25), INVALID),
    (dict(q=None), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(out=None), INVALID), (dict(lse=None), INVALID),
    (dict(qs=248), INVALID), (dict(ks=120), INVALID), (dict(vs=0), INVALID),
    (dict(qs=(1 << 32) + 8), INVALID), (dict(hd=96), UNSUPPORTED), (dict(hd=256), UNSUPPORTED),
    (dict(qs=260), UNSUPPORTED), (dict(vs=132), UNSUPPORTED), (dict(q=P[1] + 8), UNSUPPORTED),
    (dict(k=P[2] + 2), UNSUPPORTED), (dict(out=P[4] + 4), UNSUPPORTED),
    (dict(lse=P[5] + 2), UNSUPPORTED), (dict(lengths=P[0] + 1), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,code", SHARED + [
    (dict(out=P[1] + 2560), INVALID), (dict(lse=P[3]), INVALID), (dict(lse=P[4] + 64), INVALID),
    (dict(out=P[0] - 5120 + 4), INVALID)])
def test_grouped_forward_rejects(kw, code):
    assert call("hcmix_grouped_attention_forward", FWD, kw) == code


BWD = dict(batch=2, n_q=10, n_k=12, heads=4, kv=2, hd=64, causal=1, scale=0.125, lengths=P[0], q=P[1],
           qs=256, k=P[2], ks=128, v=P[3], vs=128, out=P[4], lse=P[5], dout=P[6], dq=P[7], dqs=256,
           dk=P[8], dks=128, dv=P[9], dvs=128, ws=P[10], wsb=1 << 20, stream=None)


@pytest.mark.parametrize("kw,code", SHARED + [
    (dict(dout=None), INVALID), (dict(dq=None), INVALID), (dict(dk=None), INVALID),
    (dict(dv=None), INVALID), (dict(ws=None), INVALID), (dict(wsb=2047), INVALID),
    (dict(dqs=128), INVALID), (dict(dks=64), INVALID), (dict(dvs=124), INVALID),
    (dict(dq=P[1]), INVALID), (dict(dk=P[2] + 256), INVALID), (dict(dv=P[8]), INVALID),
    (dict(ws=P[6]), INVALID), (dict(dq=P[4]), INVALID),
    # dk and dv between the rows of one packed buffer, but touching
    (dict(dks=512, dvs=512, dv=P[8] + 2 * 120), INVALID),
    (dict(dqs=260), UNSUPPORTED), (dict(dk=P[8] + 8), UNSUPPORTED), (dict(ws=P[10] + 64), UNSUPPORTED),
    (dict(dout=P[6] + 8), UNSUPPORTED)])
def test_grouped_backward_rejects(kw, code):
    assert call("hcmix_grouped_attention_backward", BWD, kw) == code


def test_grouped_workspace_query():
    q = hcmix.load().hcmix_grouped_attention_backward_workspace_bytes
    # two statistics of every query row, rows padded to 32
    assert q(2, 10, 12, 4, 2, 64) == 2 * 4 * 32 * 2 * 4
    # few key tiles, many queries: fp32 sums of dk and dv beside them
    assert q(1, 4096, 1, 4, 2, 128) > 4 * 4096 * 2 * 4
    for bad in ((0, 1, 1, 1, 1, 64), (1, 0, 1, 1, 1, 64), (1, 1, 1, 3, 2, 64), (1, 1, 1, 1, 1, 32)):
        assert q(*bad) == 0


KV = dict(batch=2, capacity=100, kv=2, hd=64)
KV_SHARED = [
    (dict(batch=0), INVALID), (dict(batch=65536), INVALID), (dict(capacity=0), INVALID),
    (dict(capacity=(1 << 24) + 1), INVALID), (dict(kv=0), INVALID), (dict(kv=2048), INVALID),
    (dict(tokens=0), INVALID), (dict(tokens=(1 << 16) + 1), INVALID), (dict(cache=None), INVALID),
    (dict(cb=65791), INVALID), (dict(hd=32), UNSUPPORTED), (dict(cache=P[5] + 128), UNSUPPORTED),
]
APPEND = dict(**KV, tokens=3, k=P[0], ks=128, v=P[1], vs=128, positions=P[2], counts=P[3], cache=P[5],
              cb=65792, stream=None)
READ = dict(**KV, tokens=3, first=P[0], lengths=P[1], cache=P[5], cb=65792, k=P[2], v=P[3], stream=None)
ATTEND = dict(batch=2, capacity=100, heads=4, kv=2, hd=64, tokens=3, scale=0.125, q=P[0], qs=256,
              lengths=P[1], longest=100, cache=P[5], cb=65792, out=P[2], ws=P[3], wsb=1 << 24,
              stream=None)


@pytest.mark.parametrize("kw,code", KV_SHARED + [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(positions=None), INVALID),
    (dict(ks=120), INVALID), (dict(vs=64), INVALID), (dict(k=P[5] + 1024), INVALID),
    (dict(positions=P[5] + 65784), INVALID), (dict(ks=132), UNSUPPORTED),
    (dict(v=P[1] + 8), UNSUPPORTED), (dict(positions=P[2] + 2), UNSUPPORTED),
    (dict(counts=P[3] + 1), UNSUPPORTED)])
def test_append_rejects(kw, code):
    assert call("hcmix_kv_cache_append", APPEND, kw) == code


@pytest.mark.parametrize("kw,code", KV_SHARED + [
    (dict(first=None), INVALID), (dict(lengths=None), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(v=P[2] + 16), INVALID), (dict(k=P[5]), INVALID),
    (dict(k=P[2] + 8), UNSUPPORTED), (dict(first=P[0] + 2), UNSUPPORTED)])
def test_read_rejects(kw, code):
    assert call("hcmix_kv_cache_read", READ, kw) == code


@pytest.mark.parametrize("kw,code", KV_SHARED + [
    (dict(q=None), INVALID), (dict(lengths=None), INVALID), (dict(out=None), INVALID),
    (dict(heads=3), INVALID), (dict(scale=0.0), INVALID), (dict(scale=INF), INVALID),
    (dict(longest=0), INVALID), (dict(longest=101), INVALID), (dict(qs=248), INVALID),
    (dict(out=P[0]), INVALID), (dict(out=P[5] + 4096), INVALID), (dict(qs=260), UNSUPPORTED),
    (dict(q=P[0] + 2), UNSUPPORTED), (dict(lengths=P[1] + 2), UNSUPPORTED)])
def test_cache_attention_rejects(kw, code):
    assert call("hcmix_kv_cache_attention", ATTEND, kw) == code


def test_cache_attention_wants_its_workspace():
    """A long sequence is split over the chip, through a workspace."""
    long = dict(capacity=10000, longest=10000, cb=1 << 30)
    need = hcmix.load().hcmix_kv_cache_attention_workspace_bytes(2, 10000, 4, 2, 64, 3, 10000)
    assert need > 0
    for kw, code in ((dict(ws=None), INVALID), (dict(wsb=need - 1), INVALID),
                     (dict(ws=P[3] + 16), UNSUPPORTED), (dict(ws=P[0]), INVALID)):
        assert call("hcmix_kv_cache_attention", {**ATTEND, **long, "cache": 1 << 40}, kw) == code


def test_cache_bytes():
    """64-token blocks of keys and values, a byte a number, two scales to a block."""
    q = hcmix.load().hcmix_kv_cache_bytes
    assert q(2, 100, 2, 64) == 2 * 2 * 2 * 2 * 64 * 64 + 256      # 64 bytes of scales, to 256
    assert q(1, 64, 1, 128) == 2 * 64 * 128 + 256
    for bad in ((0, 1, 1, 64), (1, 0, 1, 64), (1, 1, 0, 64), (1, 1, 1, 80), (65535, 1 << 24, 1024, 128)):
        assert q(*bad) == 0


# ---- the binding ----

bf, f32, i32, f64 = torch.bfloat16, torch.float32, torch.int32, torch.float64


def z(*shape, dtype=bf):
    return torch.zeros(shape, dtype=dtype)


@pytest.fixture()
def untouched(monkeypatch):
    def boom():
        raise AssertionError("the library was reached")
    monkeypatch.setattr(hcmix, "load", boom)


def refused(fn, *args, match, **kw):
    with pytest.raises(ValueError, match=match):
        fn(*args, **kw)


def test_rotary_checks(untouched):
    x, f = z(2, 5, 3, 64), z(32, dtype=f64)
    refused(hcmix.rotary, z(5, 3, 64), f, match="x")
    refused(hcmix.rotary, z(2, 5, 3, 64, dtype=torch.float16), f, match="dtype")
    refused(hcmix.rotary, x.transpose(1, 2), f, match="strides")
    refused(hcmix.rotary, x[:, ::2].expand(2, 3, 3, 64)[:, :, :, ::2], f, match="strides")
    refused(hcmix.rotary, x[:, :3], f, match="strides")          # a gap between the sequences
    refused(hcmix.rotary, x, z(32, dtype=f32), match="freqs")
    refused(hcmix.rotary, x, f, z(2, 4, dtype=i32), match="positions")
    refused(hcmix.rotary, x, f, z(2, 5, dtype=torch.int64), match="positions")
    refused(hcmix.rotary, x, f, layout="rows", match="layout")
    refused(hcmix.rotary, x, f, out=z(2, 5, 3, 32), match="out")
    refused(hcmix.rotary, x, f, match="GPU")
    refused(hcmix.rotary_frequencies, 7, device="cpu", match="rot_dim")
    refused(hcmix.rotary_frequencies, 8, base=0.0, device="cpu", match="base")
    refused(hcmix.rotary_frequencies, 8, factor=0.5, device="cpu", match="factor")
    refused(hcmix.rotary_frequencies, 8, scaling="cubic", device="cpu", match="scaling")
    refused(hcmix.rotary_frequencies, 8, scaling="yarn", device="cpu", match="yarn")


def test_frequencies_of_scaled_contexts(untouched):
    f, s = hcmix.rotary_frequencies(8, device="cpu")
    torch.testing.assert_close(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=f64))
    assert s == 1.0 and f.dtype == f64
    lin, _ = hcmix.rotary_frequencies(8, scaling="linear", factor=4.0, device="cpu")
    torch.testing.assert_close(lin, f / 4)
    ntk, _ = hcmix.rotary_frequencies(8, scaling="ntk", factor=4.0, device="cpu")
    assert ntk[0] == 1.0 and abs(ntk[3] * 4 / f[3] - 1) < 1e-12
    # turns within 1000 positions: 159, 16, 1.6, 0.16
    yarn, s = hcmix.rotary_frequencies(8, scaling="yarn", factor=4.0, original_length=1000,
                                       device="cpu")
    assert yarn[0] == f[0] and yarn[3] == f[3] / 4 and f[1] / 4 < yarn[1] < f[1]
    assert abs(s - 1.138629436111989) < 1e-12


def test_grouped_checks(untouched):
    q, k, v = z(2, 5, 4, 64), z(2, 7, 2, 64), z(2, 7, 2, 64)
    fwd, bwd = hcmix.grouped_attention_forward, hcmix.grouped_attention_backward
    refused(fwd, z(2, 5, 256), k, v, match="q")
    refused(fwd, q, z(3, 7, 2, 64), v, match="k")
    refused(fwd, q, z(2, 7, 2, 128), v, match="k")
    refused(fwd, q, k, z(2, 6, 2, 64), match="v")
    refused(fwd, q, k, z(2, 7, 2, 64, dtype=f32), match="v")
    refused(fwd, q, k.transpose(1, 2).contiguous().transpose(1, 2), v, match="strides")
    refused(fwd, q, k, v, lengths=z(3, dtype=i32), match="lengths")
    refused(fwd, q, k, v, lengths=z(2, dtype=torch.int64), match="lengths")
    refused(fwd, q, k, v, out=z(2, 5, 2, 64), match="out")
    refused(fwd, q, k, v, lse=z(2, 5, 4, dtype=f32), match="lse")
    refused(fwd, q, k, v, match="GPU")
    out, lse = z(2, 5, 4, 64), z(2, 4, 5, dtype=f32)
    refused(bwd, q, k, v, out, lse, z(2, 5, 4, 64, dtype=f32), match="dout")
    refused(bwd, q, k, v, out, z(2, 4, 6, dtype=f32), out, match="lse")
    refused(bwd, q, k, v, out, lse, out, dk=z(2, 7, 4, 64), match="dk")
    refused(bwd, q, k, v, out, lse, out, dv=z(2, 2, 7, 64).transpose(1, 2), match="strides")
    refused(bwd, q, k, v, out, lse, out, match="GPU")


def test_cache_checks(untouched):
    k, pos, c = z(2, 3, 2, 64), z(2, dtype=i32), z(1024, dtype=torch.uint8)
    refused(hcmix.kv_cache_append, z(6, 128), k, pos, c, 10, match="k")
    refused(hcmix.kv_cache_append, k, z(2, 3, 1, 64), pos, c, 10, match="v")
    refused(hcmix.kv_cache_append, k, k, z(3, dtype=i32), c, 10, match="positions")
    refused(hcmix.kv_cache_append, k, k, pos, c, 10, counts=z(2), match="counts")
    refused(hcmix.kv_cache_append, k, k, pos, None, 10, match="cache")
    refused(hcmix.kv_cache_append, k, k, pos, c, 10, match="GPU")
    refused(hcmix.kv_cache_read, c, 10, 2, 64, z(2, 1, dtype=i32), pos, 3, match="first")
    refused(hcmix.kv_cache_read, c, 10, 2, 64, pos, z(2), 3, match="lengths")
    refused(hcmix.kv_cache_read, c, 10, 2, 64, pos, pos, 3, k=z(2, 4, 2, 64), match="k")
    refused(hcmix.kv_cache_read, c, 10, 2, 64, pos, pos, 3, match="GPU")
    refused(hcmix.kv_cache_attention, z(2, 256), pos, c, 10, 2, match="q")
    refused(hcmix.kv_cache_attention, z(2, 1, 4, 64), z(2), c, 10, 2, match="lengths")
    refused(hcmix.kv_cache_attention, z(2, 1, 4, 64), pos, c, 10, 2, out=z(2, 1, 2, 64), match="out")
    refused(hcmix.kv_cache_attention, z(2, 1, 4, 64), pos, c, 10, 2, match="GPU")


def test_a_cache_that_the_library_has_no_kernel_for():
    refused(hcmix.alloc_kv_cache, 2, 10, 2, 96, "cpu", match="not supported")


def test_hybrid_decoder_is_causal_only(untouched):
    h = HybridStack([0, 1], [z(64, 64)] * 2, [z(64, 64)] * 2, [], 1, causal=False)
    refused(h.decoder, 2, 16, "cpu", match="causal")


def test_native_calls_leave_other_operands_to_the_binding():
    """Operands off the GPU, of other types or too few: None, and no error left behind."""
    m = hcmix._native()
    q, pos, c = z(2, 3, 2, 64), z(2, dtype=i32), z(1024, dtype=torch.uint8)
    f = z(32, dtype=f64)
    for call, args in ((m.rotary, (1, q, f, None, 0, 0, 1.0, None, 0)), (m.rotary, (1,)),
                       (m.grouped_forward, (1, q, q, q, 1, None, None, None, None, 0)),
                       (m.grouped_forward, (1, None, q, q, 1, None, None, None, None, 0)),
                       (m.grouped_backward, (1, 1, q, q, q, q, q, q, 1, None, None, None, None, None, 0)),
                       (m.cache_append, (1, q, q, pos, None, c, 10, 0)), (m.cache_append, ()),
                       (m.cache_read, (1, pos, pos, c, 10, 2, 64, 3, None, None, 0)),
                       (m.cache_attention, (1, 1, q, pos, c, 10, 2, None, None, None, 0)),
                       (m.heads, (q, (None,) * 4, bf, None)), (m.heads, ([1], (None,) * 4, bf, None))):
        assert call(*args) is None


@pytest.mark.gpu
def test_refusals_on_the_gpu_say_what_is_wrong():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    g = lambda *a, **k: z(*a, **k).cuda()  # noqa: E731
    q, k, f, pos = g(2, 5, 4, 64), g(2, 7, 2, 64), g(32, dtype=f64), g(2, dtype=i32)
    out, lse = g(2, 5, 4, 64), g(2, 4, 5, dtype=f32)
    cache = hcmix.alloc_kv_cache(2, 10, 2, 64, "cuda")
    for fn, args, kw, match in (
            (hcmix.rotary, (q, g(32, dtype=f32)), {}, "freqs"),
            (hcmix.rotary, (q, f.cpu()), {}, "freqs"),
            (hcmix.rotary, (q, f), dict(positions=g(2, 4, dtype=i32)), "positions"),
            (hcmix.rotary, (q, f), dict(out=g(2, 5, 3, 64)), "out"),
            (hcmix.rotary, (q, f), dict(layout="x"), "layout"),
            (hcmix.grouped_attention_forward, (q, k, g(2, 6, 2, 64)), {}, "v"),
            (hcmix.grouped_attention_forward, (q, k.cpu(), k), {}, "k"),
            (hcmix.grouped_attention_forward, (q, k, k), dict(lengths=g(3, dtype=i32)), "lengths"),
            (hcmix.grouped_attention_forward, (q, k, k), dict(out=out[:, :, ::2]), "out"),
            (hcmix.grouped_attention_backward, (q, k, k, out, lse, g(2, 5, 4, 64, dtype=f32)), {}, "dout"),
            (hcmix.grouped_attention_backward, (q, k, k, out, lse, out), dict(dv=g(2, 7, 4, 64)), "dv"),
            (hcmix.kv_cache_append, (k, k, g(3, dtype=i32), cache, 10), {}, "positions"),
            (hcmix.kv_cache_append, (k, k, pos, cache.cpu(), 10), {}, "cache"),
            (hcmix.kv_cache_read, (cache, 10, 2, 64, pos, pos.cpu(), 3), {}, "lengths"),
            (hcmix.kv_cache_attention, (q, g(2, dtype=torch.int64), cache, 10, 2), {}, "lengths")):
        refused(fn, *args, match=match, **kw)
    for fn, args, kw in ((hcmix.grouped_attention_forward, (g(2, 5, 3, 64), k, k), {}),   # 3 heads over 2
                         (hcmix.grouped_attention_forward, (g(2, 5, 2, 32),) * 3, {}),
                         (hcmix.grouped_attention_backward, (q, k, k, out, lse, out), dict(scale=0.0)),
                         (hcmix.kv_cache_append, (k, k, pos, cache, 1000), {}),           # a short cache
                         (hcmix.kv_cache_attention, (q, pos, cache, 10, 3), {}),
                         (hcmix.rotary, (q, f), dict(scale=float("nan")))):
        with pytest.raises(hcmix.HcmixError):
            fn(*args, **kw)
    torch.cuda.synchronize()
