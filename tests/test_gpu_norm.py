"""Residual addition and RMS norm on the GPU against float64.

Error bounds: the sum is one rounding of x + r (exact against the same rounding in torch). The mean of squares of cols fp32
terms is off by at most 85 2^-24 relative (at most 64 terms one after another a lane, five steps of a tree and 16 warps');
half of that in the root. Square root, quotient, two products and eps are five roundings of 2^-24. bf16 outputs half a bf16 step
(2^-8 relative, with what is before it). Blocks: the values that the quantising calls make of y, to the half steps stated."""
import numpy as np
import pytest
import torch

import fp4_ref as R4
from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu


def stream(rng, T, d, pad, dtype, scale=1.0):
    x = rng.standard_normal((T, d + pad)) * scale * np.exp(rng.standard_normal((T, 1)))
    x[:, rng.random(d + pad) < 0.02] *= 20.0
    return torch.from_numpy(x.astype(np.float32)).cuda().to(dtype)[:, :d]


def reference(s, w, eps):
    """float64 norm of the stored sum and the bound on the fp32 one's error."""
    v = s.double()
    y = v / (v.square().mean(1, keepdim=True) + eps).sqrt()
    if w is not None:
        y = y * w.double()
    return y, 48 * 2.0 ** -24 * y.abs()


SHAPES = [(1, 1), (1, 768), (3, 32), (5, 33), (2, 127), (300, 192), (77, 384), (9, 512), (130, 520), (33, 768), (6, 1131), (4, 2048),
          (5, 4096), (3, 5000), (2, 8192), (3, 16384), (2, 16385), (2, 32768)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("pad", [0, 3, 8])
def test_norm(T, d, pad, dtype):
    rng = np.random.default_rng(T + 10 * d + pad)
    x, r = stream(rng, T, d, pad, dtype), stream(rng, T, d, pad, dtype, 3.0)
    for res, w_dtype, eps in ((r, dtype, 1e-5), (None, torch.float32, 0.0), (r, None, 1.0), (r, torch.bfloat16, 1e-6)):
        w = None if w_dtype is None else stream(rng, 1, d, 0, w_dtype)[0]
        want = x if res is None else (x.float() + res.float()).to(dtype)
        y, err = reference(want, w, eps)
        s = torch.full((T + 1, d + pad), float("nan"), device="cuda", dtype=dtype)
        for out_dtype in (dtype, torch.float32 if dtype == torch.bfloat16 else torch.bfloat16):
            out = torch.full((T + 1, d + pad), float("nan"), device="cuda", dtype=out_dtype)
            cm.clearmoe_rms_norm(x, out[:T, :d], residual=res, sum_out=s[:T, :d], weight=w, eps=eps)
            assert torch.equal(s[:T, :d], want)
            assert bool(((out[:T, :d].double() - y).abs() <= err + (2.0 ** -8 * y.abs() if out_dtype == torch.bfloat16 else 0) + 1e-38).all())
            for t in (s, out):
                assert bool(t[T].isnan().all()) and bool(t[:, d:].isnan().all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("pad", [0, 3, 8])
def test_norm_to_blocks(T, d, pad, dtype):
    """The blocks that quantising the fp32 norm gives, bit for bit: the same y goes either way."""
    rng = np.random.default_rng(T + 10 * d + pad)
    x, r, w = stream(rng, T, d, pad, dtype), stream(rng, T, d, pad, dtype), stream(rng, 1, d, 0, torch.float32)[0]
    if T > 2:
        x[1, d // 2] = float("nan")
        x[2, 0] = float("inf")
    y, s = torch.empty(T, d, device="cuda"), torch.empty(T, d, device="cuda", dtype=dtype)
    cm.clearmoe_rms_norm(x, y, residual=r, weight=w)
    finite = y.isfinite().all(1)
    a, b = cm.fp8_rows(T, d), cm.fp8_rows(T, d)
    a.q.view(torch.uint8).fill_(0x33)
    cm.clearmoe_rms_norm(x, a, residual=r, sum_out=s, weight=w)
    assert torch.equal(s[finite], (x.float() + r.float()).to(dtype)[finite])
    cm.clearmoe_fp8_quantize_rows(y, b)
    n = -(-d // 128)
    assert torch.equal(a.scale[:, :n], b.scale[:, :n])
    assert torch.equal(a.q.view(torch.uint8)[finite], b.q.view(torch.uint8)[finite])
    if T > 2:  # a NaN is its whole row's; an infinity's row is zeros, and NaN where it stands
        assert bool((a.scale[1, :n] == 255).all()) and a.scale[2, :n].tolist() == [255] + [0] * (n - 1)
    a, b = cm.fp4_matrix(T, d), cm.fp4_matrix(T, d)
    a.q.fill_(0x33)
    cm.clearmoe_rms_norm(x, a, residual=r, weight=w)
    cm.clearmoe_fp4_quantize(y, b)
    assert np.array_equal(R4.scale_bytes(a.scale.cpu().numpy(), T, d), R4.scale_bytes(b.scale.cpu().numpy(), T, d))
    assert torch.equal(a.q[finite], b.q[finite])


@pytest.mark.parametrize("d", [768, 770])
def test_in_place(d):
    rng = np.random.default_rng(4)
    for dtype in (torch.bfloat16, torch.float32):
        x, r, w = stream(rng, 50, d, 0, dtype).contiguous(), stream(rng, 50, d, 0, dtype).contiguous(), stream(rng, 1, d, 0, dtype)[0]
        want, y = torch.empty_like(x), torch.empty_like(x)
        cm.clearmoe_rms_norm(x, y, residual=r, sum_out=want, weight=w)
        a, b = x.clone(), r.clone()
        out = torch.empty_like(x)
        cm.clearmoe_rms_norm(a, out, residual=b, sum_out=b, weight=w)  # the stream updated where it is
        assert torch.equal(b, want) and torch.equal(out, y) and torch.equal(a, x)
        b = r.clone()
        cm.clearmoe_rms_norm(a, a, residual=b, sum_out=b, weight=w)  # and the norm over the sublayer's output
        assert torch.equal(b, want) and torch.equal(a, y)
        a = x.clone()
        cm.clearmoe_rms_norm(a, out, residual=r, sum_out=a, weight=w)
        assert torch.equal(a, want) and torch.equal(out, y)


@pytest.mark.parametrize("d", [64, 65])
def test_special_rows(d):
    x = torch.zeros(6, d, device="cuda")
    x[1, 3] = float("nan")
    x[2, 3] = float("inf")
    x[3] = 1e-30
    x[4] = 1e25  # its squares are past fp32: the row is zero
    x[5, 1] = -2.0
    out = torch.empty_like(x)
    cm.clearmoe_rms_norm(x, out, eps=1e-6)
    assert bool((out[0] == 0).all()) and bool(out[1].isnan().all())
    assert bool(out[2, 3].isnan()) and bool((out[2, :3] == 0).all())
    assert torch.allclose(out[3], x[3] * 1000, rtol=1e-5, atol=0)
    assert bool((out[4] == 0).all())
    cm.clearmoe_rms_norm(x, out, eps=0.0)
    assert bool(out[0].isnan().all())  # 0 / 0
    assert abs(float(out[5, 1]) + d ** 0.5) < 1e-5 * d ** 0.5


def test_many_rows():
    rng = np.random.default_rng(6)
    x = torch.randn(70001, 96, device="cuda", dtype=torch.bfloat16, generator=torch.Generator("cuda").manual_seed(1))
    w = stream(rng, 1, 96, 0, torch.bfloat16)[0]
    out = torch.empty_like(x)
    cm.clearmoe_rms_norm(x, out, weight=w)
    y, err = reference(x, w, 1e-6)
    assert bool(((out.double() - y).abs() <= err + 2.0 ** -8 * y.abs()).all())


def test_far_rows():
    """Offsets past 32 bits."""
    x = torch.zeros(5, 1 << 29, dtype=torch.bfloat16, device="cuda")
    v = stream(np.random.default_rng(8), 5, 100, 0, torch.bfloat16)
    x[:, 8:108] = v
    out = torch.empty(5, 100, dtype=torch.bfloat16, device="cuda")
    cm.clearmoe_rms_norm(x[:, 8:108], x[:, 8:108], sum_out=out)
    y, err = reference(v, None, 1e-6)
    assert torch.equal(out, v)
    assert bool(((x[:, 8:108].double() - y).abs() <= err + 2.0 ** -8 * y.abs()).all())
    assert int((x[:, :8] != 0).sum()) == 0 and int((x[:, 108:116] != 0).sum()) == 0


@pytest.mark.parametrize("blocks", [4, 8])
def test_a_sublayer(blocks):
    """A stream through a norm, two products and the next norm: each step against float64 of what it was given; on a side
    stream and from a graph."""
    rng = np.random.default_rng(blocks)
    T, d, H = 200, 256, 512
    w = {n: stream(rng, 1, d, 0, torch.bfloat16)[0] for n in "ab"}
    mats = [torch.from_numpy((rng.standard_normal(s) * 0.05).astype(np.float32)).cuda() for s in ((H, d), (d, H))]
    new = cm.fp4_matrix if blocks == 4 else cm.fp8_rows
    gemm = cm.clearmoe_fp4_gemm if blocks == 4 else cm.clearmoe_fp8_gemm
    deq = cm.clearmoe_fp4_dequantize if blocks == 4 else cm.clearmoe_fp8_dequantize
    W = []
    for m in mats:
        W.append(cm.fp4_matrix(*m.shape) if blocks == 4 else cm.fp8_weight(*m.shape))
        (cm.clearmoe_fp4_quantize if blocks == 4 else cm.clearmoe_fp8_quantize_weight)(m, W[-1])
    bf = dict(device="cuda", dtype=torch.bfloat16)
    x, hid, y = torch.empty(T, d, **bf), torch.zeros(T, d, **bf), torch.empty(T, d, **bf)
    xq, zq, out = new(T, d), new(T, H), torch.empty(T, d, **bf)

    def sublayer():
        cm.clearmoe_rms_norm(x, xq, residual=hid, sum_out=hid, weight=w["a"])
        gemm(xq, W[0], zq, act=cm.ACT_RELU)
        gemm(zq, W[1], y)
        cm.clearmoe_rms_norm(y, out, residual=hid, sum_out=hid, weight=w["b"])

    def val(m):
        t = torch.empty(m.rows, m.cols, device="cuda")
        deq(m, t)
        return t.double()

    def check(x0, h0):
        torch.cuda.synchronize()
        s = (x0.float() + h0.float()).to(torch.bfloat16)
        n, err = reference(s, w["a"], 1e-6)
        step = 0.2 if blocks == 4 else 2.0 ** -4
        size = 32 if blocks == 4 else 128
        amax = n.abs().view(T, -1, size).amax(2).repeat_interleave(size, 1)
        low = 0.25 * amax / 3 if blocks == 4 else 2.0 ** -10 * 2 * amax / 448
        assert bool(((val(xq) - n).abs() <= 1.2 * err + step * n.abs() + 1.01 * low).all())
        z = (val(xq) @ val(W[0]).T).clamp(min=0)
        zerr = (d + 8) * 2.0 ** -23 * (val(xq).abs() @ val(W[0]).abs().T)
        amax = z.abs().view(T, -1, size).amax(2).repeat_interleave(size, 1)
        low = 0.25 * amax / 3 if blocks == 4 else 2.0 ** -10 * 2 * amax / 448
        assert bool(((val(zq) - z).abs() <= 1.2 * zerr + step * z + 1.01 * low).all())
        o = val(zq) @ val(W[1]).T
        oerr = (H + 8) * 2.0 ** -23 * (val(zq).abs() @ val(W[1]).abs().T)
        assert bool(((y.double() - o).abs() <= oerr + 2.0 ** -8 * o.abs()).all())
        s2 = (y.float() + s.float()).to(torch.bfloat16)
        assert torch.equal(hid, s2)
        n2, err2 = reference(s2, w["b"], 1e-6)
        assert bool(((out.double() - n2).abs() <= err2 + 2.0 ** -8 * n2.abs()).all())

    x.copy_(stream(rng, T, d, 0, torch.bfloat16))
    x0, h0 = x.clone(), hid.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        sublayer()
    check(x0, h0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sublayer()
    for _ in range(2):
        x.copy_(stream(rng, T, d, 0, torch.bfloat16))
        x0, h0 = x.clone(), hid.clone()
        graph.replay()
        check(x0, h0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("odd", ["x", "residual", "sum", "weight", "out"])
def test_each_tensor_anywhere(odd, dtype):
    """One tensor that starts and runs off 16 bytes while the others do not."""
    rng = np.random.default_rng(9)
    T, d = 37, 776

    def place(name, *shape, dt=dtype):
        pitch = shape[-1] + (3 if name == odd else 8)
        t = torch.full((*shape[:-1], pitch), float("nan"), device="cuda", dtype=dt)
        return t[..., 1:1 + shape[-1]] if name == odd else t[..., :shape[-1]]

    x, r, s, w = place("x", T, d), place("residual", T, d), place("sum", T, d), place("weight", d)
    x.copy_(stream(rng, T, d, 0, dtype))
    r.copy_(stream(rng, T, d, 0, dtype))
    w.copy_(stream(rng, 1, d, 0, dtype)[0])
    want = (x.float() + r.float()).to(dtype)
    y, err = reference(want, w, 1e-6)
    for out_dtype in (torch.bfloat16, torch.float32):
        out = place("out", T, d, dt=out_dtype)
        cm.clearmoe_rms_norm(x, out, residual=r, sum_out=s, weight=w)
        assert torch.equal(s, want)
        assert bool(((out.double() - y).abs() <= err + (2.0 ** -8 * y.abs() if out_dtype == torch.bfloat16 else 0)).all())
        for t in (s, out):
            assert int(t._base.isnan().sum()) == t._base.numel() - t.numel()
    a = cm.fp4_matrix(T, d)
    cm.clearmoe_rms_norm(x, a, residual=r, weight=w)
    got = torch.empty(T, d, device="cuda")
    cm.clearmoe_fp4_dequantize(a, got)
    amax = torch.nn.functional.pad(y.abs(), (0, -d % 32)).view(T, -1, 32).amax(2).repeat_interleave(32, 1)[:, :d]
    assert bool(((got.double() - y).abs() <= 1.2 * err + 0.2 * y.abs() + 0.25 * 1.01 * amax / 3).all())


def test_two_streams():
    xs = [torch.randn(4000, 512, device="cuda", dtype=torch.bfloat16) for _ in range(4)]
    outs, want = [torch.empty_like(x) for x in xs], []
    for x in xs:
        want.append(torch.empty_like(x))
        cm.clearmoe_rms_norm(x, want[-1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(10):
        for s, x, o in zip(streams, xs, outs):
            cm.clearmoe_rms_norm(x, o, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("pad", [0, 3])
def test_sums_of_every_bf16_value(pad):
    """Every value of bf16 (subnormal, infinite and NaN ones too) plus others: the sum that is stored is the rounded fp32 sum."""
    bits = torch.arange(65536, dtype=torch.int32, device="cuda")
    g = torch.Generator("cuda").manual_seed(3)
    x = bits.to(torch.int16).view(torch.bfloat16).view(1024, 64)
    for k in range(16):
        order = torch.randperm(65536, device="cuda", generator=g) if k < 12 else (bits + (k - 13) * 129) % 65536  # and its neighbours
        r = bits[order.long()].to(torch.int16).view(torch.bfloat16).view(1024, 64)
        a, b, s, out = (torch.zeros(1024, 64 + pad, device="cuda", dtype=torch.bfloat16)[:, :64] for _ in range(4))
        a.copy_(x)
        b.copy_(r)
        cm.clearmoe_rms_norm(a, out, residual=b, sum_out=s)
        want = (x.float() + r.float()).to(torch.bfloat16)
        assert torch.equal(s.isnan(), want.isnan())
        assert torch.equal(s[~s.isnan()], want[~want.isnan()])


def test_weights_and_bias_just_written():
    """A norm's weights and a product's bias that the kernel right before wrote, new ones each time."""
    x, W = torch.randn(300, 256, device="cuda"), cm.fp4_matrix(384, 256)
    w, b, q = torch.empty(256, device="cuda"), torch.empty(384, device="cuda"), cm.fp4_matrix(300, 256)
    cm.clearmoe_fp4_quantize(torch.randn(384, 256, device="cuda"), W)
    outs = []
    for i in range(60):
        w.fill_(float(2 ** (i % 5)))
        cm.clearmoe_rms_norm(x, q, weight=w)
        b.fill_(float(i % 7))
        outs.append(torch.empty(300, 384, device="cuda"))
        cm.clearmoe_fp4_gemm(q, W, outs[-1], bias=b)
    base = outs[0]
    for i, out in enumerate(outs):  # powers of two scale every sum exactly; the bias is added with one rounding
        assert torch.equal(out, base * 2.0 ** (i % 5) + float(i % 7))
