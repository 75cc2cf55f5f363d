"""The whole folded layer for a few tokens, and for a batch in 8-bit blocks, against float64.

Few tokens: outputs within max |err| / RMS <= 2e-2 in bf16 layers (the bf16 layers' tolerance: z and the output
are each rounded once to bf16) against a float64 layer with z rounded to bf16, relative L2 <= 1e-5 in fp32 layers
(three TF32 products per term, 2^-21 relative each). The 8-bit layer: against float64 with both operands
quantised as defined; an element of z that fp32 arithmetic puts on the other side of a rounding border moves by
one e4m3 step, 2^-3 of it at most, which 1e-3 of the elements doing so at once turn into less than 2^-8 RMS; the
same 2e-2."""
import ctypes

import numpy as np
import pytest
import torch

import fp8_ref as R
from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu


class Layer:
    """Weights of a folded layer in `kind` (bf16, f32 or fp8) and float64 copies of what they stand for."""

    def __init__(self, kind, d, H, E, seed=0, b2=False, cls=0, ln=False, T=64):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.kind, self.d, self.H, self.E, self.cls, self.ln = kind, d, H, E, cls, ln
        self.tdt = torch.float32 if kind == "f32" else torch.bfloat16
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        mats = [0.05 * rnd(H, d)] + [0.05 * rnd(d, H) for _ in range(E + 1)]
        self.m64, self.m = [], []
        for W in mats:
            if kind == "fp8":
                q = cm.fp8_weight(*W.shape)
                cm.clearmoe_fp8_quantize_weight(W, q)
                v = torch.empty(*W.shape, device="cuda")
                cm.clearmoe_fp8_dequantize(q, v)
                self.m.append(q)
                self.m64.append(v.double())
            else:
                self.m.append(W.to(self.tdt))
                self.m64.append(self.m[-1].double())
        self.b1, self.b2 = rnd(H).to(self.tdt), rnd(d).to(self.tdt) if b2 else None
        self.cent = rnd(E, d)
        self.Wg, self.bg = self.cent.to(self.tdt), (-0.5 * (self.cent ** 2).sum(1)).to(self.tdt)
        self.g = g
        self.w = cm.ffn_weights(self.m[0], self.b1, self.m[1:E + 1], self.Wg, self.bg, b2=self.b2,
                                W2=self.m[E + 1] if cls else None, cls_stride=cls, input_layernorm=ln)
        self.h = cm.clearmoe_layer_create(T, d, H, E, 4 if kind == "f32" else 16, cm.F32 if kind == "f32" else cm.BF16)

    def tokens(self, T, experts=None):
        e = torch.randint(0, self.E, (T,), generator=self.g, device="cuda") if experts is None else \
            torch.tensor(experts, device="cuda")
        x = self.cent[e] + 0.3 * torch.randn(T, self.d, generator=self.g, device="cuda")
        if self.ln:
            x = 3.0 * x + 2.0
        return x.to(self.tdt)

    def close(self):
        assert cm.clearmoe_layer_status(self.h) == 0
        cm.clearmoe_layer_destroy(self.h)

    def reference(self, x, r8=False):
        v = x.double()
        if self.ln:
            v = v - v.mean(1, keepdim=True)
            v = v / (v.square().mean(1, keepdim=True) + 1e-6).sqrt()
        a = (v @ self.Wg.double().T + self.bg.double()).argmax(1)
        if self.cls:
            a = torch.where(torch.arange(len(x), device="cuda") % self.cls == 0, self.E, a)
        q = lambda t: torch.from_numpy(R.quantize(t.cpu().numpy(), 1)[2]).cuda()  # noqa: E731
        u = (q(v) if r8 else v) @ self.m64[0].T + self.b1.double()
        z = 0.5 * u * torch.erfc(-u / np.sqrt(2.0))
        z = q(z) if r8 else z.to(self.tdt).double()
        y = torch.stack([self.m64[1 + e] @ z[t] for t, e in enumerate(a.tolist())])
        return a, y + self.b2.double() if self.b2 is not None else y

    def check(self, out, x, r8=False):
        a, y = self.reference(x, r8)
        err = out.double() - y
        if self.kind == "f32":
            assert (err.norm() / y.norm()).item() <= 1e-5
        else:
            assert (err.abs().max() / y.square().mean().sqrt()).item() <= 2e-2
        T, G = len(x), self.E + (1 if self.cls else 0)
        i32 = dict(dtype=torch.int32, device="cuda")
        idx, perm = torch.empty(T, **i32), torch.empty(T, **i32)
        counts, offsets = torch.empty(G, **i32), torch.empty(G + 1, **i32)
        cm.clearmoe_get_routing(self.h, idx=idx, counts=counts, offsets=offsets, perm=perm)
        assert torch.equal(idx.long(), a)
        assert torch.equal(counts.long(), torch.bincount(a, minlength=G))
        assert torch.equal(offsets.long(), torch.cat([a.new_zeros(1), torch.bincount(a, minlength=G).cumsum(0)]))
        assert torch.equal(perm.long(), torch.sort(a, stable=True).indices)


DIMS = {"bf16": [(64, 64), (192, 768), (320, 1280), (768, 3072), (1024, 128)],
        "fp8": [(64, 64), (192, 768), (320, 1280), (768, 3072), (1024, 192)],
        "f32": [(4, 4), (200, 800), (384, 1536), (36, 132), (512, 20)]}


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("shape", range(5))
@pytest.mark.parametrize("T", [1, 2, 9, 17, 33, 64])
def test_few(kind, shape, T):
    d, H = DIMS[kind][shape]
    L = Layer(kind, d, H, E=1 + (shape + T) % 8, seed=T + shape, b2=T % 2 == 0)
    x = L.tokens(T)
    out = torch.full((T, d), float("nan"), device="cuda", dtype=L.tdt)
    cm.clearmoe_ffn_forward_few(L.h, x, L.w, out)
    L.check(out, x)
    L.close()


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("cls,ln,T", [(1, False, 5), (7, False, 20), (0, True, 3), (7, True, 40), (64, True, 64), (2, True, 1)])
def test_few_options(kind, cls, ln, T):
    L = Layer(kind, 192, 768, E=5, seed=T + cls, b2=True, cls=cls, ln=ln)
    x = L.tokens(T)
    out = torch.full((T, 192), float("nan"), device="cuda", dtype=L.tdt)
    cm.clearmoe_ffn_forward_few(L.h, x, L.w, out)
    L.check(out, x)
    L.close()


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_few_skewed_and_repeated(kind):
    """All tokens on one expert, every other expert empty; the same call again and on another stream gives the
    same bits, and a larger call between does not change them."""
    L = Layer(kind, 192, 768, E=15, seed=3, cls=50)
    x = L.tokens(64, [11] * 64)
    out = torch.empty(64, 192, device="cuda", dtype=L.tdt)
    cm.clearmoe_ffn_forward_few(L.h, x, L.w, out)
    L.check(out, x)
    first = out.clone()
    x2, out2 = L.tokens(7), torch.empty(7, 192, device="cuda", dtype=L.tdt)
    cm.clearmoe_ffn_forward_few(L.h, x2, L.w, out2)
    small = out2.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(5):
            cm.clearmoe_ffn_forward_few(L.h, x2, L.w, out2)
            cm.clearmoe_ffn_forward_few(L.h, x, L.w, out)
    s.synchronize()
    assert torch.equal(out, first) and torch.equal(out2, small)
    L.close()


def test_few_follows_the_batch_forward():
    """The same folded weights through clearmoe_ffn_forward_folded: both within the bf16 tolerance of each other."""
    L = Layer("bf16", 384, 1536, E=4, seed=2)
    x = L.tokens(64)
    a, b = (torch.empty(64, 384, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    cm.clearmoe_ffn_forward_few(L.h, x, L.w, a)
    cm.clearmoe_ffn_forward_folded(L.h, x, L.m[0], L.b1, L.m[1:5], L.Wg, L.bg, b)
    d = (a.double() - b.double()).abs().max() / b.double().square().mean().sqrt()
    assert d.item() <= 2e-2
    L.close()


def test_ties_go_to_the_lowest_expert_and_nan_stays_in_its_token():
    L = Layer("bf16", 64, 256, E=4, seed=1)
    L.Wg[2] = L.Wg[1]
    L.bg[2] = L.bg[1]
    x = L.tokens(10, [1] * 10)
    x[4, 3] = float("nan")
    out = torch.zeros(10, 64, device="cuda", dtype=torch.bfloat16)
    cm.clearmoe_ffn_forward_few(L.h, x, L.w, out)
    idx = torch.empty(10, dtype=torch.int32, device="cuda")
    cm.clearmoe_get_routing(L.h, idx=idx)
    idx = idx.tolist()
    assert [v for t, v in enumerate(idx) if t != 4] == [1] * 9 and 0 <= idx[4] < 4
    assert bool(out[4].isnan().all()) and bool(out[[t for t in range(10) if t != 4]].isfinite().all())
    L.close()


@pytest.mark.parametrize("d,H,T,E,kw", [
    (64, 64, 1, 1, {}), (192, 768, 130, 4, {}), (320, 1280, 77, 3, dict(b2=True)), (384, 1536, 500, 8, dict(cls=197, b2=True)),
    (768, 3072, 394, 8, dict(ln=True)), (192, 768, 1000, 12, dict(ln=True, cls=197, b2=True)), (1024, 192, 129, 2, {})])
def test_ffn_fp8(d, H, T, E, kw):
    L = Layer("fp8", d, H, E, seed=T, T=T, **kw)
    x = L.tokens(T)
    out = torch.full((T, d), float("nan"), device="cuda", dtype=torch.bfloat16)
    cm.clearmoe_ffn_forward_fp8(L.h, x, L.w, out)
    L.check(out, x, r8=True)
    again = torch.empty_like(out)
    cm.clearmoe_ffn_forward_fp8(L.h, x, L.w, again)
    assert torch.equal(out, again)
    L.close()


def test_empty_experts_fp8():
    L = Layer("fp8", 192, 768, E=6, seed=8, T=300)
    x = L.tokens(300, [4] * 300)
    out = torch.full((300, 192), float("nan"), device="cuda", dtype=torch.bfloat16)
    cm.clearmoe_ffn_forward_fp8(L.h, x, L.w, out)
    L.check(out, x, r8=True)
    L.close()


def test_refusals():
    lib = cm.lib()
    L = Layer("bf16", 64, 128, E=2, T=100)
    x, out = L.tokens(100), torch.zeros(100, 64, device="cuda", dtype=torch.bfloat16)
    p, o = x.data_ptr(), out.data_ptr()
    few, fp8 = lib.clearmoe_ffn_forward_few, lib.clearmoe_ffn_forward_fp8
    assert few(L.h, p, 65, L.w.ref, o, None) == cm.EUNSUPPORTED
    assert fp8(L.h, p, 5, L.w.ref, o, None) == cm.EUNSUPPORTED
    for f in (few, fp8):
        assert f(None, p, 5, L.w.ref, o, None) == cm.EINVAL
        assert f(L.h, None, 5, L.w.ref, o, None) == cm.EINVAL
        assert f(L.h, p, 0, L.w.ref, o, None) == cm.EINVAL
        assert f(L.h, p, 101, L.w.ref, o, None) == cm.EINVAL
        assert f(L.h, p, 5, None, o, None) == cm.EINVAL
        assert f(L.h, p, 5, L.w.ref, None, None) == cm.EINVAL
        assert f(L.h, p + 2, 5, L.w.ref, o, None) == cm.EINVAL

    def changed(**kw):
        c = cm.clearmoe_ffn_weights.from_buffer_copy(L.w.c)
        for k, v in kw.items():
            at = c
            *path, last = k.split("__")
            for q in path:
                at = getattr(at, q)
            setattr(at, last, v)
        return ctypes.byref(c)

    assert few(L.h, p, 5, changed(dtype=9), o, None) == cm.EINVAL
    assert few(L.h, p, 5, changed(dtype=cm.F32), o, None) == cm.EUNSUPPORTED
    assert few(L.h, p, 5, changed(dtype=cm.FP8), o, None) == cm.EINVAL  # no scales
    for kw in (dict(E=0), dict(E=3), dict(b1=None), dict(W1__q=None), dict(W1__rows=127), dict(W1__cols=65), dict(cls_stride=-1),
               dict(cls_stride=3), dict(router__W=None), dict(W1__q=L.w.c.W1.q + 2), dict(b2=L.w.c.b1 + 2)):
        assert few(L.h, p, 5, changed(**kw), o, None) == cm.EINVAL, kw
    torch.cuda.synchronize()
    assert not out.any()
    L.close()
    F = Layer("f32", 64, 128, E=2)
    with pytest.raises(cm.ClearMoEError):
        cm.clearmoe_ffn_forward_fp8(F.h, F.tokens(4), F.w, torch.zeros(4, 64, device="cuda"))
    Q = Layer("fp8", 64, 128, E=2)
    assert few(F.h, p, 4, Q.w.ref, o, None) == cm.EUNSUPPORTED  # 8-bit weights on an fp32 handle
    with pytest.raises(ValueError):
        cm.ffn_weights(Q.m[0], Q.b1, F.m[1:3], Q.Wg, Q.bg)
    F.close()
    Q.close()


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("T,E", [(1, 1), (1, 4), (4, 2), (5, 1), (9, 3), (16, 1), (16, 8)])
def test_up_to_16_tokens_keep_z(kind, T, E):
    """Two bf16 parts of z: against float64 with z as it is, each output within its own rounding (2^-8 of it at the most) and what
    fp32 sums and 2^-17 of each z can do; z rounded to bf16 alone moves most of them further. The same from a handle for
    exactly these tokens."""
    d, H = 192, 768
    outs = []
    for T_max in (64, T):
        L = Layer(kind, d, H, E, seed=T + E, b2=True, T=T_max)
        x = L.tokens(T)
        out = torch.full((T, d), float("nan"), device="cuda", dtype=L.tdt)
        cm.clearmoe_ffn_forward_few(L.h, x, L.w, out)
        outs.append(out)
        a, _ = L.reference(x)
        v, W1 = x.double(), L.m64[0]
        u = v @ W1.T + L.b1.double()
        z = 0.5 * u * torch.erfc(-u / np.sqrt(2.0))
        du = (d / 16 + 16) * 2.0 ** -23 * (v.abs() @ W1.abs().T + L.b1.double().abs())
        dz = 1.13 * du + 4e-7 + 4e-7 * z.abs() + 2.0 ** -17 * z.abs()
        y = torch.stack([L.m64[1 + e] @ z[t] for t, e in enumerate(a.tolist())]) + L.b2.double()
        mag = torch.stack([L.m64[1 + e].abs() @ (dz + (H / 16 + 16) * 2.0 ** -23 * z.abs())[t] for t, e in enumerate(a.tolist())])
        assert bool(((out.double() - y).abs() <= 2.0 ** -8 * y.abs() + 1.01 * mag + 1e-6).all())
        rounded = torch.stack([L.m64[1 + e] @ z.to(torch.bfloat16).double()[t] for t, e in enumerate(a.tolist())]) + L.b2.double()
        assert bool(((rounded - y).abs() > mag).double().mean() > 0.5)
        L.close()
    assert torch.equal(*outs)
