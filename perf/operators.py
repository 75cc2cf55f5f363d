"""Three operators of converted layers in serving, each in its plain form and through the public entry
points of `paper_2606_28516_gb300.clearmoe`:

  * `few`: a whole folded layer (router, fc1 + GELU, the token's expert) for 1 to 64 tokens, what a step of
    an online service or of token-by-token generation has at a time, with bf16, fp32 or 8-bit weights;
  * `mm`: a product in 8-bit floating point with one power-of-two scale per block of 128: activations
    (1 x 128 blocks) quantised on the way in, weights (128 x 128 blocks) quantised once;
  * `ffn8`: a whole folded layer for a batch with both of its products in that form.

Sizes are those of the repository's own layers (DeiT-T / DeiT-S / ViT-B shapes, 197 tokens per image) and,
for the products, generic widths. The tokens of a layer are a layer-normalised Gaussian mixture, its router
the nearest centroid, its weights N(0, 0.02^2); the products get unit-variance rows of which some channels
are 30 times larger, as the activations of large models have.
"""
import math

import torch

own = False  # False: run() computes the plain forms; True: it calls the framework's operators

TOKENS_PER_IMAGE = 197
STD = 0.02


# ------------------------------------------------------------------------------------- the cases
def listed():
    n = TOKENS_PER_IMAGE
    return [
        # One token through a DeiT-T-sized layer: the smallest request there is; latency alone.
        dict(name="few_tiny_1", op="few", w="bf16", T=1, d=192, E=4, sizes="balanced"),
        # One token through a ViT-B-sized layer with 8-bit weights: a generation step of one user.
        dict(name="few_base_1_fp8", op="few", w="fp8", T=1, d=768, E=8, sizes="balanced"),
        # 13 tokens with everything a deployed block has: fc2's bias, a class token, its LayerNorm.
        dict(name="few_base_13_deployed", op="few", w="bf16", T=13, d=768, E=8, sizes="balanced", bias=True, cls=n,
             ln=True),
        # A DeiT-S layer kept in fp32, 24 tokens of skewed experts.
        dict(name="few_small_24_f32", op="few", w="f32", T=24, d=384, E=6, sizes="zipf"),
        # 64 users' tokens, every expert taken: the largest step of this form.
        dict(name="few_base_64", op="few", w="bf16", T=64, d=768, E=8, sizes="zipf"),
        # Three rows through a wide projection: the weights' bytes are all that counts.
        dict(name="mm_3_wide", op="mm", M=3, N=4096, K=4096, dtype="bf16"),
        # fc1 of a ViT-B layer for one image, with its bias and GELU.
        dict(name="mm_fc1_1img", op="mm", M=n, N=3072, K=768, dtype="bf16", bias=True, gelu=True),
        # Odd sizes throughout, fp32 in and out: rows that start anywhere, blocks cut short on both axes.
        dict(name="mm_odd_f32", op="mm", M=1001, N=777, K=1131, dtype="f32", bias=True),
        # A large batch through a wide projection: the tensor cores' rate.
        dict(name="mm_large", op="mm", M=16384, N=4096, K=4096, dtype="bf16"),
        # One image through a DeiT-S layer in 8 bits: the smallest batch.
        dict(name="ffn8_small_1img", op="ffn8", T=n, d=384, E=4, sizes="balanced"),
        # An odd token count with Zipf-skewed experts, deployed with bias, class tokens and LayerNorm.
        dict(name="ffn8_small_zipf", op="ffn8", T=9973, d=384, E=8, sizes="zipf", bias=True, cls=n, ln=True),
        # ViT-B at 256 images: the headline layer in 8 bits.
        dict(name="ffn8_base_256img", op="ffn8", T=256 * n, d=768, E=8, sizes="balanced"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["few", "few", "mm", "mm", "ffn8"])
    if op == "mm":
        c = dict(op=op, M=_log_int(rng, 1, 16384), N=_log_int(rng, 16, 8192), K=_log_int(rng, 16, 8192),
                 dtype=rng.choice(["bf16", "bf16", "f32"]))
        while c["M"] * c["N"] * c["K"] > 2 ** 38:
            c["M"] = c["M"] // 2 + 1
        if rng.random() < 0.5:  # half of the widths are whole blocks, as most models' are
            c["N"], c["K"] = -(-c["N"] // 128) * 128, -(-c["K"] // 128) * 128
        if rng.random() < 0.5:
            c["bias"] = True
            if rng.random() < 0.5:
                c["gelu"] = True
        return c
    c = dict(op=op, E=rng.randint(1, 12), sizes=rng.choice(["balanced", "zipf"]))
    if op == "few":
        c.update(w=rng.choice(["bf16", "bf16", "fp8", "fp8", "f32"]), T=_log_int(rng, 1, 64))
        c["d"] = rng.choice([192, 200, 384, 512]) if c["w"] == "f32" else rng.choice([192, 320, 384, 768, 1024])
    else:
        c.update(T=_log_int(rng, 49, 50432), d=rng.choice([192, 320, 384, 768, 768, 1024]))
        while c["T"] * c["d"] * c["d"] > 50432 * 768 * 768:
            c["T"] = c["T"] // 2 + 1
    if rng.random() < 0.4:
        c["bias"] = True
    if rng.random() < 0.3:
        c["cls"] = TOKENS_PER_IMAGE
    if rng.random() < 0.3:
        c["ln"] = True
    return c


# ------------------------------------------------------------------------------------- the inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + 29)


def _ln(x):
    x = x - x.mean(1, keepdim=True)
    return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6)


def _cluster_sizes(T, E, law):
    p = [1.0 / k ** 1.2 if law == "zipf" else 1.0 for k in range(1, E + 1)]
    edges = [int(T * sum(p[:k]) / sum(p) + 0.5) for k in range(E + 1)]
    return [b - a for a, b in zip(edges, edges[1:])]


def _blocks(W):
    """A weight matrix in 8 bits: q [N x K'] (float8_e4m3fn, K' = K rounded up to 128, zeros past K) and the
    scale exponents [ceil(N / 128) x 4 ceil(K / 512)] (uint8, biased by 127): W ~ q 2^(scale - 127)."""
    N, K = W.shape
    nb, kb, ks = -(-N // 128), -(-K // 128), 4 * -(-K // 512)
    P = torch.zeros(nb * 128, kb * 128, device=W.device)
    P[:N, :K] = W
    P = P.view(nb, 128, kb, 128)
    e = _exponent(P.abs().amax(dim=(1, 3)))
    q = torch.ldexp(P, -e[:, None, :, None]).to(torch.float8_e4m3fn).view(nb * 128, kb * 128)[:N].contiguous()
    scale = torch.zeros(nb, ks, dtype=torch.uint8, device=W.device)
    scale[:, :kb] = (e + 127).to(torch.uint8)
    return q, scale


def _inputs(case, seed):
    """Every tensor of one case, on the current GPU, from the seed alone."""
    g = _gen(seed)
    if case["op"] == "mm":
        M, N, K = case["M"], case["N"], case["K"]
        tdt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        x = torch.randn(M, K, generator=g, device="cuda")
        x *= torch.where(torch.rand(K, generator=g, device="cuda") < 0.01, 30.0, 1.0)
        W = torch.randn(N, K, generator=g, device="cuda") * STD
        b = (torch.randn(N, generator=g, device="cuda") * STD).to(tdt)
        return dict(x=x.to(tdt), W=_blocks(W), b=b)
    T, d, E, f32 = case["T"], case["d"], case["E"], case.get("w") == "f32"
    tdt, H = torch.float32 if f32 else torch.bfloat16, 4 * d
    cent = torch.randn(E, d, generator=g, device="cuda")
    lab = torch.repeat_interleave(torch.arange(E, device="cuda"),
                                  torch.tensor(_cluster_sizes(T, E, case["sizes"]), device="cuda"))
    lab = lab[torch.randperm(T, generator=g, device="cuda")]
    x = _ln(cent[lab] + 0.5 * torch.randn(T, d, generator=g, device="cuda"))
    if case.get("ln"):  # the un-normalised stream of a block: each token scaled and shifted
        s = 0.5 + 3.5 * torch.rand(T, 1, generator=g, device="cuda")
        x = x * s + torch.randn(T, 1, generator=g, device="cuda")
    m = _ln(cent) * 0.9
    mats = [STD * torch.randn(H, d, generator=g, device="cuda")]
    W2 = STD * torch.randn(d, H, generator=g, device="cuda")
    for e in range(E):  # folded experts: a common part and one of their own
        mats.append(W2 + 0.5 * STD * torch.randn(d, H, generator=g, device="cuda"))
    mats.append(W2)
    fp8 = case["op"] == "ffn8" or case["w"] == "fp8"
    mats = [_blocks(W) if fp8 else W.to(tdt) for W in mats]
    v = lambda n: (STD * torch.randn(n, generator=g, device="cuda")).to(tdt)  # noqa: E731
    return dict(x=x.to(tdt), W1=mats[0], comb=mats[1:1 + E], W2=mats[1 + E], b1=v(H), b2=v(d),
                Wg=m.to(tdt), bg=(-0.5 * (m * m).sum(1)).to(tdt))


class _State:
    """What a program keeps between calls: tensors, weights in the operators' form, buffers, the handle."""

    def __init__(self, case, tensors):
        self.case, self.t, self.h = case, tensors, None

    def __del__(self):
        if self.h is not None:
            from paper_2606_28516_gb300 import clearmoe as cm
            cm.clearmoe_layer_destroy(self.h)
            self.h = None


def prepare(case, seed):
    t = _inputs(case, seed)
    s = _State(case, t)
    if not own:
        return s
    from paper_2606_28516_gb300 import clearmoe as cm
    s.cm = cm
    mat = lambda W, n, k: cm.Fp8Matrix(W[0], W[1], n, k, weight=True) if isinstance(W, tuple) else W  # noqa: E731
    if case["op"] == "mm":
        M, N, K = case["M"], case["N"], case["K"]
        s.W, s.rows = mat(t["W"], N, K), cm.fp8_rows(M, K)
        s.out = torch.empty(M, N, dtype=t["x"].dtype, device="cuda")
        s.bias, s.act = t["b"] if case.get("bias") else None, cm.ACT_GELU if case.get("gelu") else cm.ACT_NONE
        return s
    T, d, E = case["T"], case["d"], case["E"]
    H = 4 * d
    s.h = cm.clearmoe_layer_create(T, d, H, E, 16, cm.F32 if t["x"].dtype == torch.float32 else cm.BF16)
    s.w = cm.ffn_weights(mat(t["W1"], H, d), t["b1"], [mat(W, d, H) for W in t["comb"]], t["Wg"], t["bg"],
                         b2=t["b2"] if case.get("bias") else None,
                         W2=mat(t["W2"], d, H) if case.get("cls") else None, cls_stride=case.get("cls", 0),
                         input_layernorm=bool(case.get("ln")))
    s.out = torch.empty_like(t["x"])
    return s


# ------------------------------------------------------------------------------------ the plain form
def _exponent(amax):
    """The least e with amax <= 448 2^e (448: the largest e4m3 value), held to [-127, 127]."""
    m, k = torch.frexp(amax)
    e = k - 9 + (m > 0.875)
    return torch.where(amax > 0, e, -127).clamp(-127, 127).to(torch.int32)


def _round_rows(x):
    """Rows of fp32 values rounded to 8 bits with a power-of-two scale per 128 columns, as fp32."""
    T, K = x.shape
    P = torch.nn.functional.pad(x, (0, -K % 128)).view(T, -1, 128)
    e = _exponent(P.abs().amax(2, keepdim=True))
    q = torch.ldexp(P, -e).to(torch.float8_e4m3fn).float()
    return torch.ldexp(q, e).view(T, -1)[:, :K]


def _dense(W, N, K):
    """A weight matrix as fp32, whatever it is stored in."""
    if not isinstance(W, tuple):
        return W.float()
    q, s = W
    e = s[:, :q.shape[1] // 128].to(torch.int32) - 127
    e = e.repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)
    return torch.ldexp(q.float(), e)[:, :K]


def _gelu(u):
    return 0.5 * u * (1.0 + torch.erf(u * 0.7071067811865476))


def _plain(s):
    c, t = s.case, s.t
    x = t["x"].float()
    if c["op"] == "mm":
        y = _round_rows(x) @ _dense(t["W"], c["N"], c["K"]).T
        if c.get("bias"):
            y = y + t["b"].float()
        return (_gelu(y) if c.get("gelu") else y).to(t["x"].dtype)
    T, d, E, r8 = c["T"], c["d"], c["E"], c["op"] == "ffn8"
    if c.get("ln"):
        x = _ln(x)
    a = (x @ t["Wg"].float().T + t["bg"].float()).argmax(1)
    if c.get("cls"):
        a = torch.where(torch.arange(T, device="cuda") % c["cls"] == 0, E, a)
    z = _gelu((_round_rows(x) if r8 else x) @ _dense(t["W1"], 4 * d, d).T + t["b1"].float())
    z = _round_rows(z) if r8 else z
    y = torch.empty(T, d, device="cuda")
    for e in range(E + 1 if c.get("cls") else E):
        at = (a == e).nonzero()[:, 0]
        y[at] = z[at] @ _dense(t["comb"][e] if e < E else t["W2"], d, 4 * d).T
    return (y + t["b2"].float() if c.get("bias") else y).to(t["x"].dtype)


def run(s):
    if not own:
        return _plain(s)
    cm, c, t = s.cm, s.case, s.t
    if c["op"] == "mm":
        cm.clearmoe_fp8_quantize_rows(t["x"], s.rows)
        cm.clearmoe_fp8_gemm(s.rows, s.W, s.out, bias=s.bias, act=s.act)
    elif c["op"] == "few":
        cm.clearmoe_ffn_forward_few(s.h, t["x"], s.w, s.out)
    else:
        cm.clearmoe_ffn_forward_fp8(s.h, t["x"], s.w, s.out)
    return s.out


# --------------------------------------------------------------------------------------- the work
def work(case):
    if case["op"] == "mm":
        M, N, K, b = case["M"], case["N"], case["K"], 4 if case["dtype"] == "f32" else 2
        return {"bytes": M * K * b + N * K + -(-N // 128) * -(-K // 128) + M * N * b + (N * b if case.get("bias") else 0),
                "flops": 2 * M * N * K}
    T, d, E = case["T"], case["d"], case["E"]
    H, f32, fp8 = 4 * d, case.get("w") == "f32", case["op"] == "ffn8" or case["w"] == "fp8"
    b, wb = 4 if f32 else 2, 1 if fp8 else 4 if f32 else 2
    n_cls = -(-T // case["cls"]) if case.get("cls") else 0
    # matrices read: fc1 and the experts that have a token (a class token may leave its cluster empty)
    mats = 1 + max(1 if T > n_cls else 0, sum(v > 0 for v in _cluster_sizes(T, E, case["sizes"])) - (n_cls if T < 2 * E else 0))
    mats += 1 if n_cls else 0
    return {"bytes": 2 * T * d * b + mats * d * H * wb + (H + E * (d + 1) + (d if case.get("bias") else 0)) * b,
            "flops": T * (4 * d * H + 2 * d * E)}


# ------------------------------------------------------------------------------------ 64-bit values
def _e4m3(v):
    """float64 values of magnitude at most 448 to the nearest e4m3 value, ties to even: 3 bits after the
    leading one, spaced 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def _q64(x):
    out = torch.empty_like(x)
    for k in range(0, x.shape[1], 128):
        v = x[:, k:k + 128]
        top = v.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -200) / 448.0)).clamp(-127, 127)
        e = e + (top > 448.0 * torch.exp2(e)) - (top <= 448.0 * torch.exp2(e - 1)).to(e.dtype)  # log2's rounding
        e = e.clamp(-127, 127)
        out[:, k:k + 128] = _e4m3(v * torch.exp2(-e)) * torch.exp2(e)
    return out


def _w64(W, N, K):
    if not isinstance(W, tuple):
        return W.double()
    q, s = W
    out = q.double()
    for i in range(0, N, 128):
        for j in range(0, q.shape[1], 128):
            out[i:i + 128, j:j + 128] *= torch.exp2(s[i // 128, j // 128].double() - 127)
    return out[:, :K]


def _gelu64(u):
    return 0.5 * u * torch.erfc(-u / math.sqrt(2.0))


def exact(case, seed):
    t = _inputs(case, seed)
    x = t["x"].double()
    if case["op"] == "mm":
        W, b = _w64(t["W"], case["N"], case["K"]), t["b"].double() if case.get("bias") else 0.0
        y = torch.cat([_q64(v) @ W.T + b for v in x.split(4096)])
        return _gelu64(y) if case.get("gelu") else y
    d, E, r8 = case["d"], case["E"], case["op"] == "ffn8"
    W1, Wg = _w64(t["W1"], 4 * d, d), t["Wg"].double()
    out = []
    for at in torch.arange(case["T"], device="cuda").split(8192):
        v = x[at]
        if case.get("ln"):
            v = v - v.mean(1, keepdim=True)
            v = v / (v.square().mean(1, keepdim=True) + 1e-6).sqrt()
        a = (v @ Wg.T + t["bg"].double()).argmax(1)
        z = _gelu64((_q64(v) if r8 else v) @ W1.T + t["b1"].double())
        z = _q64(z) if r8 else z
        y = torch.zeros(len(at), d, dtype=torch.float64, device="cuda")
        for e in range(E):
            y += torch.where((a == e)[:, None], z @ _w64(t["comb"][e], d, 4 * d).T, 0.0)
        if case.get("cls"):
            y = torch.where((at % case["cls"] == 0)[:, None], z @ _w64(t["W2"], d, 4 * d).T, y)
        out.append(y + t["b2"].double() if case.get("bias") else y)
    return torch.cat(out)
