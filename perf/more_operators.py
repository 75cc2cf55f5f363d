"""Operators that make the activations and weights of a serving layer smaller, each in its plain form and through the
public entry points of `paper_2606_28516_gb300.clearmoe`:

  * `mm4`: a product in 4-bit floating point with one power-of-two scale per 32 columns of a row: activations
    quantised on the way in, weights quantised once;
  * `moe4`: the same grouped by expert: tokens quantised in expert order, each expert's rows times its matrix,
    the results back in token order;
  * `mlp4`: two such products in a row, the hidden state (bias, GELU) quantised by the first one;
  * `norm`: a residual's addition and the root-mean-square norm of the sum, both returned;
  * `norm8`, `norm4`: the same with the norm's output in 8-bit or 4-bit blocks, and the product that reads it, in
    bf16 whatever the stream's type.

Sizes are those of the repository's own layers (d = 384, 768 and 1,024, 197 tokens per image) and generic widths. Rows
have unit variance with some channels ten times larger, as the activations of large models have; weights are
N(0, 0.02^2), a norm's around one.
"""
import math

import torch

own = False  # False: run() computes the plain forms; True: it calls the framework's operators

TOKENS_PER_IMAGE = 197
STD = 0.02
EPS = 1e-5


# ------------------------------------------------------------------------------------- the cases
def listed():
    n = TOKENS_PER_IMAGE
    return [
        # One token's norm at a ViT-B width: the smallest call there is; latency alone.
        dict(name="norm_1", op="norm", T=1, d=768, dtype="bf16"),
        # Odd sizes in fp32, rows that start anywhere: a slice of a wider buffer.
        dict(name="norm_odd_f32", op="norm", T=1001, d=1131, dtype="f32", pad=6),
        # The stream of a large batch: memory's rate.
        dict(name="norm_large", op="norm", T=16384, d=4096, dtype="bf16"),
        # The glue before a narrow projection in 8 bits, of a batch.
        dict(name="norm8_narrow", op="norm8", T=4096, d=4096, N=1024, dtype="bf16"),
        # One generation step of four users before a wide projection in 4 bits.
        dict(name="norm4_step", op="norm4", T=4, d=4096, N=4096, dtype="bf16"),
        # Ten images before a ViT-B-sized projection in 4 bits.
        dict(name="norm4_10img", op="norm4", T=10 * n, d=768, N=2304, dtype="bf16"),
        # Three rows through a very wide projection: the weights' bytes are all that counts.
        dict(name="mm4_3_wide", op="mm4", M=3, N=8192, K=8192, dtype="bf16"),
        # fc1 of a DeiT-S layer for one image, with its bias and GELU.
        dict(name="mm4_fc1_1img", op="mm4", M=n, N=1536, K=384, dtype="bf16", bias=True, gelu=True),
        # Odd sizes throughout, fp32 in and out: rows that start anywhere, blocks cut short.
        dict(name="mm4_odd_f32", op="mm4", M=1001, N=777, K=1131, dtype="f32", bias=True),
        # A large batch through a wide projection: the tensor cores' rate.
        dict(name="mm4_large", op="mm4", M=16384, N=4096, K=4096, dtype="bf16"),
        # The second products of eight unevenly used experts, an odd number of tokens.
        dict(name="moe4_zipf", op="moe4", T=9973, N=1024, K=4096, E=8, sizes="zipf", dtype="bf16"),
        # A whole FFN for a batch, the hidden state never wider than 4 bits.
        dict(name="mlp4_batch", op="mlp4", T=8192, d=1024, H=4096, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width, half of the time a multiple of 128, as most models' are."""
    w = _log_int(rng, lo, hi)
    return -(-w // 128) * 128 if rng.random() < 0.5 else w


def draw(rng):
    op = rng.choice(["mm4", "mm4", "mm4", "moe4", "mlp4", "norm", "norm", "norm8", "norm4"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "mm4":
        c = dict(op=op, M=_log_int(rng, 1, 16384), N=_width(rng, 16, 8192), K=_width(rng, 16, 8192), dtype=dtype)
        while c["M"] * c["N"] * c["K"] > 2 ** 38:
            c["M"] = c["M"] // 2 + 1
        if rng.random() < 0.5:
            c["bias"] = True
            if rng.random() < 0.5:
                c["gelu"] = True
    elif op == "moe4":
        c = dict(op=op, T=_log_int(rng, 1, 9973), N=_width(rng, 64, 1024), K=_width(rng, 64, 4096), E=rng.randint(1, 12),
                 sizes=rng.choice(["balanced", "zipf"]), dtype="bf16")
    elif op == "mlp4":
        c = dict(op=op, T=_log_int(rng, 1, 8192), d=_width(rng, 64, 1024), dtype="bf16")
        c["H"] = 4 * c["d"]
    else:
        c = dict(op=op, T=_log_int(rng, 1, 16384), d=_width(rng, 32, 8192), dtype=dtype)
        while c["T"] * c["d"] > 2 ** 26:
            c["T"] = c["T"] // 2 + 1
        if op != "norm":
            c["N"] = _width(rng, 64, 4096)
            while c["T"] * c["d"] * c["N"] > 2 ** 36:
                c["T"] = c["T"] // 2 + 1
        if rng.random() < 0.3:
            c["pad"] = rng.randint(1, 16)
    return c


# ------------------------------------------------------------------------------------- the inputs
def _cluster_sizes(T, E, law):
    p = [1.0 / k ** 1.2 if law == "zipf" else 1.0 for k in range(1, E + 1)]
    edges = [int(T * sum(p[:k]) / sum(p) + 0.5) for k in range(E + 1)]
    return [b - a for a, b in zip(edges, edges[1:])]


def _inputs(case, seed):
    """Every tensor of one case, on the current GPU, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + 31)
    tdt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def rows(T, d, scale=1.0):
        x = randn(T, d + case.get("pad", 0)) * scale
        x *= torch.where(torch.rand(x.shape[1], generator=g, device="cuda") < 0.01, 10.0, 1.0)
        return x.to(tdt)[:, :d]

    def weight(N, K):
        return (STD * randn(N, K)).to(tdt)

    op, t = case["op"], {}
    if op == "mm4":
        t.update(x=rows(case["M"], case["K"]), W=[weight(case["N"], case["K"])], b=(STD * randn(case["N"])).to(tdt))
    elif op == "moe4":
        T, E = case["T"], case["E"]
        sizes = _cluster_sizes(T, E, case["sizes"])
        t.update(x=rows(T, case["K"]), W=[weight(case["N"], case["K"]) for _ in range(E)],
                 perm=torch.randperm(T, generator=g, device="cuda").to(torch.int32),
                 offsets=torch.tensor([sum(sizes[:e]) for e in range(E + 1)], dtype=torch.int32, device="cuda"))
    elif op == "mlp4":
        d, H = case["d"], case["H"]
        t.update(x=rows(case["T"], d), W=[weight(H, d), weight(d, H)], b=(STD * randn(H)).to(tdt), b2=(STD * randn(d)).to(tdt))
    else:
        T, d = case["T"], case["d"]
        t.update(x=rows(T, d), r=rows(T, d, 2.0), w=(1.0 + 0.1 * randn(d)).to(tdt))
        if op != "norm":
            t["W"] = [weight(case["N"], d)]
    return t


class _State:
    """What a program keeps between calls: tensors, weights in blocks, buffers."""

    def __init__(self, case, tensors):
        self.case, self.t = case, tensors


def prepare(case, seed):
    s = _State(case, _inputs(case, seed))
    t, op = s.t, case["op"]
    if not own:
        if op == "norm8":
            s.W = [_pack8(W) for W in t.pop("W")]
        elif op != "norm":
            s.W = [_pack4(W) for W in t.pop("W")]
        return s
    from paper_2606_28516_gb300 import clearmoe as cm
    s.cm, x = cm, t["x"]
    T, K = x.shape
    s.W = []
    for W in t.pop("W", []):  # weights are quantised once
        if op == "norm8":
            s.W.append(cm.fp8_weight(*W.shape))
            cm.clearmoe_fp8_quantize_weight(W, s.W[-1])
        else:
            s.W.append(cm.fp4_matrix(*W.shape))
            cm.clearmoe_fp4_quantize(W, s.W[-1])
    if op.startswith("norm"):
        s.sum = torch.empty(T, K, dtype=x.dtype, device="cuda")
    if op == "norm":
        s.out = torch.empty(T, K, dtype=x.dtype, device="cuda")
        return s
    s.rows = cm.fp8_rows(T, K) if op == "norm8" else cm.fp4_matrix(T, K)
    if op == "mlp4":
        s.z = cm.fp4_matrix(T, case["H"])
    s.out = torch.empty(T, s.W[-1].rows, dtype=torch.bfloat16 if "norm" in op else x.dtype, device="cuda")
    return s


# ------------------------------------------------------------------------------------ the plain form
def _blocks(x, n):
    """[rows x cols] as fp32 [rows x blocks x n], zeros past the columns."""
    return torch.nn.functional.pad(x.float(), (0, -x.shape[1] % n)).view(x.shape[0], -1, n)


def _exponent(amax, top, shift):
    """The least e with amax <= m 2^(shift + e), m = 2 `top` in [1, 2), held to [-127, 127]."""
    m, k = torch.frexp(amax)
    e = k - 1 - shift + (m > top)
    return torch.where(amax > 0, e, -127).clamp(-127, 127).to(torch.int32)


def _round4(P):
    """Blocks of 32 as the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, and their exponents: 6 = 1.5 2^2."""
    e = _exponent(P.abs().amax(-1, keepdim=True), 0.75, 2)
    u = torch.ldexp(P, -e)
    step = torch.where(u.abs() < 2, 0.5, torch.where(u.abs() < 4, 1.0, 2.0))
    return torch.round(u / step) * step, e


def _rows4(x):
    """Rows rounded to 4-bit blocks, as fp32."""
    u, e = _round4(_blocks(x, 32))
    return torch.ldexp(u, e).view(x.shape[0], -1)[:, :x.shape[1]]


def _rows8(x):
    """Rows rounded to 8 bits with a power-of-two scale per 128 columns, as fp32: 448 = 1.75 2^8."""
    P = _blocks(x, 128)
    e = _exponent(P.abs().amax(-1, keepdim=True), 0.875, 8)
    q = torch.ldexp(P, -e).to(torch.float8_e4m3fn).float()
    return torch.ldexp(q, e).view(x.shape[0], -1)[:, :x.shape[1]]


def _pack4(W):
    """A weight matrix in 4-bit blocks: two codes a byte, the first in the low half, and a biased exponent per block."""
    u, e = _round4(_blocks(W, 32))
    a = u.abs()
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (u < 0).to(torch.uint8) << 3
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8), W.shape[1]


def _unpack4(W):
    q, s, K = W
    code = torch.stack([q & 15, q >> 4], -1).view(q.shape[0], q.shape[1], 32)
    a = (code & 7).float()
    a = torch.where(a < 4, a / 2, torch.where(a < 6, a - 2, 2 * a - 8))
    u = torch.where(code > 7, -a, a)
    return torch.ldexp(u, s.to(torch.int32) - 127).view(q.shape[0], -1)[:, :K]


def _pack8(W):
    """A weight matrix in 8 bits with an exponent per 128 x 128 block."""
    N, K = W.shape
    P = torch.nn.functional.pad(W.float(), (0, -K % 128, 0, -N % 128))
    P = P.view(P.shape[0] // 128, 128, -1, 128)
    e = _exponent(P.abs().amax((1, 3), keepdim=True), 0.875, 8)
    return torch.ldexp(P, -e).to(torch.float8_e4m3fn), e, N, K


def _unpack8(W):
    q, e, N, K = W
    P = torch.ldexp(q.float(), e)
    return P.reshape(P.shape[0] * 128, -1)[:N, :K]


def _gelu(u):
    return 0.5 * u * (1.0 + torch.erf(u * 0.7071067811865476))


def _plain(s):
    c, t, op = s.case, s.t, s.case["op"]
    x = t["x"]
    dt = x.dtype
    if op == "mm4":
        y = _rows4(x) @ _unpack4(s.W[0]).T
        if c.get("bias"):
            y = y + t["b"].float()
        return (_gelu(y) if c.get("gelu") else y).to(dt)
    if op == "moe4":
        q = _rows4(x)
        y = torch.empty(c["T"], c["N"], device="cuda")
        for W, at in zip(s.W, t["perm"].long().split(_cluster_sizes(c["T"], c["E"], c["sizes"]))):
            y[at] = q[at] @ _unpack4(W).T
        return y.to(dt)
    if op == "mlp4":
        z = _gelu(_rows4(x) @ _unpack4(s.W[0]).T + t["b"].float())
        return (_rows4(z) @ _unpack4(s.W[1]).T + t["b2"].float()).to(dt)
    total = (x.float() + t["r"].float()).to(dt)
    v = total.float()
    y = v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS) * t["w"].float()
    if op == "norm":
        return [total, y.to(dt)]
    y = _rows8(y) @ _unpack8(s.W[0]).T if op == "norm8" else _rows4(y) @ _unpack4(s.W[0]).T
    return [total, y.bfloat16()]


def run(s):
    if not own:
        return _plain(s)
    cm, c, t, op = s.cm, s.case, s.t, s.case["op"]
    if op == "mm4":
        cm.clearmoe_fp4_quantize(t["x"], s.rows)
        cm.clearmoe_fp4_gemm(s.rows, s.W[0], s.out, bias=t["b"] if c.get("bias") else None,
                             act=cm.ACT_GELU if c.get("gelu") else cm.ACT_NONE)
        return s.out
    if op == "moe4":
        cm.clearmoe_fp4_quantize(t["x"], s.rows, gather=t["perm"])
        cm.clearmoe_fp4_grouped_gemm(s.rows, s.W, t["offsets"], s.out, perm=t["perm"])
        return s.out
    if op == "mlp4":
        cm.clearmoe_fp4_quantize(t["x"], s.rows)
        cm.clearmoe_fp4_gemm(s.rows, s.W[0], s.z, bias=t["b"], act=cm.ACT_GELU)
        cm.clearmoe_fp4_gemm(s.z, s.W[1], s.out, bias=t["b2"])
        return s.out
    to = s.out if op == "norm" else s.rows
    cm.clearmoe_rms_norm(t["x"], to, residual=t["r"], sum_out=s.sum, weight=t["w"], eps=EPS)
    if op == "norm8":
        cm.clearmoe_fp8_gemm(s.rows, s.W[0], s.out)
    elif op == "norm4":
        cm.clearmoe_fp4_gemm(s.rows, s.W[0], s.out)
    return [s.sum, s.out]


# --------------------------------------------------------------------------------------- the work
def work(case):
    b = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    w4 = lambda N, K: N * -(-K // 32) * 17  # noqa: E731  16 bytes of values and a scale per block
    if op == "mm4":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K * b + w4(N, K) + M * N * b + (N * b if case.get("bias") else 0), "flops": 2 * M * N * K}
    if op == "moe4":
        T, N, K = case["T"], case["N"], case["K"]
        used = sum(v > 0 for v in _cluster_sizes(T, case["E"], case["sizes"]))
        return {"bytes": T * K * b + used * w4(N, K) + T * N * b + T * 4 + (case["E"] + 1) * 4, "flops": 2 * T * N * K}
    if op == "mlp4":
        T, d, H = case["T"], case["d"], case["H"]
        return {"bytes": 2 * T * d * b + w4(H, d) + w4(d, H) + (H + d) * b, "flops": 4 * T * d * H}
    T, d = case["T"], case["d"]
    if op == "norm":
        return {"bytes": 4 * T * d * b + d * b, "flops": 5 * T * d}
    N = case["N"]
    w = w4(N, d) if op == "norm4" else N * d + -(-N // 128) * -(-d // 128)
    return {"bytes": 3 * T * d * b + d * b + w + T * N * 2, "flops": 5 * T * d + 2 * T * N * d}


# ------------------------------------------------------------------------------------ 64-bit values
def _block_exponent64(top, most):
    """The least whole e with top <= most 2^e, held to [-127, 127]."""
    e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -200) / most)).clamp(-127, 127)
    e = e + (top > most * torch.exp2(e)) - (top <= most * torch.exp2(e - 1)).to(e.dtype)  # log2's own rounding
    return e.clamp(-127, 127)


def _q64(x, bits):
    """float64 rows to the nearest values of 4-bit (2 significant bits from 1 on, multiples of 0.5 below) or 8-bit
    blocks (4 significant bits from 2^-6 on, multiples of 2^-9 below), ties to even."""
    n, most, least, digits = (32, 6.0, 1.0, 1) if bits == 4 else (128, 448.0, 2.0 ** -6, 3)
    out = torch.empty_like(x)
    for k in range(0, x.shape[1], n):
        v = x[:, k:k + n]
        e = _block_exponent64(v.abs().amax(1, keepdim=True), most)
        u = v * torch.exp2(-e)
        step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=least))) - digits)
        out[:, k:k + n] = torch.round(u / step) * step * torch.exp2(e)
    return out


def _w8_64(W):
    out = W.clone()
    for i in range(0, W.shape[0], 128):
        for j in range(0, W.shape[1], 128):
            v = W[i:i + 128, j:j + 128]
            e = _block_exponent64(v.abs().amax().view(1), 448.0)
            u = v * torch.exp2(-e)
            step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
            out[i:i + 128, j:j + 128] = torch.round(u / step) * step * torch.exp2(e)
    return out


def _gelu64(u):
    return 0.5 * u * torch.erfc(-u / math.sqrt(2.0))


def exact(case, seed):
    t, op = _inputs(case, seed), case["op"]
    x = t["x"].double()
    if op == "mm4":
        W, b = _q64(t["W"][0].double(), 4), t["b"].double() if case.get("bias") else 0.0
        y = torch.cat([_q64(v, 4) @ W.T + b for v in x.split(4096)])
        return _gelu64(y) if case.get("gelu") else y
    if op == "moe4":
        q, at = _q64(x, 4), torch.empty(case["T"], dtype=torch.long, device="cuda")
        e_of = torch.bucketize(torch.arange(case["T"], device="cuda"), t["offsets"][1:].long(), right=True)
        at[t["perm"].long()] = e_of
        y = torch.zeros(case["T"], case["N"], dtype=torch.float64, device="cuda")
        for e in range(case["E"]):
            y += torch.where((at == e)[:, None], q @ _q64(t["W"][e].double(), 4).T, 0.0)
        return y
    if op == "mlp4":
        W1, W2 = _q64(t["W"][0].double(), 4), _q64(t["W"][1].double(), 4)
        return torch.cat([_q64(_gelu64(_q64(v, 4) @ W1.T + t["b"].double()), 4) @ W2.T + t["b2"].double() for v in x.split(4096)])
    total = x + t["r"].double()
    v = total.to(t["x"].dtype).double()  # the norm is of the stream as it is stored
    y = v * (v.square().mean(1, keepdim=True) + EPS).rsqrt() * t["w"].double()
    if op == "norm":
        return [total, y]
    W = t["W"][0].double()
    return [total, torch.cat([_q64(p, 4 if op == "norm4" else 8) for p in y.split(4096)]) @ (_q64(W, 4) if op == "norm4" else _w8_64(W)).T]
