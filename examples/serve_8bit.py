"""A converted layer served in 8 bits: its folded weights quantised once, a batch of images through the layer in 8-bit
blocks, then steps of a few tokens through the same weights, and a projection of the outputs as an 8-bit product.

    python examples/serve_8bit.py [--images 64] [--steps 8]

Synthetic weights of a ViT-B-sized layer (d = 768, H = 3,072, 8 experts). Prints how far each path is from the bf16
layer with the unquantised weights, and the time a call takes."""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import torch  # noqa: E402

from paper_2606_28516_gb300 import clearmoe as cm  # noqa: E402

TOKENS_PER_IMAGE = 197


def quantize(W):
    q = cm.fp8_weight(*W.shape)
    cm.clearmoe_fp8_quantize_weight(W, q)
    return q


def relative(a, b):
    return ((a.double() - b.double()).norm() / b.double().norm()).item()


def timed(call, n=20):
    call()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(n):
        call()
    torch.cuda.synchronize()
    return (time.perf_counter() - t) / n * 1e6


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--images", type=int, default=64)
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    bf16 = torch.bfloat16
    d, H, E, T = 768, 3072, 8, a.images * TOKENS_PER_IMAGE
    W1, b1, b2 = (0.02 * rnd(H, d)).to(bf16), (0.02 * rnd(H)).to(bf16), (0.02 * rnd(d)).to(bf16)
    W2 = 0.02 * rnd(d, H)
    comb = [(W2 + 0.01 * rnd(d, H)).to(bf16) for _ in range(E)]
    W2 = W2.to(bf16)
    centroids = rnd(E, d)
    Wg, bg = centroids.to(bf16), (-0.5 * (centroids ** 2).sum(1)).to(bf16)
    opts = dict(b2=b2, cls_stride=TOKENS_PER_IMAGE, input_layernorm=False)

    def tokens(n):
        e = torch.randint(0, E, (n,), generator=g, device="cuda")
        return (centroids[e] + 0.5 * rnd(n, d)).to(bf16)

    # loading: 8-bit blocks of every matrix, bound once
    w16 = cm.ffn_weights(W1, b1, comb, Wg, bg, W2=W2, **opts)
    w8 = cm.ffn_weights(quantize(W1), b1, [quantize(W) for W in comb], Wg, bg, W2=quantize(W2), **opts)
    layer = cm.clearmoe_layer_create(T, d, H, E, 16, cm.BF16)
    report = {}
    try:
        # the batch: both products in 8 bits
        x, y, ref = tokens(T), torch.empty(T, d, device="cuda", dtype=bf16), torch.empty(T, d, device="cuda", dtype=bf16)
        cm.clearmoe_ffn_forward_folded_ex(layer, x, W1, b1, comb, Wg, bg, ref, W2=W2, b2=b2, cls_stride=TOKENS_PER_IMAGE)
        cm.clearmoe_ffn_forward_fp8(layer, x, w8, y)
        report["batch in 8 bits"] = relative(y, ref)
        print(f"batch of {a.images} images: {report['batch in 8 bits']:.4f} from the bf16 layer, "
              f"{timed(lambda: cm.clearmoe_ffn_forward_fp8(layer, x, w8, y)):.1f} us a call")
        # steps of a few tokens: the same 8-bit weights, bf16 activations
        for n in sorted({1, 4, min(cm.FEW_MAX, max(1, a.steps)), cm.FEW_MAX}):
            xs, ys, rs = tokens(n), torch.empty(n, d, device="cuda", dtype=bf16), torch.empty(n, d, device="cuda", dtype=bf16)
            cm.clearmoe_ffn_forward_few(layer, xs, w16, rs)
            cm.clearmoe_ffn_forward_few(layer, xs, w8, ys)
            report[f"{n} tokens"] = relative(ys, rs)
            print(f"{n} tokens: {report[f'{n} tokens']:.4f} from the bf16 weights, "
                  f"{timed(lambda: cm.clearmoe_ffn_forward_few(layer, xs, w8, ys)):.1f} us a call")
        # a projection of the batch's outputs
        P = 0.02 * rnd(3 * d, d)
        rows, P8, out = cm.fp8_rows(T, d), quantize(P), torch.empty(T, 3 * d, device="cuda", dtype=bf16)

        def project():
            cm.clearmoe_fp8_quantize_rows(y, rows)
            cm.clearmoe_fp8_gemm(rows, P8, out)

        project()
        report["projection"] = relative(out, y.float() @ P.T)
        print(f"projection to {3 * d}: {report['projection']:.4f} from fp32, {timed(project):.1f} us a call")
        status = cm.clearmoe_layer_status(layer)
        assert status == cm.OK, cm.clearmoe_strerror(status)
    finally:
        cm.clearmoe_layer_destroy(layer)
    return report


if __name__ == "__main__":
    main()
