"""What the binding's quick path refuses on GPU tensors, and that a refused call has written nothing."""
import pytest
import torch

from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu


def test_status_and_indices():
    A, W, out = cm.fp8_rows(4, 128), cm.fp8_weight(8, 128), torch.zeros(4, 8, device="cuda")
    cm.clearmoe_fp8_quantize_rows(torch.ones(4, 128, device="cuda"), A)
    cm.clearmoe_fp8_quantize_weight(torch.ones(8, 128, device="cuda"), W)
    i = lambda *v, dtype=torch.int32: torch.tensor(v, dtype=dtype, device="cuda")  # noqa: E731
    for bad in (i(0, dtype=torch.int64), i(0, dtype=torch.uint8), i(0, dtype=torch.float32), i(), i(0, 0, 0, 0)[::2]):
        with pytest.raises(ValueError):
            cm.clearmoe_fp8_gemm(A, W, out, status=bad)
    for bad in (i(0, 4, dtype=torch.int64), i(0, 2, 4), i(0, 0, 4, 4)[::2]):
        with pytest.raises(ValueError):
            cm.clearmoe_fp8_grouped_gemm(A, [W], bad, out)
    for bad in (i(0, 1, 2, 3, dtype=torch.int64), i(0, 1, 2)):
        with pytest.raises(ValueError):
            cm.clearmoe_fp8_grouped_gemm(A, [W], i(0, 4), out, perm=bad)
        with pytest.raises(ValueError):
            cm.clearmoe_fp8_quantize_rows(torch.ones(9, 128, device="cuda"), A, gather=bad)
    torch.cuda.synchronize()
    assert not out.any()
    status = i(0)
    cm.clearmoe_fp8_gemm(A, W, out, status=status)
    assert bool((out == 128).all()) and status.item() == 0
    cm.clearmoe_fp8_grouped_gemm(A, [W], i(0, 4), out.zero_(), perm=i(3, 2, 1, 0), status=status)
    assert bool((out == 128).all()) and status.item() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("K,pitch", [(256, 256), (200, 203)])
def test_gathered_rows_outside_x_are_nan(dtype, K, pitch):
    """Every load of the kernels: aligned bf16 and fp32 rows, unaligned ones."""
    x = torch.randn(7, pitch, device="cuda").to(dtype)[:, :K]
    at = [6, -1, 0, 7, 2 ** 31 - 1, -2 ** 31, 3, 3, 2000000]
    g = cm.fp8_rows(len(at), K)
    cm.clearmoe_fp8_quantize_rows(x, g, gather=torch.tensor(at, dtype=torch.int32, device="cuda"))
    plain, got, want = cm.fp8_rows(7, K), torch.empty(len(at), K, device="cuda"), torch.empty(7, K, device="cuda")
    cm.clearmoe_fp8_quantize_rows(x, plain)
    cm.clearmoe_fp8_dequantize(g, got)
    cm.clearmoe_fp8_dequantize(plain, want)
    kb = -(-K // 128)
    for i, r in enumerate(at):
        if 0 <= r < 7:
            assert torch.equal(got[i], want[r])
            assert torch.equal(g.q.view(torch.uint8)[i], plain.q.view(torch.uint8)[r])
        else:
            assert bool(got[i].isnan().all()) and bool((g.scale[i, :kb] == 255).all())
    L = cm.lib()
    for rows in (0, -1):
        assert L.clearmoe_fp8_quantize_gathered(x.data_ptr(), rows, cm.F32, 256, None, plain.ref, None) == cm.EINVAL
    assert L.clearmoe_fp8_quantize_gathered(x.data_ptr(), 6, cm.F32, 256, None, plain.ref, None) == cm.EINVAL


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tokens_and_outputs_of_a_layer(dtype):
    d, H, other = 64, 256, torch.float32 if dtype == torch.bfloat16 else torch.bfloat16
    h = cm.clearmoe_layer_create(8, d, H, 2, 16, cm.BF16 if dtype == torch.bfloat16 else cm.F32)
    g = lambda *s, t=dtype: torch.zeros(*s, device="cuda", dtype=t)  # noqa: E731
    w = cm.ffn_weights(g(H, d), g(H), [g(d, H)] * 2, g(2, d), g(2), b2=torch.ones(d, device="cuda", dtype=dtype))
    x, out = g(4, d), g(4, d)
    for bad_x, bad_out in ((g(4, d, t=other), out), (x, g(4, d, t=other)), (x, g(3, d)), (x, g(4, d // 2)), (g(4, 2 * d), out),
                           (g(2, 2, d), out), (g(4 * d), out), (x, g(4 * d))):
        for call in (cm.clearmoe_ffn_forward_few, cm.clearmoe_ffn_forward_fp8):
            with pytest.raises(ValueError):
                call(h, bad_x, w, bad_out)
    torch.cuda.synchronize()
    assert not out.any()
    cm.clearmoe_ffn_forward_few(h, x, w, out)
    assert bool((out == 1).all())
    cm.clearmoe_layer_destroy(h)
