"""The binding's quick path and its checks: arguments that are not as they should be are refused by name before any call,
and the quick path's results are those of the call by integers."""
import pytest
import torch

from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu


def test_refused_arguments():
    A, W = cm.fp8_rows(4, 128), cm.fp8_weight(8, 128)
    x, out = torch.zeros(4, 128, device="cuda"), torch.zeros(4, 8, device="cuda")
    cm.clearmoe_fp8_quantize_weight(torch.zeros(8, 128, device="cuda"), W)
    cm.clearmoe_fp8_quantize_rows(x, A)
    for bad in (x.half(), x.cpu(), x[:3], x[:, :127], x[0], torch.zeros(128, 4, device="cuda").T):
        with pytest.raises(ValueError):
            cm.clearmoe_fp8_quantize_rows(bad, A)
    for bad in (out.half(), out.cpu(), out[:3], out[:, :7], torch.zeros(8, 4, device="cuda").T):
        with pytest.raises(ValueError):
            cm.clearmoe_fp8_gemm(A, W, bad)
    b = torch.zeros(8, device="cuda")
    for bad in (b.half(), b.cpu(), b[:7], torch.zeros(16, device="cuda")[::2]):
        with pytest.raises(ValueError):
            cm.clearmoe_fp8_gemm(A, W, out, bias=bad)
    with pytest.raises(ValueError):
        cm.clearmoe_fp8_gemm(A, W, out, status=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(cm.ClearMoEError, match="clearmoe_fp8_gemm"):
        cm.clearmoe_fp8_gemm(A, W, out, act=77)
    with pytest.raises(TypeError):
        cm.clearmoe_fp8_gemm(A, W, out, act="gelu")


def test_layers_refuse_strided_and_host_tensors():
    h = cm.clearmoe_layer_create(8, 64, 256, 2, 16, cm.BF16)
    g = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    w = cm.ffn_weights(g(256, 64), g(256), [g(64, 256)] * 2, g(2, 64), g(2))
    x, out = g(4, 64), g(4, 64)
    cm.clearmoe_ffn_forward_few(h, x, w, out)
    for bad_x, bad_out in ((x.cpu(), out), (g(4, 128)[:, ::2], out), (x, out.cpu()), (x, g(4, 128)[:, ::2])):
        with pytest.raises(ValueError):
            cm.clearmoe_ffn_forward_few(h, bad_x, w, bad_out)
        with pytest.raises(ValueError):
            cm.clearmoe_ffn_forward_fp8(h, bad_x, w, bad_out)
    with pytest.raises(cm.ClearMoEError, match="clearmoe_ffn_forward_few"):
        cm.clearmoe_ffn_forward_few(h, g(9, 64), w, g(9, 64))
    with pytest.raises(cm.ClearMoEError, match="clearmoe_ffn_forward_fp8"):
        cm.clearmoe_ffn_forward_fp8(h, x, w, out)  # not 8-bit weights
    torch.cuda.synchronize()
    assert cm.clearmoe_layer_status(h) == 0
    cm.clearmoe_layer_destroy(h)


@pytest.mark.parametrize("M", [1, 5])
def test_by_tensors_and_by_integers(M):
    """Row pitches of one row and of several, on torch's current stream and on a given one."""
    s = torch.cuda.Stream()
    x = torch.randn(M, 300, device="cuda")[:, :200]
    W, b = cm.fp8_weight(40, 200), torch.randn(40, device="cuda").to(torch.bfloat16)
    cm.clearmoe_fp8_quantize_weight(torch.randn(40, 200, device="cuda"), W)
    torch.cuda.synchronize()
    outs = []
    for stream in (None, s):
        A, out = cm.fp8_rows(M, 200), torch.zeros(M, 64, device="cuda")[:, :40]
        torch.cuda.synchronize()
        cm.clearmoe_fp8_quantize_rows(x, A, stream=stream)
        cm.clearmoe_fp8_gemm(A, W, out, bias=b, act=cm.ACT_GELU, stream=stream)
        torch.cuda.synchronize()
        outs.append(out)
    B, out = cm.fp8_rows(M, 200), torch.zeros(M, 64, device="cuda")[:, :40]
    torch.cuda.synchronize()
    calls = cm._bind_calls()
    assert calls.quantize_rows(x.data_ptr(), cm.F32, 300, None, B.addr, s.cuda_stream) == 0
    assert calls.gemm(B.addr, W.addr, b.data_ptr(), cm.BF16, cm.ACT_GELU, None, out.data_ptr(), cm.F32, 64, s.cuda_stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], out) and bool(out.abs().sum() > 0)
