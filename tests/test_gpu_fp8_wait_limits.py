"""The layer in 8 bits under wait limits of 1 to 200 microseconds: its kernels (on one SM and on pairs, 8-bit and bf16
outputs, grouped) give up between their copies, let what is in flight land, and return; the call reports
CLEARMOE_ETIMEOUT or completes; afterwards, with the usual limit, the handle gives the bits that it gave before."""
import pytest
import torch

from paper_2606_28516_gb300 import clearmoe as cm

pytestmark = pytest.mark.gpu

LIMITS = (1_000, 4_000, 16_000, 50_000, 200_000)


def _layer(T, d, H, E, cls=0, ln=False):
    g = torch.Generator(device="cuda").manual_seed(T + d + H)
    w = lambda *s: 0.02 * torch.randn(*s, generator=g, device="cuda")  # noqa: E731

    def q(n, k):
        m = cm.fp8_weight(n, k)
        cm.clearmoe_fp8_quantize_weight(w(n, k), m)
        return m

    b = lambda *s: w(*s).to(torch.bfloat16)  # noqa: E731
    weights = cm.ffn_weights(q(H, d), b(H), [q(d, H) for _ in range(E)], b(E, d), b(E), b2=b(d),
                             W2=q(d, H) if cls else None, cls_stride=cls, input_layernorm=ln)
    x, out = b(T, d) * 50, torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    h = cm.clearmoe_layer_create(T, d, H, E, 16, cm.BF16)
    return h, out, weights, lambda: cm.clearmoe_ffn_forward_fp8(h, x, weights, out)


@pytest.mark.parametrize("T,d,H,E,kw", [(9973, 768, 4096, 8, {}), (300, 768, 16384, 4, {}), (6304, 384, 4096, 4, dict(cls=197)),
                                        (2000, 192, 8192, 2, dict(ln=True)), (12000, 1024, 1024, 3, {})])
def test_gives_up_and_recovers(T, d, H, E, kw):
    h, out, _, call = _layer(T, d, H, E, **kw)
    try:
        call()
        assert cm.clearmoe_layer_status(h) == 0
        want = out.clone()
        gave_up = []
        for limit in LIMITS:
            for _ in range(4):
                cm.clearmoe_debug_set_wait(h, limit, 0)
                call()
                call()
                st = cm.clearmoe_layer_status(h)
                assert st in (0, cm.ETIMEOUT), (limit, st)
                gave_up.append(st == cm.ETIMEOUT)
                cm.clearmoe_debug_set_wait(h, 1_000_000_000, 0)
                out.fill_(float("nan"))
                call()
                assert cm.clearmoe_layer_status(h) == 0
                assert torch.equal(out, want), limit
        if d == 768:  # the two cases of long K loops; the others' waits may all end within a microsecond
            assert gave_up[0]
    finally:
        cm.clearmoe_layer_destroy(h)


def test_first_call_gives_up():
    """A handle whose first calls give up has no routing of an earlier call behind it."""
    h, want, _, call = _layer(3000, 768, 4096, 4)
    h2, out, _, call2 = _layer(3000, 768, 4096, 4)
    try:
        call()
        assert cm.clearmoe_layer_status(h) == 0
        cm.clearmoe_debug_set_wait(h2, 1_000, 1)
        for _ in range(3):
            call2()
        assert cm.clearmoe_layer_status(h2) == cm.ETIMEOUT
        cm.clearmoe_debug_set_wait(h2, 1_000_000_000, 0)
        call2()
        assert cm.clearmoe_layer_status(h2) == 0 and torch.equal(out, want)
    finally:
        cm.clearmoe_layer_destroy(h)
        cm.clearmoe_layer_destroy(h2)
