"""The example that serves a layer in 8 bits: each path's distance from the bf16 layer.

An e4m3 value is off by up to 2^-4 of itself, uniformly about 2^-4 / sqrt 3 = 3.6 % in the worst binade, 2.6 % over
one; a product of two quantised operands then by 3.7 % RMS of its sum, two such products in a row (x and W1, z and
W_comb; the GELU hands on about all of it) by 5.3 %, and weights alone, twice, by 3.7 %. Twice those are the bounds."""
import pytest

pytestmark = pytest.mark.gpu


def test_example_runs():
    from examples import serve_8bit
    r = serve_8bit.main(["--images", "3", "--steps", "5"])
    assert r["batch in 8 bits"] < 0.106
    assert all(v < 0.074 for k, v in r.items() if "tokens" in k) and len([k for k in r if "tokens" in k]) == 4
    assert r["projection"] < 0.074
