"""Products of two 4-bit matrices whose rows of scales end inside a load, with
other data right behind codes and scales.

Every product is exact and at most k additions round, by 2^-23 relative to a
partial sum that |A|^T |B| bounds; the result is binary32.
"""

import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2608_28941_amd as rrf  # noqa: E402


def followed(t):
    """t's bytes in a larger allocation, 0xff behind them (as scales: NaN)."""
    buf = torch.full((t.numel() + 4096,), 255, dtype=torch.uint8, device="cuda")
    buf[: t.numel()] = t.reshape(-1)
    return buf[: t.numel()].view(t.shape)


def quantized(k, n, gen):
    """A 4-bit matrix and its values in float64."""
    x = torch.randn(n, k, device="cuda", generator=gen) * torch.exp2(
        torch.randint(-6, 7, (n, k), device="cuda", generator=gen).float())
    A = rrf.mx4_quantize(x.t())
    return rrf.Mx4(followed(A.codes), followed(A.scales), k), A.dequantize().double()


@pytest.mark.parametrize("k", [200, 256, 700, 1200, 1400, 1700, 2300])
@pytest.mark.parametrize("m,n", [(65, 65), (65, 129), (129, 65), (641, 385), (1025, 1153), (2881, 3265), (4097, 4353)])
def test_scales_that_end_inside_a_load(k, m, n):
    """One to nine chunks of 256 rows, one row or column in the last tile."""
    say(f"mx4_product k={k} {m}x{n}, data behind it")
    gen = torch.Generator(device="cuda").manual_seed(k + m)
    A, Av = quantized(k, m, gen)
    B, Bv = quantized(k, n, gen)
    C = rrf.mx4_product(A, B).double()
    ref = Av.t() @ Bv
    tol = k * 2.0 ** -23 * (Av.abs().t() @ Bv.abs()) + 2.0 ** -24 * ref.abs()
    far = (C - ref).abs() - tol
    assert bool((far <= 0).all()), float(far.max())
