"""A 4-bit matrix times real columns of the smallest binary32 numbers, brought
back to the usual range by the matrix's scales.

A value x of B is taken as a sum of three bfloat16 parts: as it is from 2^-110
on, below cut towards zero to a multiple of 2^-133.  So for every entry of C

    |C - ref| <= length 2^-23 |A|^T |B| + 2^-133 sum |A| + 2^-24 |ref|,

the second term only where B holds such values.
"""

import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2608_28941_amd as rrf  # noqa: E402


@pytest.mark.parametrize("exponent", [-149, -140, -133, -126, -120, -112, -110, -109])
@pytest.mark.parametrize("trans", [True, False])
@pytest.mark.parametrize("n", [1, 40, 200])
def test_small_values(n, trans, exponent):
    say(f"mx4_apply trans={trans} n={n} values near 2^{exponent}")
    k, m = 320, 300
    gen = torch.Generator(device="cuda").manual_seed(-exponent)
    A = rrf.mx4_quantize(torch.randn(m, k, device="cuda", generator=gen).t())
    A = rrf.Mx4(A.codes, A.scales + 110, k)             # values of up to 2^113
    rows = k if trans else m
    # in [1, 2) times 2^exponent, either sign; rounded to multiples of 2^-149
    x = (1.0 + torch.rand(n, rows, device="cuda", generator=gen, dtype=torch.float64)) * 2.0 ** exponent
    x = x * torch.sign(torch.randn(n, rows, device="cuda", generator=gen, dtype=torch.float64))
    x = x.float()
    V = A.dequantize().double()
    V = (V.t() if trans else V).contiguous()
    b = x.double().t().contiguous()
    ref, size = V @ b, V.abs() @ b.abs()
    tol = rows * 2.0 ** -23 * size + 2.0 ** -24 * ref.abs()
    if exponent < -110:
        tol = tol + 2.0 ** -133 * V.abs().sum(1, keepdim=True)
    far = (rrf.mx4_apply(A, x.t(), trans=trans).double() - ref).abs()
    assert bool((far <= tol).all()), float((far / tol).max())
