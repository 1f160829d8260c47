"""The orthogonalised step where norms, eps and coefficients leave the usual
range."""

import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2608_28941_amd as rrf  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.mark.parametrize("eps", [1e-7, 1e-20, 1e-300, 5e-324, 1e300])
@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
def test_zero_matrix_whatever_eps(name, eps):
    """0 / (0 + eps) = 0, alone and beside another matrix, whose result does not
    depend on that."""
    say(f"zero matrix {name} eps={eps}")
    gen = torch.Generator(device="cuda").manual_seed(1)
    G = torch.randn(3, 50, 70, device="cuda", generator=gen).to(DT[name])
    G[0] = 0
    G[2] = 0
    O = rrf.orthogonalize(G, eps=eps)
    assert not bool(O[0].any()) and not bool(O[2].any())
    assert torch.equal(O[1], rrf.orthogonalize(G[1], eps=eps)) and bool(torch.isfinite(O[1]).all())
    big = torch.zeros(300, 450, device="cuda", dtype=DT[name])
    assert not bool(rrf.orthogonalize(big, eps=eps).any())
    # A step on it leaves the weights but for their decay.
    W = torch.randn(50, 70, device="cuda", generator=gen).to(DT[name])
    keep = torch.tensor(1.0 - 0.1 * 0.5, dtype=torch.float32, device="cuda")
    want = (W.float() * keep).to(DT[name])
    M = torch.zeros(50, 70, device="cuda")
    rrf.muon_step(W, M, G[0].contiguous(), lr=0.1, weight_decay=0.5, eps=eps)
    assert torch.equal(W, want) and not bool(M.any())


@pytest.mark.parametrize("coeffs", [
    ((1e-12, 0.0, 0.0),) * 3,
    ((1e-25, 0.0, 0.0), (1e3, 0.0, 0.0), (1e3, 0.0, 0.0)),
    ((1e-10, 0.0, 0.0),) * 4 + ((9e3, 0.0, 0.0),) * 4,
    ((1e-15, -1e-15, 0.0), (2.0, -1e30, 1e59)),
])
def test_coefficients_that_shrink_the_values(coeffs):
    """Singular values far below 1 on the way: X and A are stored with scales
    past binary32's range.  22 bits and binary32 sums: 16 roundings of 2^-20 a
    step, and the result's own, down to the least normal number."""
    say(f"orthogonalize {coeffs}")
    gen = torch.Generator(device="cuda").manual_seed(2)
    G = torch.randn(60, 90, device="cuda", generator=gen)
    X = G.double() / (torch.linalg.vector_norm(G.double()) + 1e-7)
    for a, b, c in coeffs:
        S = X @ X.t().contiguous()
        X = a * X + (b * S + c * S @ S) @ X
    O = rrf.orthogonalize(G, coeffs).double()
    size = float(torch.linalg.vector_norm(X))
    assert 1e-37 < size
    assert float(torch.linalg.vector_norm(O - X)) <= 16 * len(coeffs) * 2.0 ** -20 * size
