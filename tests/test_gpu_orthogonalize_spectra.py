"""The orthogonalised step on matrices whose spectra and entries spread in
different ways: few rows, columns or singular directions that carry the matrix,
power laws, heavy tails.

The iterates carry 22 bits whatever the type, so the error against binary64 is
that of the same steps in binary32 on the device, rounded once to the type, or
less; a factor of 1.5 is left for the orders of summation.
"""

import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2608_28941_amd as rrf  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def spectrum(kind, s, l, seed):
    """A float32 s x l matrix on the GPU, s <= l."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    what, *numbers = kind.split(":")
    x, y = [float(v) for v in numbers] + [0.0] * (2 - len(numbers))

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def share(n):
        """1 at a share x of n places, y at the others."""
        w = torch.full((n,), y, device="cuda")
        w[torch.randperm(n, device="cuda", generator=gen)[: max(1, int(x * n))]] = 1.0
        return w

    if what == "rows":
        return randn(s, l) * share(s)[:, None]
    if what == "cols":
        return randn(s, l) * share(l)
    if what in ("values", "power"):
        d = share(s) if what == "values" else torch.arange(1, s + 1, device="cuda") ** -x
        return (torch.linalg.qr(randn(s, s))[0] * d) @ torch.linalg.qr(randn(l, s))[0].t()
    if what == "heavy":
        return randn(s, l) * torch.exp(x * randn(s, l))
    if what == "mean":
        return randn(s, l) + x
    assert what == "gauss"
    return randn(s, l)


KINDS = ["rows:.05:1e-4", "rows:.05:1e-3", "rows:.3:1e-3", "cols:.05:1e-2", "cols:.05:1e-3", "cols:.2:1e-3",
         "values:.5:1e-3", "values:.1:1e-3", "values:.02:1e-4", "power:1", "power:2", "heavy:2", "mean:30", "gauss"]
SIDES = [(205, 700), (512, 1024), (515, 600)]


def steps(X, coeffs=rrf.MUON_COEFFS, eps=1e-7):
    X = X / (torch.linalg.vector_norm(X) + eps)
    for a, b, c in coeffs:
        S = X @ X.t().contiguous()
        X = a * X + (b * S + c * S @ S) @ X
    return X


def layout(G, wide, order):
    """G, or its transpose without wide, column- or row-major."""
    G = G if wide else G.t()
    return G.t().contiguous().t() if order == "c" else G.contiguous()


def errors(dtype, U, got, wide):
    """Distances from binary64 of got and of the binary32 steps' rounded result,
    and the result's norm."""
    ref = steps(U.double())
    plain = steps(U.float()).to(dtype).double()
    got = (got if wide else got.t()).double()
    return [float(torch.linalg.vector_norm(x)) for x in (got - ref, plain - ref, ref)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", ["bf16", "f16"])
def test_as_exact_as_binary32_rounded(name, kind):
    for q, (s, l) in enumerate(SIDES):
        say(f"orthogonalize {name} {kind} {s}x{l}")
        G = spectrum(kind, s, l, 10 + q)
        G = (G / G.abs().max()).to(DT[name])
        wide, order = q % 2 == 0, "cr"[q // 2]
        O = rrf.orthogonalize(layout(G, wide, order))
        e, plain, size = errors(DT[name], G, O, wide)
        assert e <= 1.5 * plain, (s, l, e / size, plain / size)


@pytest.mark.parametrize("kind", KINDS)
def test_bf16_step_as_exact_as_binary32_rounded(kind):
    """W = 0 and lr = scale = 1: W becomes minus the result.  The binary32
    momentum carries the matrix."""
    for q, (s, l) in enumerate(SIDES):
        say(f"muon bf16 {kind} {s}x{l}")
        G, M = spectrum(kind, s, l, 20 + q).bfloat16(), spectrum(kind, s, l, 30 + q)
        wide, order = q % 2 == 1, "rc"[q // 2]
        W = layout(torch.zeros_like(G), wide, order)
        U = G.double() + 0.9 * (0.9 * M.double() + G.double())
        rrf.muon_step(W, layout(M, wide, order), layout(G, wide, order), lr=1.0, momentum=0.9)
        e, plain, size = errors(torch.bfloat16, U, -W, wide)
        assert e <= 1.5 * plain, (s, l, e / size, plain / size)


@pytest.mark.parametrize("kind", KINDS)
def test_f32_as_exact_as_binary32(kind):
    """Steps that are taken together round X X^T where single ones round X:
    their error is that of binary32 steps too, up to sixteen roundings of a
    binary32 result."""
    for q, (s, l) in enumerate([(205, 700), (515, 2060), (600, 3001), (1030, 4100), (2000, 2100)]):
        say(f"orthogonalize f32 {kind} {s}x{l}")
        G = spectrum(kind, s, l, 40 + q)
        wide, order = q % 2 == 0, "crc"[q // 2]
        O = rrf.orthogonalize(layout(G, wide, order))
        e, plain, size = errors(torch.float32, G, O, wide)
        assert e <= 1.5 * plain + 16 * 2.0 ** -24 * size, (s, l, e / size, plain / size)
