"""The operators in every tile that the host may choose, cut off at both edges.

tests/test_tile_choice_cpu.py shows that the lists here reach all of them.
"""

import ctypes

import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2608_28941_amd as rrf  # noqa: E402
from paper_2608_28941_amd import _abi  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CODE = {"f32": _abi.RRF_F32, "bf16": _abi.RRF_BF16, "f16": _abi.RRF_F16}
PARTS = {"f32": 3, "bf16": 1, "f16": 2}
U_OUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}

# (batch, short side, long side)
ORTHO = [(1, 33, 70), (1, 511, 3067), (1, 520, 3121), (1, 1003, 6001), (1, 1030, 2061), (1, 1333, 15997),
         (1, 2001, 2603), (1, 2003, 4001), (1, 2001, 6003), (1, 2501, 15001), (1, 3001, 3907), (1, 4099, 4111),
         (1, 4501, 5851), (16, 190, 250), (5, 1000, 1402)]

# (trans, k, m, n) with the type of B
APPLY = {
    "bf16": [(0, 2051, 131, 3001), (0, 3001, 4099, 389), (0, 5003, 4099, 65), (0, 4091, 131, 2047),
             (0, 5003, 6001, 97), (0, 1301, 131, 3001), (0, 3001, 4099, 97), (0, 333, 131, 65), (0, 333, 771, 65),
             (1, 5003, 2049, 389), (1, 2051, 9001, 65), (1, 333, 2049, 3001), (1, 5003, 131, 2047),
             (1, 333, 1283, 3001), (1, 1301, 131, 3001), (1, 333, 131, 65), (1, 777, 131, 65)],
    "f16": [(0, 2051, 131, 3001), (0, 3001, 4099, 389), (0, 4091, 131, 3001), (0, 5003, 4099, 65),
            (0, 4091, 1283, 2047), (0, 515, 4099, 2047), (0, 1301, 131, 3001), (0, 4091, 4099, 97), (0, 333, 131, 65),
            (0, 333, 771, 65), (1, 333, 2049, 3001), (1, 8197, 131, 3001), (1, 333, 6001, 3001), (1, 3001, 131, 3001),
            (1, 3001, 2049, 3001), (1, 8197, 259, 2047), (1, 333, 1283, 3001), (1, 1301, 131, 3001), (1, 333, 131, 65),
            (1, 777, 131, 65)],
    "f32": [(0, 2051, 131, 3001), (0, 8197, 9001, 97), (0, 5003, 131, 2047), (0, 4091, 6001, 65),
            (0, 1029, 4099, 2047), (0, 1301, 131, 3001), (0, 777, 2049, 1543), (0, 333, 131, 65), (0, 333, 771, 65),
            (1, 333, 2049, 3001), (1, 8197, 6001, 97), (1, 333, 6001, 3001), (1, 3001, 131, 3001), (1, 5003, 771, 3001),
            (1, 333, 1283, 3001), (1, 5003, 259, 1543), (1, 333, 131, 65), (1, 777, 131, 65)],
}
APPLY_CASES = [(name, *case) for name in APPLY for case in APPLY[name]]

# (M, N, k)
PRODUCT = [(131, 65, 300), (9001, 200, 300), (4099, 2047, 300), (6001, 1543, 300)]


# --- orthogonalised steps -----------------------------------------------------------

def steps(X, coeffs=rrf.MUON_COEFFS, eps=1e-7):
    X = X / (torch.linalg.vector_norm(X) + eps)
    for a, b, c in coeffs:
        S = X @ X.t().contiguous()
        X = a * X + (b * S + c * S @ S) @ X
    return X


def padded(t, order, pad):
    """Matrices of a batch on the GPU, column- or row-major, pad elements of NaN
    behind each column or row."""
    t = t.mT if order == "c" else t
    buf = torch.full((*t.shape[:-1], t.shape[-1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    view = buf[..., : t.shape[-1]]
    view.copy_(t)
    return buf, view.mT if order == "c" else view


def entries(name, got, ref, size):
    """Every entry: the type's rounding, and before it an error that is spread
    over the matrix, of norm 1e-4 at most (binary32 steps reach 6e-5), taken as
    ten times its mean in one place."""
    tol = U_OUT[name] * 1.01 * ref.abs() + 1e-3 * size / ref.numel() ** 0.5
    far = (got.double() - ref).abs() - tol
    assert bool((far <= 0).all()), float(far.max())


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("q", range(len(ORTHO)))
def test_orthogonalize_and_step(name, q):
    """Both orientations and orders in turn, padded: the result in every entry,
    its norm-wise error against binary32 steps, and W <- 0.9 W - O."""
    batch, s, l = ORTHO[q]
    gen = torch.Generator(device="cuda").manual_seed(100 + q)
    for h in range(2):
        wide, order, pad = (q + h) % 2 == 0, "cr"[(q // 2 + h) % 2], (q + h) % 4
        say(f"orthogonalize tiles {name} {batch}x{s}x{l} wide={wide} {order} pad {pad}")
        G = torch.randn(batch, *((s, l) if wide else (l, s)), device="cuda", generator=gen).to(DT[name])
        gbuf, g = padded(G, order, pad)
        if h == 0:
            buf, out = padded(torch.zeros_like(G), order, pad)
            got = rrf.orthogonalize(g, out=out)
        else:
            W = torch.randn(G.shape, device="cuda", generator=gen).mul_(l ** -0.5).to(DT[name])
            buf, w = padded(W, order, pad)
            mbuf, m = padded(torch.zeros(G.shape, device="cuda"), order, 0)
            got = rrf.muon_step(w, m, g, lr=0.1, momentum=0.5, nesterov=False, weight_decay=1.0, scale=10.0)
            assert torch.equal(m, g.float())
        width = G.shape[-2] if order == "c" else G.shape[-1]
        assert bool(torch.isnan(buf[..., width:]).all())
        for i in range(batch):
            X = (G[i] if wide else G[i].t()).double()
            ref = steps(X)
            size = float(torch.linalg.vector_norm(ref))
            if h == 0:
                here = (got[i] if wide else got[i].t()).double()
                plain = steps(X.float()).to(DT[name]).double()
                e, f = (float(torch.linalg.vector_norm(x - ref)) for x in (here, plain))
                assert e <= 1.5 * f + 16 * 2.0 ** -24 * size, (i, e / size, f / size)
                entries(name, here, ref, size)
            else:
                want = 0.9 * W[i].double() - (ref if wide else ref.t())
                entries(name, got[i], want, size)


# --- a 4-bit matrix times real columns -----------------------------------------------

def four_bits(k, m, gen):
    x = torch.randn(m, k, device="cuda", generator=gen) * torch.exp2(
        torch.randint(-6, 7, (m, k), device="cuda", generator=gen).float())
    return rrf.mx4_quantize(x.t())


def values(A):
    return A.dequantize().double().contiguous()


def check(name, C, V, x, length):
    """Every product is exact, at most `length` additions round by 2^-23, and the
    result is rounded once."""
    ref = V @ x
    tol = length * 2.0 ** -23 * (V.abs() @ x.abs()) + U_OUT[name] * ref.abs() + (2.0 ** -25 if name == "f16" else 0.0)
    far = (C.double() - ref).abs() - tol
    assert bool((far <= 0).all()), float(far.max())


@pytest.mark.parametrize("name,trans,k,m,n", APPLY_CASES)
def test_apply(name, trans, k, m, n):
    say(f"mx4_apply tiles {name} trans={trans} k={k} m={m} n={n}")
    gen = torch.Generator(device="cuda").manual_seed(k + m + n)
    A = four_bits(k, m, gen)
    length, pad = (k if trans else m), (k + n) % 9
    x = (torch.randn(n, length, device="cuda", generator=gen) / 64).to(DT[name])
    _, view = padded(x.t(), "c", pad)
    V = values(A)
    check(name, rrf.mx4_apply(A, view, trans=bool(trans)), V.t().contiguous() if trans else V,
          x.double().t().contiguous(), length)


@pytest.mark.parametrize("name,trans,k,m,n", APPLY_CASES)
def test_apply_nonfinite(name, trans, k, m, n):
    """NaN and infinities where the formula has them, and nowhere else."""
    say(f"mx4_apply nonfinite {name} trans={trans} k={k} m={m} n={n}")
    gen = torch.Generator(device="cuda").manual_seed(k + m + n)
    A = four_bits(k, m, gen)
    A.scales[m // 2, (k - 1) // 32] = 255                       # the block that holds a column's last row
    length = k if trans else m
    x = torch.randn(n, length, device="cuda", generator=gen).to(DT[name])
    x[n - 1, length - 1] = float("inf")
    x[n // 2, 0] = float("-inf")
    x[n // 3, length // 2] = float("nan")
    V = values(A)
    ref = (V.t().contiguous() if trans else V) @ x.double().t().contiguous()
    C = rrf.mx4_apply(A, x.t(), trans=bool(trans))
    assert torch.equal(torch.isnan(C), torch.isnan(ref))
    assert torch.equal(C == float("inf"), ref == float("inf")) and torch.equal(C == -float("inf"), ref == -float("inf"))


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("trans,k,m,n", [(1, 333, 131, 1), (1, 333, 131, 20), (0, 333, 131, 1), (0, 333, 771, 40),
                                         (1, 333, 2049, 301), (1, 777, 131, 65), (0, 1301, 131, 301), (0, 333, 771, 65)])
def test_results_with_gaps(name, trans, k, m, n):
    """ldc above the rows of C: what lies between the columns stays."""
    say(f"mx4 ldc {name} trans={trans} k={k} m={m} n={n}")
    gen = torch.Generator(device="cuda").manual_seed(9)
    A = four_bits(k, m, gen)
    length, rows = (k, m) if trans else (m, k)
    x = torch.randn(n, length, device="cuda", generator=gen).to(DT[name])
    buf = torch.full((n, rows + 5), float("nan"), dtype=DT[name], device="cuda")
    lib, need = _abi.load(), ctypes.c_size_t()
    st = torch.cuda.current_stream().cuda_stream
    _abi.check(lib.rrf_mx4_apply_workspace(CODE[name], trans, k, m, n, ctypes.byref(need)), "workspace")
    ws = torch.empty(max(need.value, 16), dtype=torch.uint8, device="cuda")
    _abi.check(lib.rrf_mx4_apply(CODE[name], trans, k, m, A.codes.data_ptr(), A.scales.data_ptr(), x.data_ptr(), length,
                                 n, buf.data_ptr(), rows + 5, ws.data_ptr(), need.value, st), "apply")
    assert torch.equal(buf[:, :rows].t(), rrf.mx4_apply(A, x.t(), trans=bool(trans)))
    assert bool(torch.isnan(buf[:, rows:]).all())
    if trans:
        B = rrf.mx4_quantize(x.t())
        buf = torch.full((n, rows + 3), float("nan"), dtype=DT[name], device="cuda")
        _abi.check(lib.rrf_mx4_product(CODE[name], m, n, k, A.codes.data_ptr(), A.scales.data_ptr(), B.codes.data_ptr(),
                                       B.scales.data_ptr(), buf.data_ptr(), rows + 3, st), "product")
        assert torch.equal(buf[:, :rows].t(), rrf.mx4_product(A, B, DT[name]))
        assert bool(torch.isnan(buf[:, rows:]).all())


@pytest.mark.parametrize("n", [1, 2, 33, 64])
@pytest.mark.parametrize("trans", [1, 0])
def test_few_columns_nonfinite(n, trans):
    """As above for the kernels for few columns, one column among them."""
    for name in DT:
        test_apply_nonfinite(name, trans, 601, 90, n)


# --- two 4-bit matrices ---------------------------------------------------------------

@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,N,k", PRODUCT)
def test_product(name, M, N, k):
    say(f"mx4_product tiles {name} {M}x{N} k={k}")
    gen = torch.Generator(device="cuda").manual_seed(M + N)
    A, B = four_bits(k, M, gen), four_bits(k, N, gen)
    A.scales.sub_(8)
    check(name, rrf.mx4_product(A, B, DT[name]), values(A).t().contiguous(), values(B), k)
