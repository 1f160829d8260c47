"""The operators beside autograd: they record nothing, refuse where that would
lose a gradient silently, and mark what they write."""

import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2608_28941_amd as rrf  # noqa: E402


def test_refused_unless_detached():
    say("inputs that require grad")
    W = rrf.mx4_quantize(torch.randn(40, 64, device="cuda").t())
    x = torch.randn(3, 64, device="cuda").t().requires_grad_()
    with pytest.raises(RuntimeError, match="requires grad"):
        rrf.mx4_apply(W, x)
    with pytest.raises(RuntimeError, match="requires grad"):
        rrf.orthogonalize(x)
    want = rrf.mx4_apply(W, x.detach())
    with torch.no_grad():
        assert torch.equal(rrf.mx4_apply(W, x), want)
        assert torch.equal(rrf.orthogonalize(x), rrf.orthogonalize(x.detach()))
    # 4 bits carry no gradient
    assert not rrf.mx4_quantize(x).dequantize().requires_grad


def test_a_stale_saved_weight_is_noticed():
    say("muon_step on a weight that a graph keeps")
    W = torch.randn(20, 30, device="cuda", requires_grad=True)
    x = torch.randn(20, 30, device="cuda", requires_grad=True)
    M = torch.zeros(20, 30, device="cuda")
    y = (W * x).sum()
    rrf.muon_step(W, M, torch.randn(20, 30, device="cuda"), lr=0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    z = (M * x).sum()
    rrf.muon_step(W, M, torch.randn(20, 30, device="cuda"), lr=0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()
    out = torch.empty(20, 30, device="cuda")
    z = (out * x).sum()
    rrf.orthogonalize(W.detach(), out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()
    with torch.inference_mode():
        V = torch.randn(20, 30, device="cuda")
        rrf.muon_step(V, torch.zeros_like(V), torch.randn_like(V), lr=0.1)
        rrf.orthogonalize(V, out=V)
