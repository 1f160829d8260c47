"""Memory of calls on a given stream: nothing that such a call still uses is
handed to other work."""

import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2608_28941_amd as rrf  # noqa: E402


@pytest.mark.parametrize("op", ["orthogonalize", "muon_step"])
def test_a_dropped_workspace_is_kept_until_the_stream_is_done(op):
    """The allocator gives a freed block to the next request of its size on the
    same stream, unless another stream's work on it is known and pending."""
    say(f"{op}: workspace dropped while the call waits on its stream")
    m, n = 300, 500
    G = torch.randn(m, n, device="cuda")
    W, M = torch.randn(m, n, device="cuda"), torch.zeros(m, n, device="cuda")
    need = rrf.orthogonalize_workspace(torch.float32, m, n, momentum=op == "muon_step")
    want = rrf.orthogonalize(G)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    at = ws.data_ptr()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)             # about a tenth of a second
    if op == "orthogonalize":
        O = rrf.orthogonalize(G, workspace=ws, stream=s)
    else:
        rrf.muon_step(W, M, G, lr=0.1, workspace=ws, stream=s)
    del ws
    other = torch.empty(need, dtype=torch.uint8, device="cuda")
    pending = not s.query()
    assert pending and other.data_ptr() != at
    s.synchronize()
    if op == "orthogonalize":
        assert torch.equal(O, want)
