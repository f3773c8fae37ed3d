"""How the token-scoring calls of the binding are made: streams, arrays that are kept, rows that are reported."""
import math

import pytest
import torch

from . import test_gpu_score as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2605_28396_amd import binding
    return binding


def test_stream_zero_is_the_default_stream(B, monkeypatch):
    """The handle that the library gets; nothing is enqueued."""
    got = []
    monkeypatch.setattr(B.lib, "adwin_opd_token_logp", lambda p, ws, n, stream: got.append(stream) or 0)
    z, ids = torch.zeros(300, 50, device="cuda"), torch.zeros(300, 1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for s in (None, 0, torch.cuda.default_stream(), side, side.cuda_stream):
            B.adwin_opd_token_logp(z, ids, stream=s)
    assert got == [side.cuda_stream, None, None, side.cuda_stream, side.cuda_stream]


def test_a_head_is_laid_out_again_in_its_arrays(B):
    """A captured product goes on with the weights that set() brings; other sizes get arrays of their own."""
    V, H, T = 3001, 200, 20
    W = [torch.randn(V, H, generator=S._gen(k)).cuda() for k in range(3)]
    h = torch.randn(T, H, generator=S._gen(9)).cuda()
    want = [B.QuantHead(w).logits(h) for w in W]
    head = B.QuantHead(W[0])
    at = head.W_q.data_ptr(), head.W_scale.data_ptr()
    z = torch.empty_like(want[0])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        head.logits(h, z=z)
    for k in (1, 2, 0, 1):
        head.set(W[k])
        assert (head.W_q.data_ptr(), head.W_scale.data_ptr()) == at
        z.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, want[k]), k
    for other in (W[0][:, :100].contiguous(), W[0][:5], W[0][:, :199]):
        head.set(other)
        assert torch.equal(head.logits(h[:, :other.shape[1]]), B.QuantHead(other).logits(h[:, :other.shape[1]]))
    with pytest.raises(ValueError):
        B.adwin_opd_quant_rows(W[0], q=torch.empty(V, H, dtype=torch.int8, device="cuda"))
    with pytest.raises(ValueError):
        B.adwin_opd_quant_rows(W[0], scale=torch.empty(V, device="cuda").half())
