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


def test_a_head_reports_what_it_could_not_compute(B):
    W, h = torch.randn(70, 64, generator=S._gen(1)), torch.randn(9, 64, generator=S._gen(2))
    W[13, 5] = math.nan
    h[4, 60] = math.inf
    head = B.QuantHead(W.cuda())
    assert torch.equal(head.row_status.cpu(), (torch.arange(70) == 13).int() * B.ADWIN_DEV_NONFINITE)
    at = head.row_status.data_ptr()
    assert torch.equal(B.adwin_opd_quant_rows(W.cuda(), row_status=1)["row_status"], head.row_status)
    z, status = head.logits(h.cuda(), row_status=True)
    assert torch.equal(z, head.logits(h.cuda())) and torch.all(z[4] == 0) and torch.all(z[:, 13] == 0)
    assert torch.equal(status.cpu(), (torch.arange(9) == 4).int() * B.ADWIN_DEV_NONFINITE)
    W[13, 5] = 0
    head.set(W.cuda())
    assert torch.all(head.row_status == 0) and head.row_status.data_ptr() == at


def test_the_offline_teacher_leaves_excluded_rows_out(B):
    import importlib.util
    import os
    spec = importlib.util.spec_from_file_location("offline_teacher_rows", os.path.join(os.path.dirname(os.path.dirname(
        os.path.abspath(__file__))), "examples", "offline_teacher.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    V, H, T = 500, 64, 40
    h_t, W_t = torch.randn(T, 2 * H, generator=S._gen(1)).bfloat16(), torch.randn(V, 2 * H, generator=S._gen(2)).bfloat16() * 0.1
    h_s, W_s = torch.randn(T, H, generator=S._gen(3)).bfloat16(), torch.randn(V, H, generator=S._gen(4)).bfloat16() * 0.1
    ids = S._ids(T, 1, V, 5)[:, 0].cuda()
    sound = example.teacher_answers(B.QuantHead(W_t.cuda()), h_t.cuda(), ids, top=6, slab=16)
    h_t[3, 7], h_t[20, 0] = math.nan, math.inf
    got = example.teacher_answers(B.QuantHead(W_t.cuda()), h_t.cuda(), ids, top=6, slab=16)
    kept = torch.ones(T, dtype=torch.bool, device="cuda")
    kept[[3, 20]] = False
    assert all(torch.equal(got[k][kept], sound[k][kept]) for k in sound)
    assert torch.all(got["top_ids"][~kept] == -1) and torch.all(got["top_logp"][~kept] == 0) and torch.all(got["logp"][~kept] == 0)
    # a student's row that is not finite counts as little as one without answers
    want = {k: v.clone() for k, v in got.items()}
    want["top_ids"][11], want["top_logp"][11] = -1, 0
    clean = h_s.clone()
    h_s[11, 2] = math.nan
    loss, dh, dW = example.student_step(h_s.cuda(), W_s.cuda(), got, bonus=0.05)
    loss_want, dh_want, dW_want = example.student_step(clean.cuda(), W_s.cuda(), want, bonus=0.05)
    assert float(loss) == float(loss_want) and torch.equal(dh, dh_want) and torch.equal(dW, dW_want)
    W_t[9, 9] = math.nan
    with pytest.raises(ValueError):
        example.teacher_answers(B.QuantHead(W_t.cuda()), h_t.cuda(), ids)
