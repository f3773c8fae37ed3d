"""The sequence-distillation example where a teacher's state is not finite: such beams have no continuations, the others have theirs."""
import pytest
import torch

from .test_gpu_sequence_teacher import ex  # noqa: F401

pytestmark = pytest.mark.gpu


def test_beams_whose_state_is_not_finite_have_no_continuations(ex):  # noqa: F811
    n, K, steps, V, H = 6, 4, 9, 500, 130
    body = ex.Body(V, H, seed=1)
    W = torch.randn(V, H, generator=torch.Generator("cuda").manual_seed(2), device="cuda") * (4 / H ** 0.5)
    head = ex.B.BlockHead(W)
    first = torch.arange(1, n + 1, dtype=torch.int32, device="cuda")
    clean, _ = ex.decode(body, head, first, K, steps)
    lost = next(t for t in range(n) if not (clean == t + 1).any())   # its first token leads no other sequence astray
    others = [t for t in range(n) if t != lost]
    body.E[lost + 1] = torch.nan
    tokens, length = ex.decode(body, head, first, K, steps)
    assert length[lost] == 0 and torch.all(tokens[lost] == ex.END)
    assert torch.all(length[others] > 0) and torch.all(tokens[others][:, 0] > 0)
    student = ex.Student(V, H, seed=4)
    loss, _, grad = student.gradients(first, tokens, length)          # the lost sequence takes no part
    assert torch.isfinite(loss) and all(torch.isfinite(g).all() for g in grad.values())
    assert torch.all(grad["dh"].view(n, steps, H)[lost] == 0)
