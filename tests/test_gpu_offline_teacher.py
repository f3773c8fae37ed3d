"""The example's path, teacher's head in 8-bit integers to the student's gradients, against the same in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("offline_teacher", os.path.join(ROOT, "examples", "offline_teacher.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _inputs(V=3001, H=192, T=70):
    g = torch.Generator().manual_seed(1)
    h_t, W_t = torch.randn(T, 2 * H, generator=g).bfloat16(), (torch.randn(V, 2 * H, generator=g) * 0.08).bfloat16()
    h_s, W_s = torch.randn(T, H, generator=g).bfloat16(), (torch.randn(V, H, generator=g) * 0.1).bfloat16()
    ids = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    return h_t, W_t, h_s, W_s, ids


def _quantised(x):
    a = x.double().abs().amax(dim=1, keepdim=True)
    return torch.round(x.double() * 127 / a), a / 127


def test_teacher_answers(example):
    h_t, W_t, _, _, ids = _inputs()
    offsets, window = np.array([0, 30, 70]), np.array([20, 64])
    ids = example.admitted_ids(ids.cuda(), offsets, window)
    assert int((ids < 0).sum()) == 10
    got = example.teacher_answers(example.B.QuantHead(W_t.cuda()), h_t.cuda(), ids, top=6, slab=32)
    (qh, sh), (qW, sW) = _quantised(h_t), _quantised(W_t)
    z = (qh @ qW.t()) * sh * sW[:, 0]
    z = z.float().bfloat16()              # the logits are kept in bf16; a border case may fall to the other side
    lp = torch.log_softmax(z.double(), dim=1)
    scored = ids.cpu() >= 0
    want = torch.where(scored, lp.gather(1, ids.cpu().clamp(min=0).long()[:, None])[:, 0], 0.)
    step = z.float().abs().max() * 2.0 ** -7
    assert torch.all((got["logp"].cpu().double() - want).abs() <= step + 1e-4)
    assert torch.all(got["top_ids"][~scored.cuda()] == -1) and torch.all(got["top_logp"][~scored.cuda()] == 0)
    top = torch.topk(lp, 6, dim=1).values
    assert torch.all((got["top_logp"].cpu().double() - top)[scored].abs() <= step + 1e-4)


def test_student_step(example):
    h_t, W_t, h_s, W_s, ids = _inputs()
    ids[3] = -1
    answers = example.teacher_answers(example.B.QuantHead(W_t.cuda()), h_t.cuda(), ids.cuda(), top=12)
    loss, dh, dW = example.student_step(h_s.cuda(), W_s.cuda(), answers, bonus=0.05)
    # the same from the logits that the step saw, in 64 bits
    z = (h_s.cuda() @ W_s.cuda().t()).cpu().double().requires_grad_()
    at, t = answers["top_ids"].cpu(), answers["top_logp"].cpu().double()
    scored = at[:, 0] >= 0
    lp = torch.log_softmax(z, dim=1)
    q = lp.gather(1, at.clamp(min=0).long())
    rows = (t.exp() * (t - q)).sum(1) + 0.05 * (lp.exp() * lp).sum(1)
    want = rows[scored].mean()
    want.backward()
    assert abs(float(loss) - float(want.detach())) <= 1e-5 * (1 + abs(float(want.detach())))
    dz = z.grad
    assert torch.all(dz[3] == 0)
    # dz is rounded to bf16 (half a step, 2^-8), the products sum it in fp32 and round once more
    for got, w, size in ((dh, dz @ W_s.double(), dz.abs() @ W_s.double().abs()), (dW, dz.t() @ h_s.double(), dz.t().abs() @ h_s.double().abs())):
        assert torch.all((got.cpu().double() - w).abs() <= 1.01 * 2.0 ** -8 * (size + w.abs()) + 1e-9)


def test_loss_falls(example):
    h_t, W_t, h_s, W_s, ids = (x.cuda() for x in _inputs())
    answers = example.teacher_answers(example.B.QuantHead(W_t), h_t, ids)
    weights, losses = W_s.float(), []
    for _ in range(8):
        loss, _, dW = example.student_step(h_s, weights.bfloat16(), answers)
        losses.append(float(loss))
        weights -= 0.5 * dW.float()
    assert losses[-1] < losses[0]
