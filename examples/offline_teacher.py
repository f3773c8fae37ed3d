"""Distillation from a teacher whose answers are kept, not its logits.

The teacher's head is laid out once in 8-bit integers.  A pass over finished rollouts turns its hidden states, a
slab of rows at a time, into what training needs of it: the log-probability of every sampled token and the `top`
alternatives with theirs, some hundred bytes a row in place of 300 KB of logits.  A training step then evaluates the
student at these tokens alone.  With q_k and t_k the student's and the kept teacher's log-probabilities of a row's
alternatives, its loss is the teacher's cross-entropy on them, over its least value, less an entropy bonus,

    sum_k e^{t_k} (t_k - q_k) - bonus H,

whose derivatives by q and H go back through adwin_opd_token_logp_grad to the student's logits, and from there to its
hidden states and head.  Rows outside the windows carry the id -1: they are not scored and get no gradient.  So do rows
whose hidden states hold an inf or NaN, the teacher's or the student's.

    python examples/offline_teacher.py [--rollouts 8] [--length 512] [--vocab 32000] [--steps 20]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_28396_amd import binding as B  # noqa: E402


def admitted_ids(ids, offsets, window):
    """ids with -1 on the rows outside the windows."""
    n = B.adwin_opd_plan_host(offsets, window)["n"]
    out = torch.full_like(ids, -1)
    for lo, k in zip(offsets[:-1], n):
        out[lo:lo + k] = ids[lo:lo + k]
    return out


def teacher_answers(head: B.QuantHead, h_t, ids, top=20, slab=2048):
    """What training needs of the teacher: `logp` [T] of the sampled tokens, `top_ids` and `top_logp` [T, top]."""
    if bool((head.row_status != 0).any()):
        raise ValueError(f"weights of {int((head.row_status != 0).sum())} entries of the teacher's head hold an inf or NaN")
    T, V = h_t.shape[0], head.W_q.shape[0]
    z = torch.empty(min(slab, T), (V + 7) & ~7, dtype=torch.bfloat16, device=h_t.device)[:, :V]
    parts = []
    for lo in range(0, T, slab):
        rows = slice(lo, min(lo + slab, T))
        here = z[:rows.stop - lo]
        _, status = head.logits(h_t[rows], z=here, row_status=True)
        parts.append(B.adwin_opd_token_logp(here, torch.where(status == 0, ids[rows], -1), top=top))
    return {k: torch.cat([p[k] for p in parts]) for k in ("logp", "top_ids", "top_logp")}


def student_step(h_s, W_s, answers, bonus=0.0):
    """Loss per scored row and its gradients by the student's hidden states and head."""
    z = h_s @ W_s.t()
    ids, t = answers["top_ids"], answers["top_logp"]
    out = B.adwin_opd_token_logp(z, ids)
    scored = (ids >= 0) & (out["norm"][:, 1:] > 0)          # norm is 0, 0 where the student's logits are not finite
    count = scored.any(dim=1).sum().clamp(min=1)
    p_t = torch.where(scored, t.exp(), 0.)
    loss = ((p_t * (t - out["logp"])).sum() - bonus * out["entropy"].sum()) / count
    g_logp = -p_t / count
    g_entropy = torch.full_like(out["entropy"], -bonus) / count
    # z is not needed any more: its gradient takes its place
    dz = B.adwin_opd_token_logp_grad(z, ids, out["norm"], g_logp, entropy=out["entropy"], g_entropy=g_entropy, dz=z)["dz"]
    return loss, dz @ W_s, dz.t() @ h_s.masked_fill(~scored.any(dim=1, keepdim=True), 0)      # 0 times NaN is none


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rollouts", type=int, default=8)
    ap.add_argument("--length", type=int, default=512)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    g = torch.Generator("cuda").manual_seed(0)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(torch.bfloat16)

    lengths = np.random.default_rng(0).integers(a.length // 2, a.length, size=a.rollouts, endpoint=True)
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    window = lengths * 3 // 4
    T = int(offsets[-1])
    h_t, W_t = normal(T, 2 * a.hidden), normal(a.vocab, 2 * a.hidden, scale=0.05)
    h_s, W_s = normal(T, a.hidden), normal(a.vocab, a.hidden, scale=0.05)
    ids = torch.randint(0, a.vocab, (T,), generator=g, device="cuda", dtype=torch.int32)
    ids = admitted_ids(ids, offsets, window)

    answers = teacher_answers(B.QuantHead(W_t), h_t, ids)
    weights = W_s.float()
    for step in range(a.steps):
        loss, _, dW = student_step(h_s, weights.to(torch.bfloat16), answers, bonus=0.01)
        weights -= 100.0 * dW.float()
        if step % 5 == 0 or step + 1 == a.steps:
            print(f"step {step}: loss {float(loss):.4f}", flush=True)


if __name__ == "__main__":
    main()
