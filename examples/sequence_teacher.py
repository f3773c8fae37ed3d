"""Distillation from sequences: a teacher, its head in 8-bit floats, writes target sequences by beams; the student learns them through
a head in 8-bit floats of its own.

Decoding: logits of every beam (BlockHead), the best continuations of each sequence (adwin_opd_beam_select), tokens and states moved to
where these are (adwin_opd_beam_reorder).  Training: logits, log-probabilities of the targets and their gradient by the logits
(adwin_opd_token_logp, adwin_opd_token_logp_grad), and on to hidden states and weights (BlockHead.grad); the bodies are a few lines
of torch.

    python examples/sequence_teacher.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_28396_amd import binding as B  # noqa: E402

END = 0


class Body:
    """A recurrent body: the hidden state of a context is the last one, turned, plus the last token's embedding."""

    def __init__(self, V, H, seed, device="cuda"):
        g = torch.Generator(device).manual_seed(seed)
        self.E = torch.randn(V, H, generator=g, device=device)
        self.R = torch.randn(H, H, generator=g, device=device) / H ** 0.5

    def step(self, state, token):
        return torch.tanh(state @ self.R + self.E[token.long()])


def decode(body, head, first, beams, steps, length_power=0.6):
    """Sequences of `steps` tokens at most behind the tokens first [n]: the best of each by its score a token^length_power, tokens
    [n, steps] and lengths [n] (behind the end: END; 0 where none of its beams could go on)."""
    n, dev = first.shape[0], first.device
    state = body.step(torch.zeros(n * beams, head.H, device=dev), first.repeat_interleave(beams))
    tokens = torch.full((n * beams, steps), END, dtype=torch.int32, device=dev)
    score = torch.full((n, beams), -torch.inf, device=dev)
    score[:, 0] = 0                                       # the others are copies of the first until they have gone on
    finished = length = torch.zeros(n, beams, dtype=torch.int32, device=dev)
    carried = B.BeamStates([state, tokens], beams)        # in place: rows that stay are not touched
    for t in range(steps):
        z, status = head.logits(state, row_status=True)
        # a state that holds an inf or NaN has no logits, and its beam no continuations
        score = score.masked_fill((status.view(n, beams) != 0) & (finished == 0), -torch.inf)
        best = B.adwin_opd_beam_select(z, score, beams, finished=finished, length=length, end=END, length_power=length_power)
        score, finished, length = best["score"], best["finished"], best["length"]
        carried.reorder(best["parent"])
        token = best["token"].clamp(min=END).view(-1)     # -1: fewer continuations than beams; their score is -inf
        tokens[:, t] = token
        state.copy_(body.step(state, token))
    return tokens.view(n, beams, steps)[:, 0], length[:, 0]


class Student:
    def __init__(self, V, H, seed, device="cuda"):
        self.body = Body(V, H, seed, device)
        g = torch.Generator(device).manual_seed(seed + 1)
        self.W = torch.randn(V, H, generator=g, device=device) / H ** 0.5
        self.head = B.BlockHead(self.W, gradients=True)
        self.parameters = [self.body.E.requires_grad_(), self.body.R.requires_grad_()]

    def hidden(self, first, targets):
        """Hidden states of the contexts of every target, [n steps, H]."""
        state = torch.zeros(first.shape[0], self.W.shape[1], device=first.device)
        rows, token = [], first
        for t in range(targets.shape[1]):
            state = self.body.step(state, token)
            rows.append(state)
            token = targets[:, t]
        return torch.stack(rows, dim=1).flatten(0, 1)

    def gradients(self, first, targets, length):
        """Mean negative log-probability of the targets, hidden states, and the gradients by these and the head."""
        n, steps = targets.shape
        h = self.hidden(first, targets)
        z, status = self.head.logits(h.detach(), z_dtype=B.ADWIN_DT_F32, row_status=True)
        inside = torch.arange(steps, device=first.device)[None] < length[:, None]
        ids = torch.where(inside.flatten() & (status == 0), targets.flatten(), -1).to(torch.int32)
        scored = (ids >= 0).sum().clamp(min=1)
        out = B.adwin_opd_token_logp(z, ids)
        g = (-1.0 / scored).expand(n * steps).contiguous()
        dz = B.adwin_opd_token_logp_grad(z, ids, out["norm"], g)["dz"]
        return -out["logp"].sum() / scored, h, self.head.grad(dz, h.detach(), dh_dtype=B.ADWIN_DT_F32, status=status)

    def train_step(self, first, targets, length, lr):
        loss, h, grad = self.gradients(first, targets, length)
        h.backward(grad["dh"])
        with torch.no_grad():
            for p in self.parameters:
                p -= lr * p.grad
                p.grad = None
            self.W -= lr * grad["dW"]
        self.head.set(self.W)                             # laid out again, in the same arrays
        return loss


def main(n=64, beams=4, steps=24, V=2000, H=256, epochs=20):
    teacher = Body(V, H, seed=1)
    W = torch.randn(V, H, generator=torch.Generator("cuda").manual_seed(2), device="cuda") * (4 / H ** 0.5)
    first = torch.randint(1, V, (n,), generator=torch.Generator("cuda").manual_seed(3), device="cuda", dtype=torch.int32)
    targets, length = decode(teacher, B.BlockHead(W), first, beams, steps)
    student = Student(V, H, seed=4)
    for epoch in range(epochs):
        loss = student.train_step(first, targets, length, lr=20.0)
        if epoch % 5 == 0 or epoch == epochs - 1:
            print(f"epoch {epoch:3d}  negative log-probability of the teacher's tokens {loss.item():.4f}", flush=True)


if __name__ == "__main__":
    main()
