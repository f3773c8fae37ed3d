"""Scoring given tokens: a head kept in 8-bit integers, log-probabilities of given tokens, and their gradient.

Every case is a plain dict; `op` says which operator it takes.

* quant_rows      -- bf16 or fp32 rows to 8-bit integers with one scale per row: what lays a head out, and what a
  product does to its tokens.
* quant_logits    -- hidden states times a head that is kept in 8-bit integers, with a scale per token and one per
  vocabulary entry, to logits in bf16 or fp32.
* token_logp      -- logits in, log-probabilities of `given` tokens per row, entropy and the `top` most likely tokens
  with theirs out.
* token_logp_grad -- what the loss says of those log-probabilities and entropies, back to the logits.

Rows outside the windows carry negative ids: they are not scored and get a zero gradient.
"""
from __future__ import annotations

import math

import torch

own = False                 # True: the framework's calls, False: the same in elementary operations

V_FULL = 151936             # vocabulary of the benchmark configurations
PAD = 128                   # the contraction of the 8-bit product goes over whole lines of memory


def _rows(name, T, H, dtype):
    return {"name": name, "op": "quant_rows", "T": T, "H": H, "dtype": dtype}


def _product(name, T, V, H, dtype, out):
    return {"name": name, "op": "quant_logits", "T": T, "V": V, "H": H, "dtype": dtype, "out": out}


def _logp(name, T, V, dtype, given, top, temperature=1.0, unscored=0, masked=0):
    return {"name": name, "op": "token_logp", "T": T, "V": V, "dtype": dtype, "given": given, "top": top,
            "temperature": temperature, "unscored": unscored, "masked": masked}


def _grad(name, T, V, dtype, given, entropy, out, temperature=1.0, unscored=0, masked=0):
    return {"name": name, "op": "token_logp_grad", "T": T, "V": V, "dtype": dtype, "given": given, "entropy": entropy,
            "out": out, "temperature": temperature, "unscored": unscored, "masked": masked}


def listed():
    return [
        # the hidden states of a few running rollouts, one new token each
        _rows("rows_decode", 64, 4096, "bf16"),
        # the student's head, laid out anew after every optimizer step
        _rows("rows_head", V_FULL, 2048, "bf16"),
        # the teacher scores one token as it arrives: every weight is read for one row
        _product("product_one_token", 1, V_FULL, 4096, "bf16", "bf16"),
        # one new token of each rollout of a batch
        _product("product_decode", 48, V_FULL, 2048, "bf16", "fp32"),
        # a test-sized head with an odd vocabulary and a hidden size that is no multiple of a tile
        _product("product_ragged", 701, 11907, 632, "fp32", "fp32"),
        # a slab of whole rollouts through the teacher's head
        _product("product_rollouts", 4096, V_FULL, 4096, "bf16", "bf16"),
        # serving: the sampled token of one step with its alternatives
        _logp("logp_one_token", 1, V_FULL, "bf16", 1, 20),
        # odd vocabulary, part of it masked out, at a sampling temperature
        _logp("logp_masked", 777, 32771, "fp32", 4, 64, temperature=0.7, unscored=100, masked=5000),
        # whole rollouts: the sampled token and the alternatives that the student is later held to
        _logp("logp_rollouts", 8192, V_FULL, "bf16", 1, 20, unscored=512),
        # a debugging run's batch: latency
        _grad("grad_small", 37, V_FULL, "bf16", 1, False, "bf16", unscored=8),
        # odd vocabulary with masked entries, entropy bonus, gradient in 32 bits
        _grad("grad_masked", 777, 32771, "fp32", 4, True, "fp32", temperature=0.7, unscored=100, masked=5000),
        # the student's logits at the teacher's alternatives, with an entropy bonus
        _grad("grad_rollouts", 8192, V_FULL, "bf16", 20, True, "bf16", unscored=1024),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    op = ("quant_rows", "quant_logits", "token_logp", "token_logp_grad")[rng.randrange(4)]
    types = ("bf16", "bf16", "fp32")
    dtype, out = types[rng.randrange(3)], types[rng.randrange(3)]
    V = V_FULL if rng.random() < 0.4 else log(300, V_FULL)
    if op == "quant_rows":
        H = 128 * rng.randint(1, 32) if rng.random() < 0.5 else log(64, 4096)
        case = _rows("", log(1, min(V_FULL, (V_FULL * 2048 * 2) // (H * (4 if dtype == "fp32" else 2)))), H, dtype)
    elif op == "quant_logits":
        H = 128 * rng.randint(1, 32) if rng.random() < 0.5 else log(64, 4096)
        case = _product("", log(1, min(4096, (4096 * V_FULL) // (V * (2 if out == "fp32" else 1)))), V, H, dtype, out)
    else:
        wide = 2 if dtype == "fp32" or (op == "token_logp_grad" and out == "fp32") else 1
        T = log(1, min(8192, (8192 * V_FULL) // (V * wide)))
        given = (1, 1, 2, 7, 20, 64)[rng.randrange(6)]
        temperature = 1.0 if rng.random() < 0.6 else round(rng.uniform(0.4, 1.6), 2)
        unscored = 0 if rng.random() < 0.4 else rng.randrange(max(1, T // 3))
        masked = 0 if rng.random() < 0.7 else rng.randrange(V // 4)
        if op == "token_logp":
            top = (0, 1, 5, 20, 20, 64)[rng.randrange(6)]
            case = _logp("", T, V, dtype, given, top, temperature, unscored, masked)
        else:
            case = _grad("", T, V, dtype, given, rng.random() < 0.5, out, temperature, unscored, masked)
    return {k: v for k, v in case.items() if k != "name"}


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _generator(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _quantised(x):
    """Rows x as (integers, scale): scale = largest magnitude / 127, integers to the nearest, ties to even."""
    wide = x.float() if x.dtype == torch.bfloat16 else x.double()    # a quotient next to a half needs its bits
    most = wide.abs().amax(dim=1, keepdim=True)
    q = torch.where(most > 0, torch.round(wide * 127 / torch.where(most > 0, most, 1)), 0)
    return q, (most.float() / 127).squeeze(1)


def _logits(T, V, dtype, masked, g):
    """Logits like a trained policy's: a spread of a few nats, a handful of likely tokens in every row."""
    z = torch.empty(T, V, dtype=dtype, device="cuda")
    step = max(1, (1 << 28) // V)
    for lo in range(0, T, step):
        n = min(step, T - lo)
        z[lo:lo + n] = torch.randn(n, V, generator=g, device="cuda") * 1.8
    likely = torch.randint(0, V, (T, 8), generator=g, device="cuda")
    high = (0.3 + 0.9 * torch.rand(T, 8, generator=g, device="cuda")) * (math.log(V) + 2)
    z.scatter_(1, likely, high.to(dtype))
    if masked:                                    # the same entries in every row: what a grammar or a tokenizer rules out
        z[:, torch.randperm(V, generator=g, device="cuda")[:masked]] = -math.inf
    return z, likely


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["op"] == "quant_rows":
        x = torch.randn(case["T"], case["H"], generator=g, device="cuda")
        s["x"] = (x * (0.3 + torch.rand(case["T"], 1, generator=g, device="cuda"))).to(_type(case["dtype"]))
        return s
    if case["op"] == "quant_logits":
        T, V, H = case["T"], case["V"], case["H"]
        s["h"] = torch.randn(T, H, generator=g, device="cuda").to(_type(case["dtype"]))
        W = (torch.randn(V, H, generator=g, device="cuda") * 0.02).to(torch.bfloat16)
        q, s["W_scale"] = _quantised(W)           # the head as it is kept: integers padded with zeros to whole lines
        s["W_q"] = torch.zeros(V, (H + PAD - 1) // PAD * PAD, dtype=torch.int8, device="cuda")
        s["W_q"][:, :H] = q.to(torch.int8)
        return s
    T, V, G = case["T"], case["V"], case["given"]
    s["z"], likely = _logits(T, V, _type(case["dtype"]), case["masked"], g)
    ids = torch.randint(0, V, (T, G), generator=g, device="cuda", dtype=torch.int32)
    n = min(4, G)
    ids[:, :n] = likely[:, :n].to(torch.int32)    # sampled tokens are mostly likely ones
    if case["masked"]:                            # and never ruled out
        free = torch.nonzero(torch.isfinite(s["z"][0])).squeeze(1).to(torch.int32)
        ids = free[ids.long() % free.numel()].contiguous()
    if case["unscored"]:
        ids[torch.randperm(T, generator=g, device="cuda")[:case["unscored"]]] = -1
    s["ids"] = ids
    if case["op"] == "token_logp_grad":
        first = _logp_plain(s["z"], ids, case["temperature"], 0)
        s["norm"], s["entropy"] = first["norm"], first["entropy"]
        s["g_logp"] = torch.randn(T, G, generator=g, device="cuda") / T
        s["g_entropy"] = torch.rand(T, generator=g, device="cuda") * (0.1 / T) if case["entropy"] else None
    return s


def _logp_plain(z, ids, temperature, top):
    scored = (ids >= 0).any(dim=1)
    x = z.float()
    most = x.amax(dim=1)
    x = (x - most[:, None]) / temperature
    e = torch.exp(x)
    total = e.sum(dim=1)
    log_total = torch.log(total)
    entropy = log_total - torch.where(e > 0, e * x, 0).sum(dim=1) / total
    logp = torch.gather(x, 1, ids.clamp(min=0).long()) - log_total[:, None]
    out = {"logp": torch.where(ids >= 0, logp, 0), "entropy": torch.where(scored, entropy, 0),
           "norm": torch.where(scored[:, None], torch.stack([most, total], dim=1), 0)}
    if top:
        # one key per logit, larger for the larger logit and then for the lower index
        bits = z.float().view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() * (1 << 32)
        key += (1 << 31) - 1 - torch.arange(z.shape[1], device=z.device)
        at = torch.topk(key, min(top, z.shape[1]), dim=1).values
        at = ((1 << 31) - 1 - (at & 0xffffffff)).long()
        out["top_ids"] = torch.where(scored[:, None], at, -1).to(torch.int32)
        out["top_logp"] = torch.where(scored[:, None], torch.gather(x, 1, at) - log_total[:, None], 0)
    return out


def _grad_plain(s, case):
    x = (s["z"].float() - s["norm"][:, :1]) / case["temperature"]
    total = s["norm"][:, 1:]
    scored = (s["ids"] >= 0).any(dim=1, keepdim=True)
    total = torch.where(scored, total, 1)
    p = torch.exp(x) / total
    g = torch.where(s["ids"] >= 0, s["g_logp"], 0)
    dz = -p * g.sum(dim=1, keepdim=True)
    if s["g_entropy"] is not None:
        lp = torch.where(p > 0, x - torch.log(total), 0)
        dz -= s["g_entropy"][:, None] * p * (lp + s["entropy"][:, None])
    dz.scatter_add_(1, s["ids"].clamp(min=0).long(), g)
    return torch.where(scored, dz / case["temperature"], 0).to(_type(case["out"]))


def run(state):
    case = state["case"]
    if own:
        from paper_2605_28396_amd import binding as B
        if case["op"] == "quant_rows":
            out = B.adwin_opd_quant_rows(state["x"])
            return {"values": out["q"][:, :case["H"]] * out["scale"][:, None], "scale": out["scale"]}
        dt = B.ADWIN_DT_BF16 if case.get("out") == "bf16" else B.ADWIN_DT_F32
        if case["op"] == "quant_logits":
            return {"z": B.adwin_opd_quant_logits(state["h"], state["W_q"], state["W_scale"], z_dtype=dt)["z"]}
        if case["op"] == "token_logp":
            out = B.adwin_opd_token_logp(state["z"], state["ids"], temperature=case["temperature"], top=case["top"])
            return {k: out[k] for k in ("logp", "entropy", "norm") + (("top_ids", "top_logp") if case["top"] else ())}
        return {"dz": B.adwin_opd_token_logp_grad(
            state["z"], state["ids"], state["norm"], state["g_logp"], entropy=state["entropy"],
            g_entropy=state["g_entropy"], temperature=case["temperature"], dz_dtype=dt)["dz"]}
    if case["op"] == "quant_rows":
        q, scale = _quantised(state["x"])
        return {"values": q.float() * scale[:, None], "scale": scale}
    if case["op"] == "quant_logits":
        q, scale = _quantised(state["h"])
        z = torch.matmul(q.float(), state["W_q"][:, :case["H"]].float().t())
        return {"z": (z * scale[:, None] * state["W_scale"]).to(_type(case["out"]))}
    if case["op"] == "token_logp":
        return _logp_plain(state["z"], state["ids"], case["temperature"], case["top"])
    return {"dz": _grad_plain(state, case)}


def work(case):
    size = {"bf16": 2, "fp32": 4}
    T = case["T"]
    if case["op"] == "quant_rows":                # integers and scales out
        return {"bytes": T * case["H"] * (size[case["dtype"]] + 1) + 4 * T, "flops": 3 * T * case["H"]}
    V = case["V"]
    if case["op"] == "quant_logits":
        H = case["H"]
        return {"bytes": T * H * size[case["dtype"]] + V * (H + 4) + T * V * size[case["out"]], "flops": 2 * T * V * H}
    G, live = case["given"], T - case["unscored"]
    if case["op"] == "token_logp":
        return {"bytes": live * V * size[case["dtype"]] + T * (8 * G + 12 + 8 * case["top"]), "flops": 6 * live * V}
    return {"bytes": live * V * size[case["dtype"]] + T * V * size[case["out"]] + T * (8 * G + 16), "flops": 6 * live * V}


def exact(case, seed):
    """What run() returns, by the definitions in 64 bits."""
    s = prepare(case, seed)
    if case["op"] in ("quant_rows", "quant_logits"):
        x = (s["x"] if case["op"] == "quant_rows" else s["h"]).double()
        top = x.abs().max(dim=1, keepdim=True).values
        step = top / 127.0
        q = (x * 127.0 / top.clamp(min=1e-300)).round()
        if case["op"] == "quant_rows":
            return {"values": q * step, "scale": step[:, 0]}
        z = torch.empty(case["T"], case["V"], dtype=torch.float64, device="cuda")
        for lo in range(0, case["V"], 16384):
            w = s["W_q"][lo:lo + 16384, :case["H"]].double().mul_(s["W_scale"][lo:lo + 16384, None].double())
            z[:, lo:lo + 16384] = (q * step) @ w.t()
        return {"z": z}
    T, V, G = case["T"], case["V"], case["given"]
    rows = max(1, (1 << 26) // V)
    parts = []
    for lo in range(0, T, rows):
        ids = s["ids"][lo:lo + rows].long()
        raw = s["z"][lo:lo + rows]
        live = ids.max(dim=1).values >= 0
        lp = torch.log_softmax(raw.double() / case["temperature"], dim=1)
        p = lp.exp()
        plp = torch.nan_to_num(p * lp, nan=0.0)
        zero = torch.zeros((), dtype=torch.float64, device="cuda")
        if case["op"] == "token_logp":
            peak = raw.double().max(dim=1).values
            part = {"logp": torch.where(ids >= 0, lp.gather(1, ids.clamp(min=0)), zero),
                    "entropy": torch.where(live, -plp.sum(dim=1), zero),
                    "norm": torch.where(live[:, None], torch.stack(
                        [peak, ((raw.double() - peak[:, None]) / case["temperature"]).exp().sum(dim=1)], 1), zero)}
            if case["top"]:
                at = torch.sort(raw.float(), dim=1, descending=True, stable=True).indices[:, :case["top"]]
                part["top_ids"] = torch.where(live[:, None], at, -1).to(torch.int32)
                part["top_logp"] = torch.where(live[:, None], lp.gather(1, at), zero)
        else:
            gl = torch.where(ids >= 0, s["g_logp"][lo:lo + rows].double(), zero)
            dz = torch.zeros_like(lp).scatter_add_(1, ids.clamp(min=0), gl) - p * gl.sum(dim=1, keepdim=True)
            if s["g_entropy"] is not None:
                # H = -sum p log p:  dH/dz_j = -p_j (log p_j + H)
                dz += s["g_entropy"][lo:lo + rows, None].double() * (p * plp.sum(dim=1, keepdim=True) - plp)
            part = {"dz": torch.where(live[:, None], dz / case["temperature"], zero)}
        parts.append(part)
    return {k: torch.cat([q[k] for q in parts]) for k in parts[0]}
