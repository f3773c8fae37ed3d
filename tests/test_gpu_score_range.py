"""The token-scoring operators at the ends of their ranges: masks of large finite values, logits and temperatures whose quotient passes
what fp32 counts one by one, scales and derivatives near the ends of the type.  References and tolerances are those of
test_gpu_score.py, in 64 bits."""
import math

import pytest
import torch

from . import test_gpu_score as S

pytestmark = pytest.mark.gpu
U = S.U


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2605_28396_amd import binding
    return binding


def _f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def _check_logp(B, out, z, ids, tau, top):
    """Against the reference in 64 bits, with the tolerances that test_gpu_score.py derives: u S of the sum and 2 u |log p| of a
    log-probability of any size (S._check_logp counts that part up to 1e30)."""
    V, ref = z.shape[1], S._reference(z, ids, tau, top)
    n = math.ceil(V / 256) + 8 + 36 + 2 * (math.log(V) + 1)
    tol = {k: U * (n + 2 * ref["log_s"].abs()[:, None] + 2 * torch.where(torch.isinf(ref[k]), 0., ref[k]).abs()) for k in ("logp", "top_logp")}
    tol["entropy"], tol["norm"] = U * n * (2 + 2 * ref["mean"]), U * n * ref["norm"] * torch.tensor([0., 1.])
    for k, t in tol.items():
        got, want = out[k].double().cpu(), ref[k]
        off = torch.where(torch.isinf(want) & (got == want), 0., (got - want).abs())
        assert torch.all(off <= t), (k, float((off - t).max()))
    assert torch.equal(out["top_ids"].cpu(), ref["top_ids"])


MASKS = [-1e6, -1e7, -1e9, -5e9, -1e10, -1e12, -1e20, -1e30, -1e32, -1e37]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(8, 300), (8, 9001), (1, 70001), (264, 9001)])
@pytest.mark.parametrize("tau", [1.0, 0.5, 0.7])
def test_finite_masks(B, dtype, T, V, tau):
    """Most entries at a mask's value, whole blocks of a row, all but one, and rows of nothing else: one piece and several."""
    rows = []
    for k, mask in enumerate(MASKS):
        z = S._logits(4, V, dtype, 20 + k)
        keep = torch.randperm(V, generator=S._gen(V, k))[:max(1, V // 50)]
        z[0] = torch.full((V,), mask, dtype=dtype).index_copy(0, keep, z[0, keep])
        z[1, V // 8:V - V // 4] = mask
        z[2, :V - 1] = mask
        z[3] = mask
        rows.append(z)
    rows = torch.cat(rows)
    tau = _f32(tau)
    rows = rows.repeat((max(T, len(rows)) + len(rows) - 1) // len(rows), 1)
    ids = S._ids(len(rows), 3, V, 7)
    ids[2, 0] = V - 1
    for at in range(0, len(rows) - T + 1, T):
        z, i = rows[at:at + T], ids[at:at + T]
        out = B.adwin_opd_token_logp(z.cuda(), i.cuda(), temperature=tau, top=9, row_status=True)
        assert torch.all(out["row_status"] == 0)
        _check_logp(B, out, z, i, tau, 9)
        if V > 20000 and at % 5:
            continue                                               # the gradient is one kernel for all of these
        gl, gh = torch.randn(T, 3, generator=S._gen(at)), torch.randn(T, generator=S._gen(at, 1))
        dz = B.adwin_opd_token_logp_grad(z.cuda(), i.cuda(), out["norm"], gl.cuda(), entropy=out["entropy"], g_entropy=gh.cuda(),
                                         temperature=tau, dz_dtype=B.ADWIN_DT_F32)["dz"].cpu()
        want, tol = S._grad_reference(z, i, out["norm"].cpu(), out["entropy"].cpu(), gl, gh, tau)
        assert torch.all((dz.double() - want).abs() <= tol + U * want.abs() * 1.001)
        assert torch.all((dz != 0).any(dim=1))


@pytest.mark.parametrize("T,V", [(3, 500), (2, 20001), (300, 3000)])
@pytest.mark.parametrize("at,spread,tau", [(0.0, 20.0, 1e-6), (0.0, 20.0, 1e-8), (100.0, 1.0, 1e-8), (0.0, 3.0, 1e-20), (1e6, 10.0, 1.0),
                                           (3e7, 40.0, 1.0), (3e9, 1e3, 1.0), (-3e9, 1e3, 1.0), (-1e30, 0.0, 1.0), (1e30, 1e24, 1.0), (5.0, 3.0, 1e30)])
def test_far_logits_and_temperatures(B, T, V, at, spread, tau):
    """Logits whose quotient by the temperature is far from 0 on either side, with their differences small or large."""
    z = torch.randn(T, V, generator=S._gen(T, V), dtype=torch.float64).mul_(spread).add_(at).float()
    tau = _f32(tau)
    ids = S._ids(T, 2, V, 3)
    ids[:, 1] = z.argmax(dim=1).int()
    out = B.adwin_opd_token_logp(z.cuda(), ids.cuda(), temperature=tau, top=5, row_status=True)
    assert torch.all(out["row_status"] == 0)
    _check_logp(B, out, z, ids, tau, 5)


# few tokens, the tiles of 128 entries, those of 256
@pytest.mark.parametrize("T,V,H", [(3, 500, 300), (40, 1000, 256), (100, 3001, 512), (300, 9001, 384), (1100, 33001, 1500)])
@pytest.mark.parametrize("z_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("token,entry", [(1e-20, 1e-20), (1e-30, 1e-7), (1e22, 1e22), (1e35, 1e-30), (1e-30, 1e35)])
def test_product_of_far_scales(B, T, V, H, z_dtype, token, entry):
    """Scales whose product leaves fp32, or all but does, with logits inside it, zero sums and logits beyond it: tokens and entries of
    such magnitudes among ordinary ones."""
    g = torch.Generator("cuda").manual_seed(T)
    h = torch.randn(T, H, generator=g, device="cuda")
    W = torch.randn(V, H, generator=g, device="cuda") * 0.05
    h[::2] *= token
    W[::3] *= entry
    h[0, :] = 0
    h[0, H // 2:] = token                                          # times an entry with zeros there: a sum of 0
    W[3, H // 2:] = 0
    W[6] = 0
    (qh, sh, _), (qW, sW, _) = S._quantised(h.cpu()), S._quantised(W.cpu())
    got = B.QuantHead(W).logits(h, z_dtype=B._DTYPE[z_dtype])
    least = 2.0 ** -149 if z_dtype == torch.float32 else 2.0 ** -133
    qh, sh, qW, sW = (x.cuda().double() for x in (qh, sh, qW, sW))
    for lo in range(0, V, 16384):
        want = (qh @ qW[lo:lo + 16384].t().contiguous()) * sh[:, None] * sW[lo:lo + 16384]
        beyond = want.abs() * (1 + 2.0 ** -7) > torch.finfo(z_dtype).max
        tol = want.abs() * (3.01 * U + (torch.finfo(z_dtype).eps / 2 if z_dtype != torch.float32 else 0)) + 2 * least
        z = got[:, lo:lo + 16384].double()
        assert torch.all(((z - want).abs() <= tol) | beyond) and not torch.any(torch.isnan(z))
        assert torch.all(z[beyond].abs() >= torch.finfo(z_dtype).max * (1 - 2.0 ** -6))
    assert torch.all(got[0, 3] == 0) and torch.all(got[:, 6] == 0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(4, 700), (3, 30001)])
def test_large_derivatives_of_masked_rows(B, dtype, T, V):
    """Derivatives by the entropy as a scaled loss has them: a masked entry's gradient is 0, not 0 times inf."""
    z, ids = S._logits(T, V, dtype, 1), S._ids(T, 2, V, 2)
    z[:, V // 2:] = -math.inf
    z[1, :V // 2 - 1] = torch.finfo(dtype).min
    z[2, ::3] = -1e10
    f = B.adwin_opd_token_logp(z.cuda(), ids.cuda())
    for size in (1.0, 1e9, 1e20, 1e33):
        gl, gh = torch.randn(T, 2, generator=S._gen(T)) * size, torch.randn(T, generator=S._gen(V)) * size
        dz = B.adwin_opd_token_logp_grad(z.cuda(), ids.cuda(), f["norm"], gl.cuda(), entropy=f["entropy"], g_entropy=gh.cuda(),
                                         dz_dtype=B.ADWIN_DT_F32)["dz"].cpu().double()
        want, tol = S._grad_reference(z, ids, f["norm"].cpu(), f["entropy"].cpu(), gl, gh, 1.0)
        assert torch.all((dz - want).abs() <= tol + U * want.abs() * 1.001), size


def _least_us(call, n=20, times=5):
    """Microseconds of a call among others, the least of several measurements."""
    call()
    us = []
    for _ in range(times):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(n):
            call()
        b.record()
        torch.cuda.synchronize()
        us.append(a.elapsed_time(b) * 1e3 / n)
    return min(us)


@pytest.mark.parametrize("T,V,top,finite", [(264, 30011, 64, 100), (1000, 100003, 20, 500)])
def test_heavily_masked_rows_are_selected_in_one_pass(B, T, V, top, finite):
    """Alternatives of rows that a mask leaves few entries of, more than `top` all the same: no slower than of whole rows by a
    factor (going through the rows again, round by round, took eight times as long)."""
    z = torch.randn(T, V, generator=torch.Generator("cuda").manual_seed(T), device="cuda").bfloat16()
    masked = torch.full_like(z, -math.inf)
    keep = torch.randperm(V, generator=S._gen(V))[:finite].cuda()
    masked[:, keep] = z[:, keep]
    ids = keep[:1].int().repeat(T, 1)
    out = B.adwin_opd_token_logp(masked, ids, top=top)
    few = T // 40
    _check_logp(B, {k: v[:few] for k, v in out.items()}, masked[:few].cpu(), ids[:few].cpu(), 1.0, top)
    assert _least_us(lambda: B.adwin_opd_token_logp(masked, ids, top=top)) <= 3 * _least_us(lambda: B.adwin_opd_token_logp(z, ids, top=top))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(5, 400), (3, 790), (300, 600), (300, 1560), (264, 9001), (2, 70001)])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_few_finite_entries(B, dtype, T, V, top):
    """Rows with fewer finite entries than alternatives, as many, and some more; with and without one wave that has them all."""
    z = torch.full((T, V), -math.inf)
    for t in range(T):
        n = (0, top - 1, top, top + 1, 3 * top)[t % 5] + (t % 5 == 0)
        at = torch.randperm(V if t % 2 else max(V // 5, 3 * top), generator=S._gen(t, V))[:n]
        z[t, at.clamp(max=V - 1)] = torch.randn(len(at), generator=S._gen(t))
    z = z.to(dtype)
    ids = z.argmax(dim=1).int()[:, None].contiguous()
    out = B.adwin_opd_token_logp(z.cuda(), ids.cuda(), top=top, row_status=True)
    assert torch.equal(out["row_status"].cpu() != 0, torch.isinf(z).all(dim=1))
    _check_logp(B, out, z, ids, 1.0, top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [151936, 40003])
@pytest.mark.parametrize("rows", ["equal", "policy", "peaked early"])
def test_sums_of_long_rows(B, dtype, V, rows):
    """s and log p of rows that a workgroup sums whole, to the roundings that there are: n_v vectors of N entries to a thread, whose
    terms are summed first (log2 N of them one after the other), the edge, six steps over the lanes and three over the waves; a
    term itself is off by u (2 + 2 |x| + 3.5), the reference at most 5 above it, and the move to the largest logit by 6.5 u more.  Sums of
    n equal terms are off by u (n + 1) / 2 only, as the partial sums are smaller than the last one."""
    T, N = 264, 8 if dtype == torch.bfloat16 else 4
    g = torch.Generator("cuda").manual_seed(V)
    if rows == "equal":
        z = (torch.arange(T, device="cuda") / 37 - 3)[:, None].repeat(1, V)
    else:
        z = torch.randn(T, V, generator=g, device="cuda") * 1.8
        at = torch.randint(0, V if rows == "policy" else 2000, (T, 8), generator=g, device="cuda")
        z.scatter_(1, at, (0.3 + 0.9 * torch.rand(T, 8, generator=g, device="cuda")) * (math.log(V) + 2) + 4 * (rows != "policy"))
    z = z.to(dtype)
    ids = torch.randint(0, V, (T, 2), generator=g, device="cuda", dtype=torch.int32)
    out = B.adwin_opd_token_logp(z, ids)
    x = z.double()
    x -= x.amax(dim=1, keepdim=True)
    e = x.exp()
    s = e.sum(dim=1)
    mean = -(e * x).sum(dim=1) / s
    vectors = math.ceil(V / (256 * N))
    chain = (vectors + 1) / 2 if rows == "equal" else vectors
    tol = U * (chain + math.log2(N) + 1 + 9 + 12 + 2 * mean)
    assert torch.equal(out["norm"][:, 0], z.float().amax(dim=1))
    assert torch.all((out["norm"][:, 1].double() / s - 1).abs() <= tol)
    logp = x.gather(1, ids.long()) - torch.log(s)[:, None]
    assert torch.all((out["logp"].double() - logp).abs() <= tol[:, None] + U * (2 * logp.abs() + 2 * torch.log(s)[:, None].abs()))
