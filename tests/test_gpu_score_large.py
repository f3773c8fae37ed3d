"""The token-scoring operators on arrays that pass the caches, in every type: other instantiations of their kernels serve these
(quant_rows from 96 MiB on, log-probabilities and their gradient from 320 MiB on).  All outputs are held to 64 bits, on the GPU, some
rows at a time; tolerances are those of test_gpu_score.py."""
import math

import pytest
import torch

from . import test_gpu_score as S

pytestmark = pytest.mark.gpu
U = S.U
TYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2605_28396_amd import binding
    return binding


def _pitched(T, V, pitch, dtype, seed, scale=2.0):
    """Rows `pitch` entries apart; what lies between them is not theirs."""
    g = torch.Generator("cuda").manual_seed(seed)
    flat = torch.full((T, pitch), 1e4, dtype=dtype, device="cuda")
    for lo in range(0, T, 512):
        n = min(512, T - lo)
        flat[lo:lo + n, :V] = torch.randn(n, V, generator=g, device="cuda") * scale
    return flat[:, :V]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,H,pitch", [(14000, 4096, 4096), (30000, 2048, 2056), (1000, 60000, 60000), (60000, 1000, 1008)])
def test_quant_rows_past_the_caches(B, dtype, N, H, pitch):
    x = _pitched(N, H, pitch, dtype, N)
    assert N * H * x.element_size() > 96 << 20
    x[5] = 0
    x[N - 2, H - 1] = math.inf
    x[7, 3] = math.nan
    x[9, :4] = torch.tensor([254.0, 1.0, 3.0, -5.0])             # ties
    out = B.adwin_opd_quant_rows(x, row_status=True)
    for lo in range(0, N, 2048):
        w = x[lo:lo + 2048].double()
        fine = torch.isfinite(w).all(dim=1, keepdim=True)
        a = torch.where(fine, w, 0.).abs().amax(dim=1, keepdim=True)
        q = torch.where(a > 0, torch.round(w * 127 / torch.where(a > 0, a, 1.)), 0.).to(torch.int8)
        assert torch.equal(out["q"][lo:lo + 2048, :H], q) and torch.all(out["q"][lo:lo + 2048, H:] == 0)
        assert torch.equal(out["scale"][lo:lo + 2048], (a / torch.full_like(a, 127)).float()[:, 0])
        assert torch.equal(out["row_status"][lo:lo + 2048] == B.ADWIN_DEV_NONFINITE, ~fine[:, 0])


@pytest.mark.parametrize("z_dtype,T,V,pitch", [(torch.bfloat16, 1200, 151936, 151936), (torch.float32, 600, 151937, 151937), (torch.float32, 3000, 32771, 32776),
                                               (torch.bfloat16, 6000, 30001, 30008), (torch.float32, 90000, 1000, 1000)])
def test_log_probabilities_past_the_caches(B, z_dtype, T, V, pitch):
    """Forward, then the gradient in either type and in place."""
    z = _pitched(T, V, pitch, z_dtype, T)
    assert T * V * z.element_size() > 320 << 20
    z[3, V // 3:V // 2] = -math.inf
    z[4] = -math.inf
    z[6, V - 1] = math.nan
    z[8, :V - 1] = torch.finfo(z_dtype).min
    g = torch.Generator("cuda").manual_seed(V)
    ids = torch.randint(0, V, (T, 3), generator=g, device="cuda", dtype=torch.int32)
    ids[::3, 2] = ids[::3, 1]                                    # the same token twice
    ids[10] = -1
    ids[T - 1, 0] = V
    tau, top = 0.75, 20
    out = B.adwin_opd_token_logp(z, ids, temperature=tau, top=top, row_status=True)
    gl, gh = torch.randn(T, 3, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")
    dz = {dt: B.adwin_opd_token_logp_grad(z, ids, out["norm"], gl, entropy=out["entropy"], g_entropy=gh, temperature=tau,
                                          dz_dtype=B._DTYPE[dt])["dz"] for dt in TYPES}
    n = math.ceil(V / 256) + 8 + 36 + 2 * (math.log(V) + 1)
    rows = max(8, (1 << 25) // V)
    for lo in range(0, T, rows):
        at = slice(lo, min(lo + rows, T))
        i, raw = ids[at], z[at].double()
        ok = (i >= 0) & (i < V)
        live = ok.any(dim=1)
        m = raw.amax(dim=1)
        fine = live & torch.isfinite(m) & ~torch.isnan(raw).any(dim=1)
        f1 = fine[:, None]
        x = torch.where(f1, (raw - torch.where(fine, m, 0.)[:, None]) / tau, 0.)
        e = x.exp()
        s = e.sum(dim=1)
        p = e / s[:, None]
        mean = -torch.where(p > 0, p * x, 0.).sum(dim=1)
        log_s = torch.log(s)
        lp = x - log_s[:, None]
        lp = torch.where(lp < -torch.finfo(torch.float32).max, -math.inf, lp)          # beyond fp32
        want = torch.where(ok & f1, lp.gather(1, i.clamp(0, V - 1).long()), 0.)
        got = out["logp"][at].double()
        off = torch.where(torch.isinf(want) & (want == got), 0., (got - want).abs())
        assert torch.all(off <= U * (n + 2 * log_s.abs()[:, None] + 2 * torch.where(torch.isinf(want), 0., want).abs()))
        assert torch.all((out["entropy"][at].double() - torch.where(fine, log_s + mean, 0.)).abs() <= U * n * (2 + 2 * mean))
        assert torch.equal(out["norm"][at, 0].double(), torch.where(fine, m, 0.))
        assert torch.all((out["norm"][at, 1].double() - torch.where(fine, s, 0.)).abs() <= U * n * s)
        status = (i >= V).any(dim=1).int() * B.ADWIN_DEV_BAD_ID + (live & ~fine).int() * B.ADWIN_DEV_NONFINITE
        assert torch.equal(out["row_status"][at], status.int())
        order = torch.sort(torch.nan_to_num(raw, nan=0.), dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(out["top_ids"][at], torch.where(f1, order, -1).int())
        want = torch.where(f1, lp.gather(1, order), 0.)
        got = out["top_logp"][at].double()
        off = torch.where(torch.isinf(want) & (want == got), 0., (got - want).abs())
        assert torch.all(off <= U * (n + 2 * log_s.abs()[:, None] + 2 * torch.where(torch.isinf(want), 0., want).abs()))
        # the gradient, of the norm and entropy that the forward call wrote
        want, tol = _gradient(z[at], i, out["norm"][at], out["entropy"][at], gl[at], gh[at], tau)
        for dt in TYPES:
            half = U if dt == torch.float32 else 2.0 ** -8
            assert torch.all((dz[dt][at].double() - want).abs() <= tol + half * want.abs() * 1.001), (dt, lo)
    B.adwin_opd_token_logp_grad(z, ids, out["norm"], gl, entropy=out["entropy"], g_entropy=gh, temperature=tau, dz=z)
    assert torch.equal(z, dz[z_dtype])


def test_gradients_of_mixed_types_take_the_same_time(B):
    """From bf16 to fp32 as many bytes as from fp32 to bf16: 32 bytes of a lane stored past the caches took 1.6 to 1.75 times as long."""
    from .test_gpu_score_range import _least_us
    T, V = 2000, 100000
    us = {}
    for z_dtype, dz_dtype in (TYPES, TYPES[::-1]):
        z, dz = _pitched(T, V, V, z_dtype, 1), torch.empty(T, V, dtype=dz_dtype, device="cuda")
        ids, g = torch.zeros(T, 1, dtype=torch.int32, device="cuda"), torch.ones(T, 1, device="cuda")
        norm = B.adwin_opd_token_logp(z, ids)["norm"]
        us[z_dtype] = _least_us(lambda: B.adwin_opd_token_logp_grad(z, ids, norm, g, dz=dz))
    assert us[torch.bfloat16] <= 1.45 * us[torch.float32], us


def _gradient(z, ids, norm, entropy, gl, gh, tau):
    """S._grad_reference on the GPU."""
    V = z.shape[1]
    fine = norm[:, 1] > 0
    f1 = fine[:, None]
    s = torch.where(fine, norm[:, 1].double(), 1.)
    x = torch.where(f1, (z.double() - norm[:, :1].double()) / tau, -math.inf)
    p = torch.exp(x) / s[:, None]
    lp = torch.where(p > 0, x - torch.log(s)[:, None], 0.)
    g = torch.where((ids >= 0) & (ids < V) & f1, gl.double(), 0.)
    own, size = torch.zeros_like(p), torch.zeros_like(p)
    at = ids.clamp(0, V - 1).long()
    for k in range(ids.shape[1]):                                # one after the other: no atomics in the reference
        own[torch.arange(len(p), device="cuda"), at[:, k]] += g[:, k]
        size[torch.arange(len(p), device="cuda"), at[:, k]] += g[:, k].abs()
    a, gH, H = g.sum(dim=1, keepdim=True), gh.double()[:, None], entropy.double()[:, None]
    dz = (own - p * a - gH * p * (lp + H)) / tau
    parts = p * (g.abs().sum(dim=1, keepdim=True) + gH.abs() * (lp.abs() + H.abs() + 2)) + size
    depth = torch.where(p > 0, x.abs(), 0.)
    return torch.where(f1, dz, 0.), U * (16 + 4 * depth + 2 * ids.shape[1]) * parts / tau
