"""The token-scoring operators against plain computations in 64 bits.

Tolerances.  u = 2^-24 is half a step of fp32; eps / 2 of a type is half a step of it.
  * an exponential relative to the row's reference: its argument d = c z - r is rounded once (u |d|) and carries the
    rounding of c (u |d|), the hardware's exponential one step more: relative error <= u (2 + 2 |d| ln 2) with |x| = |d| ln 2 nats
    below the largest logit (up to 16 more at the reference);
  * their sum: positive terms, at most n = ceil(V / 256) + 8 of them one after the other (a thread's, the waves'), so relative error
    <= u (n + 2 + 2 E|x|), where E|x|, the mean of |x| under p, is at most ln V + 1 (entropy and log s are); with 2 * 16 for the
    reference: S = n + 36 + 2 (ln V + 1), tol(s) = u S;
  * logp = x - log s: u (S + 2 |logp| + 2 |log s|), entropy = log s - t / s: u S (2 + 2 E|x|);
  * gradient: p to u (6 + 4 |x|) of given norm and entropy, a sum of G terms, four products: see _grad_tolerance.
Integers are exact: the quantised rows and the alternatives' ids.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2605_28396_amd import binding
    return binding


def _gen(*key):
    return torch.Generator().manual_seed(hash(key) & 0x7fffffff)


def _strided(x, pad, shift):
    """x on the GPU with `pad` entries between its rows and `shift` in front; what lies between is not x's."""
    T, V = x.shape
    flat = torch.full((shift + T * (V + pad) + 8,), 1e4, dtype=x.dtype, device="cuda")
    view = flat[shift:shift + T * (V + pad)].view(T, V + pad)[:, :V]
    view.copy_(x)
    return view


# ---- rows to integers -----------------------------------------------------------------------------------------------

def _quantised(x):
    a = x.double().abs().amax(dim=1, keepdim=True)
    fine = torch.isfinite(x.double()).all(dim=1, keepdim=True)
    a = torch.where(fine, a, 0.)
    q = torch.where(a > 0, torch.round(x.double() * 127 / torch.where(a > 0, a, 1)), 0.)
    return q.to(torch.int8), (a / 127).float()[:, 0], fine[:, 0]     # (on the GPU torch multiplies an fp32 tensor by 1 / 127)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,H,pad,shift", [(1, 1, 0, 0), (3, 7, 0, 0), (5, 128, 0, 0), (9, 129, 0, 0), (4, 632, 8, 8), (7, 640, 3, 1),
                                           (130, 1000, 0, 0), (2, 4096, 0, 0), (6, 4104, 0, 0), (3, 9001, 5, 3), (2, 65536, 0, 0)])
def test_quant_rows(B, dtype, N, H, pad, shift):
    x = torch.randn(N, H, generator=_gen(N, H)) * torch.logspace(-3, 3, N)[:, None]
    x = x.to(dtype)
    x[0, 0] = 0
    q, s, _ = _quantised(x)
    out = B.adwin_opd_quant_rows(_strided(x, pad, shift), row_status=True)
    assert out["q"].shape == (N, B.ADWIN_QUANT_PITCH(H))
    assert torch.equal(out["q"][:, :H].cpu(), q) and torch.all(out["q"][:, H:] == 0)
    assert torch.equal(out["scale"].cpu(), s) and torch.all(out["row_status"] == 0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quant_rows_at_the_border(B, dtype):
    """Ties, quotients next to a half, rows of zeros, of the smallest and the largest numbers, inf and NaN."""
    big, tiny = torch.finfo(dtype).max, 2.0 ** -130
    x = torch.zeros(9, 300, dtype=torch.float64)
    x[0, :255] = (torch.arange(255) - 127) / 2                   # a = 63.5: 127 x / a = 2 x, no ties
    x[1, :254] = (torch.arange(254) - 126.5)                     # a = 127.5
    x[1, 299] = 127
    x[2, :128] = torch.arange(128) + 0.5
    x[2, 200] = 254                                              # a = 254: 127 x / a = x / 2, ties at odd x
    x[2, 201:290] = torch.arange(89) * 2 + 1
    x[4] = tiny * torch.linspace(-1, 1, 300)
    x[5] = big * torch.linspace(-1, 1, 300)
    x[6] = torch.randn(300, generator=_gen(1)); x[6, 7] = math.inf
    x[7] = torch.randn(300, generator=_gen(2)); x[7, 299] = math.nan
    x[8] = torch.randn(300, generator=_gen(3)); x[8, 0] = -math.inf; x[8, 1] = math.nan
    x = x.to(dtype)
    if dtype == torch.float32:                                   # half steps, and the numbers next to them
        h = (torch.arange(100) + 0.5) * (float(x[0].abs().max()) / 127)
        x[0, :300] = torch.cat([h.float(), torch.nextafter(h.float(), torch.tensor(0.)), torch.nextafter(h.float(), torch.tensor(1e9))])
        x[0, 0] = 63.5
    q, s, fine = _quantised(x)
    out = B.adwin_opd_quant_rows(x.cuda(), row_status=True)
    assert torch.equal(out["q"][:, :300].cpu(), q)
    assert torch.equal(out["scale"].cpu(), s)
    assert torch.equal(out["row_status"].cpu() == B.ADWIN_DEV_NONFINITE, ~fine)


# ---- the product ----------------------------------------------------------------------------------------------------

PRODUCTS = [(1, 1, 1), (1, 1000, 64), (2, 33, 128), (3, 4099, 129), (5, 300, 632), (16, 513, 256), (17, 2000, 640), (31, 1031, 1000),
            (32, 256, 384), (33, 777, 4096), (48, 900, 2048), (64, 515, 512), (65, 640, 130), (100, 3001, 512), (128, 1024, 1024),
            (129, 300, 2560), (200, 1111, 896), (256, 512, 128), (257, 700, 1280), (300, 4100, 640), (520, 1027, 2048), (1000, 2050, 384),
            (8, 20, 65536)]


@pytest.mark.parametrize("T,V,H", PRODUCTS)
@pytest.mark.parametrize("h_dtype,z_dtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                             (torch.float32, torch.bfloat16), (torch.float32, torch.float32)])
def test_quant_logits(B, T, V, H, h_dtype, z_dtype):
    h = torch.randn(T, H, generator=_gen(T, H)).to(h_dtype)
    W = (torch.randn(V, H, generator=_gen(V, H)) * torch.logspace(-2, 1, V)[:, None]).to(torch.bfloat16)
    h[T // 2] = 0
    W[V // 3] = 0
    head = B.QuantHead(W.cuda())
    qh, sh, _ = _quantised(h)
    qW, sW, _ = _quantised(W)
    want = (qh.double() @ qW.double().t()) * sh.double()[:, None] * sW.double()
    # the sum, the product of the scales and their product are rounded to fp32, the result to its type
    tol = want.abs() * (3.01 * U + (torch.finfo(z_dtype).eps / 2 if z_dtype != torch.float32 else 0))
    got = head.logits(h.cuda(), z_dtype=B._DTYPE[z_dtype])
    assert got.dtype == z_dtype and got.shape == (T, V)
    assert torch.all((got.double().cpu() - want).abs() <= tol)
    # into rows that lie apart and begin anywhere, from rows that do
    flat = torch.full((T * (V + 3) + 5,), 7.0, dtype=z_dtype, device="cuda")
    view = flat[1:1 + T * (V + 3)].view(T, V + 3)[:, :V]
    head.logits(_strided(h, 3, 1), z=view)
    assert torch.equal(view, got)
    flat[1:1 + T * (V + 3)].view(T, V + 3)[:, :V] = 7.0
    assert torch.all(flat == 7.0)


@pytest.mark.parametrize("T,V,H", [(17, 70001, 128), (33, 70008, 250), (64, 66000, 256), (5, 600011, 128), (100, 70001, 384), (64, 90000, 2600),
                                   (200, 40000, 128), (256, 33001, 384), (20, 131072, 4096), (400, 32003, 1000), (777, 33001, 1500), (300, 30000, 2000), (256, 50001, 4000),
                                   (140, 70001, 4096), (500, 60007, 700), (3000, 40010, 250), (2050, 66003, 256), (4000, 33000, 384)])
def test_quant_logits_wide(B, T, V, H):
    """Vocabularies of more tiles than there are compute units, where other kernels serve than above."""
    g = torch.Generator("cuda").manual_seed(T)
    h = torch.randn(T, H, generator=g, device="cuda").bfloat16()
    W_q = torch.randint(-127, 128, (V, B.ADWIN_QUANT_PITCH(H)), generator=g, device="cuda", dtype=torch.int8)
    W_q[:, H:] = 0
    W_scale = torch.rand(V, generator=g, device="cuda") + 0.01
    qh, sh, _ = _quantised(h)
    for dtype in (torch.bfloat16, torch.float32):
        got = B.adwin_opd_quant_logits(h, W_q, W_scale, z_dtype=B._DTYPE[dtype])["z"]
        for lo in range(0, V, 16384):
            W = W_q[lo:lo + 16384, :H].double()
            want = (qh.double() @ W.t().contiguous()) * sh.double()[:, None] * W_scale[lo:lo + 16384].double()
            tol = want.abs() * (3.01 * U + (torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 0))
            assert torch.all((got[:, lo:lo + 16384].double() - want).abs() <= tol), (dtype, lo)


def test_quant_logits_of_one_k_step(B):
    """Tiles whose whole contraction is one k-step: the loads run two tiles ahead."""
    T, V, H = 8200, 150001, 100
    g = torch.Generator("cuda").manual_seed(3)
    h = torch.randn(T, H, generator=g, device="cuda")
    W_q = torch.randint(-127, 128, (V, 128), generator=g, device="cuda", dtype=torch.int8)
    W_q[:, H:] = 0
    W_scale = torch.rand(V, generator=g, device="cuda") + 0.01
    qh, sh, _ = _quantised(h)
    got = B.adwin_opd_quant_logits(h, W_q, W_scale)["z"]
    for lo in range(0, V, 8192):
        want = (qh.double() @ W_q[lo:lo + 8192, :H].double().t().contiguous()) * sh.double()[:, None] * W_scale[lo:lo + 8192].double()
        assert torch.all((got[:, lo:lo + 8192].double() - want).abs() <= want.abs() * (3.01 * U + 2.0 ** -8)), lo


def test_quant_logits_largest_sums(B):
    """Every product at its largest, of either sign: the integer sums come to their bound."""
    H = 65536
    h = torch.ones(3, H, dtype=torch.bfloat16)
    h[1] = -1
    W = torch.ones(40, H, dtype=torch.bfloat16)
    W[::3] = -1
    z = B.QuantHead(W.cuda()).logits(h.cuda(), z_dtype=B.ADWIN_DT_F32).double().cpu()
    want = h[:, :1].double() * W[:, 0].double() * H
    assert torch.all((z - want).abs() <= want.abs() * 5.01 * U)      # two scales 1/127 are rounded as well


@pytest.mark.parametrize("T", [1, 40, 300])
def test_quant_logits_excluded_rows(B, T):
    h = torch.randn(T, 256, generator=_gen(T))
    h[T - 1, 3] = math.nan
    out = B.adwin_opd_quant_logits(h.cuda(), *_head(B, 77, 256), row_status=True, z_dtype=B.ADWIN_DT_F32)
    assert torch.all(out["z"][T - 1] == 0) and int(out["row_status"][T - 1]) == B.ADWIN_DEV_NONFINITE
    assert torch.all(out["row_status"][:T - 1] == 0) and torch.all(torch.isfinite(out["z"]))


def _head(B, V, H):
    out = B.adwin_opd_quant_rows(torch.randn(V, H, generator=_gen(V, H, 1)).cuda())
    return out["q"], out["scale"]


# ---- log-probabilities ----------------------------------------------------------------------------------------------

def _reference(z, ids, tau, top):
    """In 64 bits, on the CPU, with the rules for what is not scored and for excluded rows."""
    T, V = z.shape
    zd = z.double()
    ok = (ids >= 0) & (ids < V)
    live = ok.any(dim=1) if ids.shape[1] else torch.ones(T, dtype=torch.bool)
    m = zd.amax(dim=1)
    fine = live & torch.isfinite(m) & ~torch.isnan(zd).any(dim=1)
    x = torch.where(fine[:, None], (zd - torch.where(fine, m, 0.)[:, None]) / tau, 0.)
    e = torch.exp(x)
    s = e.sum(dim=1)
    p = e / s[:, None]
    mean = torch.where(p > 0, p * x, 0.).sum(dim=1)
    ref = {"entropy": torch.where(fine, torch.log(s) - mean, 0.), "mean": -mean, "log_s": torch.log(s),
           "norm": torch.where(fine[:, None], torch.stack([m, s], dim=1), 0.), "fine": fine, "live": live,
           "bad": (ids >= V).any(dim=1) if ids.shape[1] else torch.zeros(T, dtype=torch.bool)}
    lp = x - torch.log(s)[:, None]
    if ids.shape[1]:
        ref["logp"] = torch.where(ok & fine[:, None], lp.gather(1, ids.clamp(0, V - 1).long()), 0.)
    if top:
        at = torch.argsort(zd + 0.0, dim=1, descending=True, stable=True)[:, :top]
        k = at.shape[1]
        ref["top_ids"] = torch.full((T, top), -1, dtype=torch.int32)
        ref["top_logp"] = torch.zeros(T, top, dtype=torch.float64)
        ref["top_ids"][:, :k] = torch.where(fine[:, None], at, -1).to(torch.int32)
        ref["top_logp"][:, :k] = torch.where(fine[:, None], lp.gather(1, at), 0.)
    return ref


def _close(got, want, tol, what):
    got, want = got.double().cpu(), want.double()
    same = torch.isinf(want) & (got == want)
    off = torch.where(same, 0., (got - want).abs())
    assert torch.all(off <= torch.where(same, 0., tol)), (what, float((off - tol).max()))


def _check_logp(B, out, z, ids, tau, top):
    V = z.shape[1]
    ref = _reference(z, ids, tau, top)
    S = math.ceil(V / 256) + 8 + 36 + 2 * (math.log(V) + 1)
    row = U * (S + 2 * ref["log_s"].abs())[:, None]
    if ids.shape[1]:
        _close(out["logp"], ref["logp"], row + 2 * U * ref["logp"].abs().clamp(max=1e30), "logp")
    _close(out["entropy"], ref["entropy"], U * S * (2 + 2 * ref["mean"]), "entropy")
    assert torch.equal(out["norm"][:, 0].double().cpu(), ref["norm"][:, 0])
    _close(out["norm"][:, 1], ref["norm"][:, 1], U * S * ref["norm"][:, 1], "norm")
    if top:
        assert torch.equal(out["top_ids"].cpu(), ref["top_ids"])
        _close(out["top_logp"], ref["top_logp"], row + 2 * U * ref["top_logp"].abs().clamp(max=1e30), "top_logp")
    if "row_status" in out:
        want = ref["bad"].int() * B.ADWIN_DEV_BAD_ID + (ref["live"] & ~ref["fine"]).int() * B.ADWIN_DEV_NONFINITE
        assert torch.equal(out["row_status"].cpu(), want.int())
    return ref


def _logits(T, V, dtype, key, spread=2.0):
    return (torch.randn(T, V, generator=_gen(T, V, key)) * spread).to(dtype)


def _ids(T, G, V, key):
    return torch.randint(0, V, (T, G), generator=_gen(T, G, V, key), dtype=torch.int32)


ROWS = [(1, 1), (2, 2), (3, 7), (5, 64), (4, 255), (3, 256), (2, 2047), (3, 2049), (7, 4096), (2, 8193), (3, 11907), (2, 20000),
        (300, 1030), (1, 40000), (2, 65537), (1, 151936), (3, 151937)]


@pytest.mark.parametrize("T,V", ROWS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("G,top,tau,pad,shift", [(1, 20, 1.0, 0, 0), (0, 1, 1.0, 0, 0), (5, 64, 0.7, 3, 1), (128, 0, 1.3, 8, 0)])
def test_token_logp(B, T, V, dtype, G, top, tau, pad, shift):
    z, ids = _logits(T, V, dtype, 1), _ids(T, G, V, 2)
    if G > 1:
        ids[::2, 1] = -1
        ids[:, -1] = ids[:, 0]
    out = B.adwin_opd_token_logp(_strided(z, pad, shift), ids.cuda() if G else None, temperature=tau, top=top, row_status=True)
    assert set(out) == {"entropy", "norm", "row_status"} | ({"logp"} if G else set()) | ({"top_ids", "top_logp"} if top else set())
    _check_logp(B, out, z, ids, tau, top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [9, 700, 5001, 70001])
@pytest.mark.parametrize("T", [1, 40])
def test_token_logp_masks(B, dtype, V, T):
    """Masked entries (-inf, the type's lowest value), rows that they leave empty or with one entry, NaN, +inf, ids that are not
    scored or do not exist."""
    low = torch.finfo(dtype).min
    rows = []
    for k in range(10):
        z = _logits(1, V, dtype, 10 + k)[0]
        if k == 1: z[torch.randperm(V, generator=_gen(V))[:V // 2]] = -math.inf
        if k == 2: z[:] = -math.inf; z[V // 3] = 2.0                # one token left
        if k == 3: z[:] = -math.inf                                # none
        if k == 4: z[:V - 1] = low                                 # all but the last masked with the lowest value
        if k == 5: z[:] = low                                      # every entry at the lowest value: uniform
        if k == 6: z[V // 2] = math.nan
        if k == 7: z[V - 1] = math.inf
        if k == 8: z[:V // 2] = low; z[V // 2:] = -math.inf
        if k == 9: z[: V - V // 8] = -math.inf
        rows.append(z)
    z = torch.stack(rows)
    ids = _ids(10, 3, V, 5)
    ids[2, 0] = V // 3
    ids[2, 1] = 0                                                  # a masked token is asked for: -inf
    both = torch.cat([z, z]), torch.cat([ids, ids])
    both[1][10] = -1                                               # a row that is not scored
    both[1][11, 0] = V                                             # and ids that do not exist
    both[1][12] = torch.tensor([V, V + 5, -3])
    z, ids = (torch.cat([x] * max(1, T // 20)) for x in both)
    for at in range(0, len(z), T):
        zs, i = z[at:at + T], ids[at:at + T]
        out = B.adwin_opd_token_logp(zs.cuda(), i.cuda(), top=9, row_status=True)
        _check_logp(B, out, zs, i, 1.0, 9)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V", [(3, 300), (2, 5000), (2, 40001), (40, 9000)])
@pytest.mark.parametrize("order", ["rising", "falling", "equal", "two values", "late peak", "far apart", "zeros of either sign"])
def test_token_logp_orders(B, dtype, T, V, order):
    """Alternatives of rows whose order is the worst for a bound taken early, ties, and a wide range."""
    z = torch.linspace(-8, 8, V).repeat(T, 1)
    if order == "falling": z = z.flip(1)
    if order == "equal": z = torch.full((T, V), 0.5)
    if order == "two values": z = (torch.arange(V) % 3 == 0).float().repeat(T, 1)
    if order == "late peak": z = _logits(T, V, torch.float32, 3); z[:, V - V // 7:] += 12
    if order == "far apart": z = _logits(T, V, torch.float32, 4, 300.0)
    if order == "zeros of either sign": z = torch.where(torch.arange(V) % 2 == 0, -0.0, 0.0).repeat(T, 1)
    z = z.to(dtype).contiguous()
    ids = _ids(T, 2, V, 6)
    for top in (1, 13, 64):
        _check_logp(B, B.adwin_opd_token_logp(z.cuda(), ids.cuda(), top=top), z, ids, 1.0, top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("order", ["rising", "falling", "equal", "two values", "late peak", "peak in one wave", "masked but few", "lowest but few",
                                   "masked at first", "nan at last", "far at last"])
def test_token_logp_many_long_rows(B, dtype, order):
    """The same where a workgroup goes through a whole row in many steps: calls of many rows."""
    T, V = 264, 30011
    low = torch.finfo(dtype).min
    z = torch.linspace(-8, 8, V).repeat(2, 1)
    if order == "falling": z = z.flip(1)
    if order == "equal": z = torch.full((2, V), 0.5)
    if order == "two values": z = (torch.arange(V) % 3 == 0).float().repeat(2, 1)
    if order in ("late peak", "nan at last", "far at last"): z = _logits(2, V, torch.float32, 3); z[:, V - V // 7:] += 12
    if order == "peak in one wave": z = _logits(2, V, torch.float32, 5); z[:, (torch.arange(V) // 8) % 256 < 64] += 9
    if order == "masked but few": z = torch.full((2, V), -math.inf); z[:, ::1000] = _logits(2, 31, torch.float32, 6)
    if order == "lowest but few": z = torch.full((2, V), low); z[:, 5::1000] = _logits(2, 31, torch.float32, 6)[:, :len(range(5, V, 1000))]
    if order == "masked at first": z = _logits(2, V, torch.float32, 7); z[:, :V - V // 8] = -math.inf
    if order == "nan at last": z[1, V - 1] = math.nan
    if order == "far at last": z[1, V - 2] = 1e30
    z = z.to(dtype)
    ids = torch.tensor([[3, 17], [V - 1, 5]], dtype=torch.int32)
    many, many_ids = z.repeat(T // 2, 1).cuda(), ids.repeat(T // 2, 1).cuda()
    for top in (1, 20, 64):
        out = B.adwin_opd_token_logp(many, many_ids, top=top, row_status=True)
        # sixteen rows begin at every place that 16 bytes have for a row; the order of its sums goes by that, and by nothing else
        _check_logp(B, {k: v[:16] for k, v in out.items()}, z.repeat(8, 1), ids.repeat(8, 1), 1.0, top)
        for k, v in out.items():
            assert torch.equal(v[16:], v[:-16]), k


def test_token_logp_small_forms(B):
    z = _logits(6, 50, torch.float32, 1)
    ids = _ids(6, 1, 50, 1)
    a = B.adwin_opd_token_logp(z.cuda(), ids.cuda())
    b = B.adwin_opd_token_logp(z.cuda(), ids[:, 0].contiguous().cuda())
    assert a["logp"].shape == (6, 1) and b["logp"].shape == (6,) and torch.equal(a["logp"][:, 0], b["logp"])
    empty = B.adwin_opd_token_logp(z[:0].cuda(), ids[:0].cuda(), top=3)
    assert empty["logp"].shape == (0, 1) and empty["top_ids"].shape == (0, 3)
    assert B.adwin_opd_quant_rows(z[:0].cuda())["q"].shape == (0, 128)
    assert B.adwin_opd_token_logp_grad(z[:0].cuda(), ids[:0].cuda(), empty["norm"], empty["logp"])["dz"].shape == (0, 50)
    with pytest.raises(B.AdwinError):
        B.adwin_opd_token_logp(z.cuda(), ids.cuda(), temperature=0.0)
    with pytest.raises(B.AdwinError):
        B.adwin_opd_token_logp(z.cuda(), ids.cuda(), top=65)
    for bad in (ids.long().cuda(), ids[:3].cuda(), ids):
        with pytest.raises(ValueError):
            B.adwin_opd_token_logp(z.cuda(), bad)


# ---- gradient -------------------------------------------------------------------------------------------------------

def _grad_reference(z, ids, norm, entropy, gl, gh, tau):
    """dz in 64 bits from the given norm and entropy, and its tolerance before the last rounding."""
    V = z.shape[1]
    fine = norm[:, 1] > 0
    s = torch.where(fine, norm[:, 1].double(), 1.)
    x = torch.where(fine[:, None], (z.double() - norm[:, :1].double()) / tau, -math.inf)
    p = torch.exp(x) / s[:, None]
    lp = torch.where(p > 0, x - torch.log(s)[:, None], 0.)
    ok = (ids >= 0) & (ids < V) & fine[:, None]
    g = torch.where(ok, gl.double(), 0.)
    own, size = torch.zeros_like(p), torch.zeros_like(p)
    own.scatter_add_(1, ids.clamp(0, V - 1).long(), g)
    size.scatter_add_(1, ids.clamp(0, V - 1).long(), g.abs())
    a, gH, H = g.sum(dim=1, keepdim=True), gh.double()[:, None], entropy.double()[:, None]
    dz = (own - p * a - gH * p * (lp + H)) / tau
    depth = torch.where(p > 0, x.abs(), 0.)
    parts = p * (g.abs().sum(dim=1, keepdim=True) + gH.abs() * (lp.abs() + H.abs() + 2)) + size
    return torch.where(fine[:, None], dz, 0.), U * (16 + 4 * depth + 2 * ids.shape[1]) * parts / tau


@pytest.mark.parametrize("T,V", [(1, 1), (2, 3), (3, 257), (5, 2049), (40, 1031), (3, 11907), (2, 40000), (1, 151937), (300, 700)])
@pytest.mark.parametrize("z_dtype,dz_dtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                              (torch.float32, torch.bfloat16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("G,with_entropy,tau,pad,shift", [(1, False, 1.0, 0, 0), (5, True, 0.7, 3, 1), (128, True, 1.3, 8, 8),
                                                          (0, True, 1.0, 0, 0)])
def test_token_logp_grad(B, T, V, z_dtype, dz_dtype, G, with_entropy, tau, pad, shift):
    z, ids = _logits(T, V, z_dtype, 1), _ids(T, G, V, 2)
    if V > 100: z[:, 50:60] = -math.inf
    if G > 1:
        ids[::2, 1] = -1
        ids[:, -1] = ids[:, 0]                                     # the same token twice
        ids[T - 1, 2] = V + 3
        if T > 3: ids[2] = -1
    zc = _strided(z, pad, shift)
    idc = ids.cuda() if G else None
    f = B.adwin_opd_token_logp(zc, idc, temperature=tau)
    gl = torch.randn(T, G, generator=_gen(T, G, 3))
    gh = torch.randn(T, generator=_gen(T, 4))
    kw = dict(entropy=f["entropy"], g_entropy=gh.cuda()) if with_entropy else {}
    out = B.adwin_opd_token_logp_grad(zc, idc, f["norm"], gl.cuda() if G else None, temperature=tau, dz_dtype=B._DTYPE[dz_dtype], **kw)
    want, tol = _grad_reference(z, ids, f["norm"].cpu(), f["entropy"].cpu(), gl, gh if with_entropy else torch.zeros(T), tau)
    tol = tol + torch.finfo(dz_dtype).eps / 2 * want.abs() * 1.001
    assert out["dz"].dtype == dz_dtype
    assert torch.all((out["dz"].double().cpu() - want).abs() <= tol)
    # into rows that lie apart; what lies between them stays
    flat = torch.full((T * (V + 5) + 9,), 7.0, dtype=dz_dtype, device="cuda")
    view = flat[2:2 + T * (V + 5)].view(T, V + 5)[:, :V]
    B.adwin_opd_token_logp_grad(zc, idc, f["norm"], gl.cuda() if G else None, temperature=tau, dz=view, **kw)
    assert torch.equal(view, out["dz"])
    view[:] = 7.0
    assert torch.all(flat == 7.0)
    if z_dtype == dz_dtype:                                        # in place
        B.adwin_opd_token_logp_grad(zc, idc, f["norm"], gl.cuda() if G else None, temperature=tau, dz=zc, **kw)
        assert torch.equal(zc, out["dz"])


def test_token_logp_grad_of_excluded_rows(B):
    z = _logits(5, 3000, torch.float32, 1)
    z[0, 7] = math.nan; z[1, 8] = math.inf; z[2] = -math.inf; z[4] = torch.finfo(torch.float32).min
    ids = _ids(5, 2, 3000, 1)
    ids[3] = -1
    f = B.adwin_opd_token_logp(z.cuda(), ids.cuda())
    g = torch.ones(5, 2).cuda()
    dz = B.adwin_opd_token_logp_grad(z.cuda(), ids.cuda(), f["norm"], g, entropy=f["entropy"], g_entropy=g[:, 0].contiguous())["dz"].cpu()
    assert torch.all(dz[:4] == 0)
    want, tol = _grad_reference(z[4:], ids[4:], f["norm"][4:].cpu(), f["entropy"][4:].cpu(), torch.ones(1, 2), torch.ones(1), 1.0)
    assert torch.all((dz[4:].double() - want).abs() <= tol + U * want.abs())


def test_gradient_by_differences(B):
    """dz against central differences of the loss that the forward call puts out."""
    T, V, G, tau = 3, 37, 4, 0.8
    z, ids = _logits(T, V, torch.float32, 1), _ids(T, G, V, 2)
    ids[0, 2] = ids[0, 1]
    gl, gh = torch.randn(T, G, generator=_gen(1)), torch.randn(T, generator=_gen(2))
    f = B.adwin_opd_token_logp(z.cuda(), ids.cuda(), temperature=tau)
    dz = B.adwin_opd_token_logp_grad(z.cuda(), ids.cuda(), f["norm"], gl.cuda(), entropy=f["entropy"], g_entropy=gh.cuda(),
                                     temperature=tau)["dz"].double().cpu()
    step = 2.0 ** -6
    moved = z.repeat_interleave(2 * V, 0)                          # row t, entry j, up and down
    k = torch.arange(2 * V)
    for t in range(T):
        moved[t * 2 * V + k, k // 2] += torch.where(k % 2 == 0, step, -step)
    o = B.adwin_opd_token_logp(moved.cuda(), ids.repeat_interleave(2 * V, 0).cuda(), temperature=tau)
    loss = (o["logp"].double().cpu() * gl.repeat_interleave(2 * V, 0)).sum(1) + o["entropy"].double().cpu() * gh.repeat_interleave(2 * V, 0)
    loss = loss.view(T, V, 2)
    # third derivatives of log p and H by x are below 2 and 12; the loss is rounded to about 2^-20 of its parts
    size = gl.abs().sum(1) + gh.abs()
    tol = (step ** 2 / 6 * 12 / tau ** 3 + 2.0 ** -19 / step) * size.double()[:, None]
    assert torch.all((dz - (loss[..., 0] - loss[..., 1]) / (2 * step)).abs() <= tol)


# ---- calls ----------------------------------------------------------------------------------------------------------

def test_rows_beyond_32_bit_offsets(B):
    """Rows whose bytes begin beyond 2^32 give what they give by themselves."""
    V, T = 151937, 15000
    z = torch.empty(T, V, dtype=torch.bfloat16, device="cuda")
    for lo in range(0, T, 1000):
        z[lo:lo + 1000] = torch.randn(1000, V, generator=torch.Generator("cuda").manual_seed(lo), device="cuda")
    ids = torch.randint(0, V, (T, 2), generator=torch.Generator("cuda").manual_seed(1), device="cuda", dtype=torch.int32)
    ids[:T - 40] = -1
    out = B.adwin_opd_token_logp(z, ids, top=5)
    part = B.adwin_opd_token_logp(z[T - 40:].clone(), ids[T - 40:].contiguous(), top=5)
    ref = _reference(z[T - 40:].cpu(), ids[T - 40:].cpu(), 1.0, 5)
    assert torch.equal(out["top_ids"][T - 40:].cpu(), ref["top_ids"]) and torch.equal(part["top_ids"], out["top_ids"][T - 40:])
    _close(out["logp"][T - 40:], ref["logp"], torch.tensor(U * 800.), "logp")
    g = torch.ones(T, 2, device="cuda")
    dz = B.adwin_opd_token_logp_grad(z, ids, out["norm"], g)["dz"]
    want = B.adwin_opd_token_logp_grad(z[T - 40:].clone(), ids[T - 40:].contiguous(), out["norm"][T - 40:].contiguous(), g[:40])["dz"]
    assert torch.equal(dz[T - 40:], want) and torch.all(dz[:T - 40] == 0)
    del dz, z
    torch.cuda.empty_cache()
    h = torch.randn(T, 128, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    W_q, W_s = _head(B, V, 128)
    logits = B.adwin_opd_quant_logits(h, W_q, W_s)["z"]
    assert torch.equal(logits[T - 300:], B.adwin_opd_quant_logits(h[T - 300:], W_q, W_s)["z"])


def test_calls_on_another_stream(B):
    z, ids = _logits(50, 9000, torch.bfloat16, 1).cuda(), _ids(50, 3, 9000, 1).cuda()
    want = B.adwin_opd_token_logp(z, ids, top=7)
    W_q, W_s = _head(B, 9000, 200)
    h = torch.randn(50, 200, device="cuda")
    want_z = B.adwin_opd_quant_logits(h, W_q, W_s)["z"]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for s in (side, side.cuda_stream):
        got = B.adwin_opd_token_logp(z, ids, top=7, stream=s)
        got_z = B.adwin_opd_quant_logits(h, W_q, W_s, stream=s)["z"]
        dz = B.adwin_opd_token_logp_grad(z, ids, got["norm"], got["logp"], stream=s)["dz"]
        side.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in want) and torch.equal(got_z, want_z)
        assert torch.equal(dz, B.adwin_opd_token_logp_grad(z, ids, want["norm"], want["logp"])["dz"])


@pytest.mark.parametrize("T", [2, 70])
def test_calls_replay_from_a_graph(B, T):
    V, H = 20000, 384
    h, z = torch.randn(T, H, device="cuda"), torch.empty(T, V, dtype=torch.bfloat16, device="cuda")
    W_q, W_s = _head(B, V, H)
    ids = _ids(T, 2, V, 1).cuda()

    def step():
        B.adwin_opd_quant_logits(h, W_q, W_s, z=z)
        out = B.adwin_opd_token_logp(z, ids, top=8)
        out["dz"] = B.adwin_opd_token_logp_grad(z, ids, out["norm"], out["logp"], entropy=out["entropy"], g_entropy=out["entropy"])["dz"]
        return out
    B.adwin_opd_init()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for k in range(4):
        h.copy_(torch.randn(T, H, device="cuda", generator=torch.Generator("cuda").manual_seed(k)))
        ids[0] = k
        for v in out.values():
            v.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = {n: v.clone() for n, v in out.items()}
        want = step()
        assert all(torch.equal(got[n], want[n]) for n in want), k


def test_outputs_that_are_not_wanted(B):
    """NULL outputs at the C ABI: what is asked for is the same."""
    import ctypes as C
    z, ids = _logits(9, 5000, torch.bfloat16, 1).cuda(), _ids(9, 2, 5000, 1).cuda()
    want = B.adwin_opd_token_logp(z, ids, top=6, row_status=True)
    for names in (("logp",), ("entropy",), ("norm",), ("top_ids",), ("top_logp",), ("row_status",), ("logp", "top_ids"), ()):
        p = B.adwin_opd_logp_problem()
        p.struct_bytes = C.sizeof(p)
        p.T, p.ld_z, p.V, p.G, p.top, p.z_dtype, p.temperature = 9, 5000, 5000, 2, 6, B.ADWIN_DT_BF16, 1.0
        p.z, p.ids = z.data_ptr(), ids.data_ptr()
        got = {n: torch.full_like(want[n], 5) for n in names}
        for n, t in got.items():
            setattr(p, n, t.data_ptr())
        need = B.adwin_opd_token_logp_workspace_bytes(p)
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        assert B.lib.adwin_opd_token_logp(C.byref(p), ws.data_ptr(), need, None) == 0
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in names), names
