"""Products whose contraction has more than 32 blocks, exactly; how far bf16 results may be off, to the bit that the matrix units cut;
and rows to blocks of arrays past the caches.

Tolerances.  u = 2^-24 is half a step of fp32.  For bf16 results the matrix units take eight products at a time, entries 8 i to 8 i + 7 of a
row, each cut towards zero at 2^-13 of the largest's power of two, and add them to a sum in fp32, which is not cut.  The largest itself has
eight bits and is not cut: with G the sum over these groups of the largest |a b|, all cuts are below 7 * 2^-13 G.  Additions in fp32, of K / 8
groups and of parts: (K / 8 + 64) 2 u S, S = sum |a b|.  Then half a step of bf16, 2^-8 |c|.
"""
import pytest
import torch

from .test_gpu_block import F8, U, _gen, _product, _up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2605_28396_amd import binding
    return binding


# Entries of -1 to 1 and scales of 1 and 2, at random: products of 0 to 4, of which nothing is cut, and sums within 2^20, exact in fp32.
LONG = [(1, 20, 65536), (5, 33, 9000), (40, 60, 30001), (100, 1000, 33333), (200, 2000, 30001), (700, 600, 50007), (600, 2050, 24000),
        (2049, 4097, 40000), (3000, 3001, 33000), (512, 2048, 151936), (3, 40001, 8200), (17, 70001, 4500), (1, 30001, 10100), (1100, 300, 5000),
        (5, 30001, 4600), (32, 40003, 4100)]


@pytest.mark.parametrize("M,N,K", LONG)
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("a_tile,b_tile", [(1, 128), (1, 1)])
def test_every_block_of_a_long_contraction_counts_once(B, M, N, K, fmt, a_tile, b_tile):
    g, P = torch.Generator("cuda").manual_seed(M + N + K), _up(K, 128)
    kept, scales, wide = [], [], []
    for n, tile in ((M, a_tile), (N, b_tile)):
        q = torch.zeros(n, P, device="cuda")
        q[:, :K] = torch.randint(-1, 2, (n, K), generator=g, device="cuda")
        e = torch.zeros((n + tile - 1) // tile, _up(P // 128, 4), dtype=torch.uint8, device="cuda")
        e[:, :P // 128] = torch.randint(127, 129, (e.shape[0], P // 128), generator=g, device="cuda").to(torch.uint8)
        kept.append(q)
        scales.append(e)
        by_row = torch.ldexp(torch.ones((), device="cuda"), e.int() - 127).repeat_interleave(tile, dim=0)[:n, :P // 128]
        wide.append((q.view(n, -1, 128) * by_row[:, :, None]).view(n, P))
    want = torch.zeros(M, N, dtype=torch.float64, device="cuda")
    for k in range(0, P, 8192):
        want += wide[0][:, k:k + 8192].double() @ wide[1][:, k:k + 8192].double().t().contiguous()
    status = (torch.rand(M, generator=g, device="cuda") < 0.1).int()
    a, b = kept[0].to(F8[fmt][0]), kept[1].to(torch.float8_e4m3fn)
    del kept, wide
    for c_dtype, dt in ((B.ADWIN_DT_F32, torch.float32), (B.ADWIN_DT_BF16, torch.bfloat16)):
        c = B.adwin_opd_block_product(a, scales[0], b, scales[1], a_tile=a_tile, b_tile=b_tile, c_dtype=c_dtype)["c"]
        assert torch.equal(c, want.to(dt)), c_dtype
        c = B.adwin_opd_block_product(a, scales[0], b, scales[1], a_tile=a_tile, b_tile=b_tile, c_dtype=c_dtype, a_status=status)["c"]
        assert torch.equal(c, torch.where((status != 0)[:, None], 0, want).to(dt)), c_dtype


CUT = [(1, 700, 4096), (64, 515, 512), (129, 300, 2560), (300, 200, 20000), (700, 1500, 4096), (2100, 2300, 1024), (600, 1030, 24000)]


def _largest_of_eight(a, b):
    """Sum over the groups of eight of the largest |a b|, [M, N]."""
    a, b = a.abs().float(), b.abs().float()
    out = torch.zeros(a.shape[0], b.shape[0], device="cuda")
    for k in range(0, a.shape[1], 8):
        most = a[:, k, None] * b[None, :, k]
        for i in range(k + 1, min(k + 8, a.shape[1])):
            most = torch.maximum(most, a[:, i, None] * b[None, :, i])
        out += most
    return out.double()


@pytest.mark.parametrize("M,N,K", CUT)
@pytest.mark.parametrize("fmt,spread", [("e4m3", 0.0), ("e5m2", 0.0), ("e4m3", 2.0), ("e5m2", 3.0)])
def test_bf16_results_are_cut_no_further_than_is_said(B, M, N, K, fmt, spread):
    a = torch.randn(M, K, generator=_gen(M, K)) * torch.exp(spread * torch.randn(M, K, generator=_gen(K, M)))
    b = torch.randn(N, K, generator=_gen(N, K)) * torch.exp(spread / 2 * torch.randn(N, K, generator=_gen(K, N)))
    qa, qb, c = _product(B, a.cuda(), b.cuda(), 1, 1, fmt, B.ADWIN_DT_BF16)
    xa, xb = _values(qa), _values(qb)
    want, S = xa @ xb.t().contiguous(), xa.abs() @ xb.abs().t().contiguous()
    tol = 7 * 2.0 ** -13 * _largest_of_eight(xa, xb) * (1 + 4 * U) + (K / 8 + 64) * 2 * U * S
    tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs() + 2.0 ** -126
    off = ((c.double() - want).abs() / tol).max()
    assert off <= 1, off
    if spread == 0:
        # In all, cuts are some e = 1.4e-5 of the result's norm for normal entries.  A result c whose error is d rounds to another bf16 number than the
        # exact one with probability |d| / step, step <= 2^-7 |c|, and by a step then.  Of n results of norm n^(1/2), the squares that this changes
        # have the mean |d| step <= 2^-7 |c d| each, 2^-7 e n in all (Cauchy), and the variance |d| step^3 <= 2^-21 |c^3 d| each,
        # 2^-21 (15 n)^(1/2) e n^(1/2) in all (the mean of c^6 is 15): within six deviations.
        e, n = 1.4e-5, M * N
        flips = (c.double() - want.to(torch.bfloat16).double()).norm() / want.norm()
        assert flips ** 2 <= 2.0 ** -7 * e + 6 * (2.0 ** -21 * 15 ** 0.5 * e / n) ** 0.5, flips


def _values(q):
    s = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), q["scale"].int() - 127)
    return q["q"].double() * s.repeat_interleave(128, dim=1)[:, :q["q"].shape[1]]


@pytest.mark.parametrize("M,N", [(1, 1), (300, 600), (2000, 4000)])
def test_sums_are_not_cut(B, M, N):
    """65,408 products of 2^-16 behind a product of 1, and in front of it: a sum that were cut as products are would stay at 1."""
    K = 65536
    for first in (True, False):
        a, b = (torch.full((n, K), 2.0 ** -8, device="cuda") for n in (M, N))
        block, one = (slice(0, 128), 0) if first else (slice(K - 128, K), K - 1)
        for x in (a, b):
            x[:, block] = 0
            x[:, one] = 1
        for c_dtype, dt in ((B.ADWIN_DT_F32, torch.float32), (B.ADWIN_DT_BF16, torch.bfloat16)):
            c = _product(B, a, b, 1, 1, "e4m3", c_dtype)[2]
            assert torch.all(c == torch.tensor(1 + (K - 128) * 2.0 ** -16).to(dt)), (first, c_dtype)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype,N,H", [(torch.bfloat16, 13000, 4096), (torch.bfloat16, 1300, 40008), (torch.float32, 9000, 4096),
                                       (torch.float32, 17000, 4104)])
def test_rows_past_the_caches(B, dtype, fmt, N, H):
    """Arrays of more than 96 MiB, of more than 256 in fp32, against calls of fewer rows, whose blocks are the same."""
    x = torch.empty(N, H, device="cuda", dtype=dtype)
    x.copy_(torch.randn(N, H, generator=torch.Generator("cuda").manual_seed(N), device="cuda"))
    x[7, 5], x[N - 1, H - 1] = float("nan"), float("inf")
    f8, step = B.ADWIN_F8_E4M3 if fmt == "e4m3" else B.ADWIN_F8_E5M2, 512
    excluded = (torch.arange(N, device="cuda") % 11 == 3).int()
    for tile in (1, 128):
        for along, across in ((True, False), (True, True)):
            for x_status in (None, excluded):
                got = B.adwin_opd_block_rows(x, tile=tile, f8=f8, along=along, across=across, row_status=True, x_status=x_status)
                for lo in range(0, N, step):
                    hi = min(lo + step, N)
                    want = B.adwin_opd_block_rows(x[lo:hi], tile=tile, f8=f8, along=along, across=across, row_status=True,
                                                  x_status=None if x_status is None else x_status[lo:hi])
                    for name, t in want.items():
                        if name.endswith("_t"):
                            at = lo // (1 if name == "q_t" else 128)
                            part = got[name][:, at:at + t.shape[1]]
                        else:
                            at = lo // (tile if name == "scale" else 1)
                            part = got[name][at:at + t.shape[0]]
                        assert torch.equal(part.contiguous().view(torch.uint8), t.contiguous().view(torch.uint8)), (name, tile, across, lo)
