"""Rows that a head leaves out, forward and backward, and what its gradients say of infinities and NaN.

Blocks of an excluded row are those of a row of zeros, exactly; so gradients are held to those of rows of zeros, bit by bit, and to the
formula in 64 bits with the tolerance of products (test_gpu_block)."""
import math

import pytest
import torch

from .test_gpu_block import F8, U, _gen, _strided, blocks, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2605_28396_amd import binding
    return binding


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,H,pad,shift", [(1, 5, 0, 0), (3, 128, 0, 0), (130, 640, 0, 0), (300, 1003, 0, 0), (257, 513, 3, 1), (5, 9001, 0, 0)])
def test_excluded_rows_are_zeros(B, dtype, N, H, pad, shift):
    x = torch.randn(N, H, generator=_gen(N, H)).to(dtype)
    status = torch.zeros(N, dtype=torch.int32)
    status[::3] = torch.tensor([2, -1, 1 << 30], dtype=torch.int32).repeat(N)[:len(status[::3])]
    zeros = torch.where((status != 0)[:, None], torch.zeros((), dtype=dtype), x)
    x[0] = math.nan                                                  # excluded rows hold anything
    x[3 if N > 3 else 0, H // 2] = torch.finfo(dtype).max
    word = status.clone()
    if N > 4:
        x[4, 1] = zeros[4, 1] = math.inf
        word[4] = B.ADWIN_DEV_NONFINITE
    for f8 in (B.ADWIN_F8_E4M3, B.ADWIN_F8_E5M2):
        for tile in (1, 128):
            for along, across in ((True, False), (True, True), (False, True)):
                kw = dict(tile=tile, f8=f8, along=along, across=across, row_status=True)
                got = B.adwin_opd_block_rows(_strided(x, pad, shift), x_status=status.cuda(), **kw)
                want = B.adwin_opd_block_rows(_strided(zeros, pad, shift), **kw)
                for name in want:
                    if name == "row_status":
                        assert torch.equal(got[name].cpu(), word), (tile, along, across)
                    else:
                        assert torch.equal(got[name].view(torch.uint8), want[name].view(torch.uint8)), (name, tile, along, across)
                kw["row_status"] = False
                got = B.adwin_opd_block_rows(_strided(x, pad, shift), x_status=status.cuda(), **kw)
                for name in got:
                    assert torch.equal(got[name].view(torch.uint8), want[name].view(torch.uint8)), (name, tile, along, across)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("h_dtype,z_dtype", [(torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("V,H,T", [(1003, 300, 200), (1024, 256, 77), (300, 129, 5)])
def test_gradients_leave_out_what_the_logits_left_out(B, fmt, h_dtype, z_dtype, V, H, T):
    f8 = B.ADWIN_F8_E4M3 if fmt == "e4m3" else B.ADWIN_F8_E5M2
    head = B.BlockHead(torch.randn(V, H, generator=_gen(V)).cuda() * 0.1, gradients=True)
    h = torch.randn(T, H, generator=_gen(T, H)).to(h_dtype).cuda()
    dz = (torch.randn(T, V, generator=_gen(T, V)) / T).to(z_dtype).cuda()
    left, wrong = [1, T - 2], [0, T // 2]
    h[1, 7] = math.nan
    h[T - 2, H - 1] = -math.inf
    dz[1] = 1e30                                                     # a row that is left out holds anything
    dz[0, 5], dz[T // 2, V - 1] = math.inf, math.nan
    _, status = head.logits(h, row_status=True)
    assert status.nonzero().flatten().tolist() == left
    out = head.grad(dz, h, f8=f8, dh_dtype=B.ADWIN_DT_F32, status=status, row_status=True)
    word = B.ADWIN_DEV_NONFINITE
    assert out["dz_status"].tolist() == [word if t in left + wrong else 0 for t in range(T)]
    assert out["h_status"].tolist() == [word if t in left else 0 for t in range(T)]
    assert torch.all(out["dh"][left] == 0)
    # the same of rows of zeros, bit by bit
    dz0, h0 = torch.where(dz.isfinite(), dz, 0), h.clone()
    dz0[left] = 0
    h0[left] = 0
    same = head.grad(dz0, h0, f8=f8, dh_dtype=B.ADWIN_DT_F32, row_status=True)
    assert torch.equal(out["dh"], same["dh"]) and torch.equal(out["dW"], same["dW"])
    assert not same["dz_status"].any() and not same["h_status"].any()
    # the sum over the other tokens
    dt = values(*blocks(dz0.cpu().float().t(), 1, fmt)[:2], 1).cuda()[:, :T]
    ht = values(*blocks(h0.cpu().float().t(), 1, "e4m3")[:2], 1).cuda()[:, :T]
    want, S = dt @ ht.t(), dt.abs() @ ht.abs().t()
    assert torch.all((out["dW"].double() - want).abs() <= (T / 8 + 64) * 2 * U * S + 1e-37)
    # each way by itself, and without the words
    only = head.grad(dz, f8=f8, dh_dtype=B.ADWIN_DT_F32, status=status, row_status=True)
    assert set(only) == {"dh", "dz_status"} and torch.equal(only["dh"], out["dh"]) and torch.equal(only["dz_status"], out["dz_status"])
    only = head.grad(dz, h, f8=f8, want_dh=False, status=status)
    assert set(only) == {"dW"} and torch.equal(only["dW"], out["dW"])


def test_no_tokens(B):
    head = B.BlockHead(torch.randn(300, 129, generator=_gen(1)).cuda(), gradients=True)
    e = torch.empty(0, 300, device="cuda"), torch.empty(0, 129, device="cuda")
    out = head.grad(*e, status=torch.empty(0, dtype=torch.int32, device="cuda"), row_status=True)
    assert out["dh"].shape == (0, 129) and out["dW"].abs().max() == 0 and out["dz_status"].shape == out["h_status"].shape == (0,)


def test_words_of_other_sizes_and_types_are_refused(B):
    head = B.BlockHead(torch.randn(300, 129, generator=_gen(1)).cuda(), gradients=True)
    dz, h = torch.randn(9, 300, generator=_gen(2)).cuda(), torch.randn(9, 129, generator=_gen(3)).cuda()
    for bad in (torch.zeros(8, dtype=torch.int32).cuda(), torch.zeros(9).cuda(), torch.zeros(9, dtype=torch.int32),
                torch.zeros(18, dtype=torch.int32).cuda()[::2]):
        with pytest.raises(ValueError):
            head.grad(dz, h, status=bad)
    word = torch.zeros(9, dtype=torch.int32).cuda()
    with pytest.raises(B.AdwinError):                                # the words that are asked for and those that are written
        B.adwin_opd_block_rows(dz, row_status=word, x_status=word)


def test_captured_gradients_take_the_words_of_every_replay(B):
    V, H, T = 515, 260, 150
    head = B.BlockHead(torch.randn(V, H, generator=_gen(5)).cuda() * 0.1, gradients=True)
    hs = [torch.randn(T, H, generator=_gen(6, k)).to(torch.bfloat16).cuda() for k in range(3)]
    ds = [torch.randn(T, V, generator=_gen(7, k)).cuda() for k in range(3)]
    hs[1][5, 5] = math.nan; hs[2][140] = math.inf; ds[2][3, 3] = math.nan

    def step(h, d):
        z, status = head.logits(h, row_status=True)
        return {"z": z, **head.grad(d, h, status=status, row_status=True)}
    want = [step(h, d) for h, d in zip(hs, ds)]
    h, d, side = hs[0].clone(), ds[0].clone(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(h, d)
    for k in (1, 2, 0, 1):
        h.copy_(hs[k]); d.copy_(ds[k])
        graph.replay()
        eager = step(hs[(k + 1) % 3], ds[(k + 1) % 3])
        torch.cuda.synchronize()
        for name in got:
            assert torch.equal(got[name], want[k][name]) and torch.equal(eager[name], want[(k + 1) % 3][name]), (k, name)
