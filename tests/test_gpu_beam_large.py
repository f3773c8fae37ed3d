"""Decoding by beams past the caches, and moves of every number of beams: against smaller calls, whose results are the same bits, and
against indexing."""
import pytest
import torch

from .test_gpu_beam import NAMES
from .test_gpu_score import _gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2605_28396_amd import binding
    return binding


@pytest.mark.parametrize("dtype,n,V", [(torch.bfloat16, 320, 151936), (torch.bfloat16, 320, 150001), (torch.float32, 192, 151936),
                                       (torch.float32, 192, 149999)])
def test_logits_past_the_caches(B, dtype, n, V):
    """More than 320 MiB of logits against calls of 64 sequences, which have as many rows to a piece of work."""
    K, keep, step = 4, 8, 64
    z = torch.empty(n * K, V, dtype=dtype, device="cuda")
    z.copy_(torch.randn(n * K, V, generator=torch.Generator("cuda").manual_seed(V), device="cuda") * 2)
    assert z.numel() * z.element_size() > 320 << 20
    z[5, 100:] = -torch.inf
    z[9, V - 1] = torch.nan
    score = -3 * torch.rand(n, K, generator=_gen(n)).cuda()
    finished = (torch.rand(n, K, generator=_gen(n, 1)) < 0.1).int().cuda()
    length = torch.randint(0, 40, (n, K), generator=_gen(n, 2), dtype=torch.int32).cuda()
    kw = dict(temperature=0.8, end=17, length_power=0.6, row_status=True)
    got = B.adwin_opd_beam_select(z, score, keep, finished=finished, length=length, **kw)
    for lo in range(0, n, step):
        hi = lo + step
        want = B.adwin_opd_beam_select(z[K * lo:K * hi], score[lo:hi], keep, finished=finished[lo:hi], length=length[lo:hi], **kw)
        for name in (*NAMES, "row_status"):
            assert torch.equal(got[name][lo:hi], want[name]), (name, lo)


def _indexed(x, y, parent, K, length):
    """y [n keep, P, E] after the move of x [n K, P, E]."""
    n, keep = parent.shape
    x, y = x.view(n, K, *x.shape[1:]), y.view(n, keep, *y.shape[1:])
    take = torch.take_along_dim(x, parent.clamp(0, K - 1).long()[:, :, None, None].expand(n, keep, *x.shape[2:]), dim=1)
    moves = ((parent >= 0) & (parent < K))[:, :, None, None]
    if length is not None:
        moves = moves & (torch.arange(x.shape[2], device=x.device)[None, None, :, None] < length[:, None, None, None])
    return torch.where(moves, take, y).flatten(0, 1)


@pytest.mark.parametrize("K,keep", [(3, 3), (5, 8), (8, 5), (16, 16), (17, 17), (20, 32), (32, 32), (33, 33), (64, 64), (4, 64)])
@pytest.mark.parametrize("large", [False, True])
def test_moves_of_every_number_of_beams(B, K, keep, large):
    """Widths of 16 bytes with bytes left over behind the last, in place and into other arrays; `large`: past the caches."""
    n, E = 5, 20                                                     # positions of 40 bytes, two of them whole vectors of 16
    P = (360 << 20) // (n * keep * 2 * E) // 2 * 2 if large else 206
    g = torch.Generator("cuda").manual_seed(K + 100 * keep)

    def state(rows):
        x = torch.empty(rows, P + 2, E, dtype=torch.bfloat16, device="cuda")
        x.view(torch.int16).random_(-30000, 30000, generator=g)
        return x[:, :P - 1]
    parent = torch.randint(-1, K + 1, (n, keep), generator=_gen(K, keep), dtype=torch.int32).cuda()
    length = torch.tensor([P, P // 3, 0, P - 2, 7], dtype=torch.int32, device="cuda")
    x, y = state(n * K), state(n * keep)
    for l in (None, length):
        out = state(n * keep).copy_(y)
        B.adwin_opd_beam_reorder([x], parent, l, out=[out])
        assert torch.equal(out.view(torch.int16), _indexed(x.view(torch.int16), y.view(torch.int16), parent, K, l)), l
        if K == keep:
            at = state(n * K).copy_(x)
            B.adwin_opd_beam_reorder([at], parent, l)
            assert torch.equal(at.view(torch.int16), _indexed(x.view(torch.int16), x.view(torch.int16), parent, K, l)), ("in place", l)
