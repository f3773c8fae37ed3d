"""Equal beams in any order of memory: the same logits give the same bits wherever their rows begin, so that beams of the same logits and
scores rank by rising beam, exactly."""
import pytest
import torch

from .test_gpu_beam import NAMES
from .test_gpu_score import _gen, _strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2605_28396_amd import binding
    return binding


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,K,V,size,temperature,power", [(2, 6, 4001, 2.0, 1.0, 0.0), (1, 4, 50257, 2.0, 0.7, 0.6), (1, 4, 50257, 2.0, 1e-7, 0.0),
                                                          (5, 64, 2003, 2.0, 1.0, 0.6), (1, 9, 7, 2.0, 1.0, 0.0), (2, 3, 4001, 3e7, 1.0, 0.0),
                                                          (1, 16, 9, 0.5, 1.3, 0.0), (300, 2, 8191, 4.0, 1.0, 1.0)])
def test_equal_beams_rank_by_rising_beam_wherever_their_rows_begin(B, dtype, n, K, V, size, temperature, power):
    row = (size * torch.randn(1, V, generator=_gen(V, K))).to(dtype)
    row[0, V // 3] = size * 8                                        # one best token
    z = row.repeat(n * K, 1)
    score = torch.full((n, K), -1.25).cuda()
    length = torch.full((n, K), 7, dtype=torch.int32).cuda()
    per = 16 // z.element_size()
    first = None
    for pad in (0, 1, per - V % per):                                # rows one after the other, and all alike
        for shift in range(per):
            got = B.adwin_opd_beam_select(_strided(z, pad, shift), score, K, temperature=temperature, length=length, length_power=power)
            assert got["parent"].tolist() == [list(range(K))] * n, (pad, shift)
            assert torch.all(got["token"] == V // 3), (pad, shift)
            first = got if first is None else first
            for name in NAMES:
                assert torch.equal(got[name], first[name]), (name, pad, shift)
