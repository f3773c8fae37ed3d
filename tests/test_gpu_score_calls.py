"""How the token-scoring calls of the binding are made: streams, arrays that are kept, rows that are reported."""
import math

import pytest
import torch

from . import test_gpu_score as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2605_28396_amd import binding
    return binding


def test_stream_zero_is_the_default_stream(B, monkeypatch):
    """The handle that the library gets; nothing is enqueued."""
    got = []
    monkeypatch.setattr(B.lib, "adwin_opd_token_logp", lambda p, ws, n, stream: got.append(stream) or 0)
    z, ids = torch.zeros(300, 50, device="cuda"), torch.zeros(300, 1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for s in (None, 0, torch.cuda.default_stream(), side, side.cuda_stream):
            B.adwin_opd_token_logp(z, ids, stream=s)
    assert got == [side.cuda_stream, None, None, side.cuda_stream, side.cuda_stream]
