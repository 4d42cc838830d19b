"""Attention of new tokens (fireq_chunk.h) at the ends of its arguments: scales, windows, caps and row counts; long and short sequences in one batch."""
import numpy as np
import pytest
import torch

from test_gpu_chunk import Batch, SCALE, fq  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs, Hq, Hkv", [([(4, 300)], 4, 2), ([(4, 1500), (3, 900)], 4, 1), ([(9, 300)], 4, 2), ([(70, 400)], 4, 2)])
@pytest.mark.parametrize("at", [40, 100, 140, 200])
@pytest.mark.parametrize("scale", [0.0, 1e-38, 3e-32])
def test_scales_next_to_zero_beside_rows_that_begin_later_and_earlier(fq, seqs, Hq, Hkv, at, scale):  # noqa: F811
    """A row whose scores are all alike keeps its weights when rows with other ranges, worked on beside it, take theirs."""
    b = Batch(seqs, Hq, Hkv, 16, 83)
    odd = np.arange(b.T) % 3 == 0
    b.qs[odd] = scale
    for early in (odd, ~odd):
        first = np.where(early, 0, at).astype(np.int32)
        end = np.concatenate([np.full(k, n) for k, n in seqs]).astype(np.int32)
        rows = [i for i in range(b.T) if i % 13 < 2 or i == b.T - 1]
        out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, first=torch.as_tensor(first).cuda(), end=torch.as_tensor(end).cuda())
        assert torch.isfinite(out.float()).all()
        b.check(out, first=first, end=end, rows=rows)
