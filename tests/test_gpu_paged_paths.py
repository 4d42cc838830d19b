"""Paged cache and attention on the GPU: what lies over what, and the paths that sizes and bounds choose."""
import numpy as np
import pytest

import paged_util as pu
from test_gpu_paged import _check_attention, _filled, _queries, _rotation, fq  # noqa: F401 (fq: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _gpu(*arrays):
    return [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


def test_outputs_over_inputs_are_refused_and_between_tiles_are_not(fq):
    rng = np.random.default_rng(21)
    lens, page = [70, 33], 32
    ref, table, _ = _filled(rng, lens, 2, page)
    q, qs = _queries(rng, 2, 4, 1)
    pool = torch.zeros((ref.b.shape[0], 3, 2, page // 16, 2080), dtype=torch.uint8, device="cuda")
    cache = pool[:, 1]
    cache.copy_(torch.from_numpy(ref.b))
    buf = torch.empty(2 * 4 * 256, dtype=torch.uint8, device="cuda")
    Q = buf[:1024].view(2, 4, 128)
    Q.copy_(torch.from_numpy(q))
    S, T, L = _gpu(qs, table, np.array(lens, np.int32))
    want = fq.fq_kv4_attention(Q, S, cache, T, L, 0.1)
    _check_attention(ref, table, lens, q, qs, 2, want, 0.1)
    for out in (buf.view(torch.bfloat16).view(2, 4, 128), pool[1, 1].view(-1)[:2048].view(torch.bfloat16).view(2, 4, 128)):
        with pytest.raises(fq.FireqError):
            fq.fq_kv4_attention(Q, S, cache, T, L, 0.1, out=out)
    other = pool[1, 2].view(-1)[:2048].view(torch.bfloat16).view(2, 4, 128)    # another layer's page
    assert torch.equal(fq.fq_kv4_attention(Q, S, cache, T, L, 0.1, out=other).view(torch.int16), want.view(torch.int16))
    assert np.array_equal(cache.cpu().numpy(), ref.b)
