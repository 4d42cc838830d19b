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


def _attention_within(q, q_scale, K, V, kc, ks, vs, out_scale):
    """pu.attention with the score's error counted as include/fireq_paged.h states it: 2^-12 of the largest term of the zero-point form, the
    zero point's own 8 |q| among them (a channel of code -8 has no product)."""
    o, tol = pu.attention(q, q_scale, K, V, kc, ks, vs, out_scale)
    f = float(q_scale) * out_scale
    s = K @ pu.E4M3[q] * f
    p = np.exp(s - s.max())
    e = 2.0 ** -12 * (np.abs(pu.E4M3[q])[None, :] * np.maximum(kc + 8, 8)).max(1) * np.abs(ks[:, 0]) * f
    return o, tol + ((p * e) @ np.abs(V) + (p * e).sum() * np.abs(o)) / p.sum()


@pytest.mark.parametrize("low", [3, 7, 11])
def test_scores_of_queries_with_an_outlier(fq, low):
    """One channel 2^low above the others: the others' products lose their last bits, by no more than the header says."""
    rng = np.random.default_rng(low)
    lens = [2, 40, 333, 17, 64, 9]
    ref, table, _ = _filled(rng, lens, 1, 16)
    for b, n in enumerate(lens):                          # the outlier's codes are one number in all tokens, the lowest or the highest too
        for t in range(n):
            slot = int(table[b, t // 16]) * 16 + t % 16
            codes, sc = ref.get(slot, 0, False)
            codes[77] = (-8, 7, 0)[b % 3]
            ref.put(slot, 0, False, codes, 0x38)
    x = rng.standard_normal((len(lens), 16, 128)) * 2.0 ** -low
    x[..., 77] = np.sign(x[..., 77])
    qs = (np.abs(x).max(-1) / 448).astype(np.float32)
    q = pu.to_e4m3((x / qs[..., None]).astype(np.float32))
    qs *= np.float32(2.0 ** low)
    got = fq.fq_kv4_attention(*_gpu(q, qs, ref.b, table, np.array(lens, np.int32)), 0.02).double().cpu().numpy()
    for b, n in enumerate(lens):
        kv = list(ref.tokens([int(table[b, t // 16]) * 16 + t % 16 for t in range(n)], 0))
        for r in range(16):
            o, tol = _attention_within(q[b, r], qs[b, r], *kv, 0.02)
            assert (np.abs(got[b, r] - o) <= tol).all(), (b, r)
