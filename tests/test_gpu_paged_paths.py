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


def _random_cache(rng, pages, heads, page):
    """Any codes, scales between 0.05 and 1.6 of both signs: every token is one."""
    ref = pu.Cache(pages, heads, page, rng, stale_nan=False)
    s = rng.integers(0x15, 0x3D, ref.b[..., 2048:].shape) | 0x80 * (rng.random(ref.b[..., 2048:].shape) < 0.1)
    ref.b[..., 2048:] = s.astype(np.uint8)
    return ref


def _tokens(ref, slots, h):
    """What ref.tokens gives, all tokens at once."""
    slots = np.asarray(slots)
    flat = ref.b[slots // ref.page, h].reshape(len(slots), -1)
    out = []
    for value in (False, True):
        at = np.stack([pu.places(t, value)[0] for t in range(ref.page)])[slots % ref.page]
        sh = np.stack([pu.places(t, value)[1] for t in range(ref.page)])[slots % ref.page]
        sc = np.array([pu.scale_place(t, value) for t in range(ref.page)])[slots % ref.page]
        c = (np.take_along_axis(flat, at, 1) >> sh & 15).astype(int) - 8
        out.append((c, pu.E4M3[flat[np.arange(len(slots)), sc]][:, None]))
    (kc, ks), (vc, vs) = out
    return kc * ks, vc * vs, kc, ks, vs


def _check_rows(ref, table, lens, q, qs, Hkv, got, scale, rows, pre=(), prefix=0):
    """Rows (sequence, query head) against 64 bits."""
    G = q.shape[1] // Hkv
    for b, r in rows:
        slots = [int(pre[t // ref.page]) * ref.page + t % ref.page for t in range(prefix)] + [int(table[b, t // ref.page]) * ref.page + t % ref.page for t in range(lens[b])]
        o, tol = pu.attention(q[b, r], qs[b, r], *_tokens(ref, slots, r // G), scale)
        mine = got[b, r].double().cpu().numpy()
        assert (np.abs(mine - o) <= tol).all(), (b, r)


def _parts(fq, B, Hq, Hkv, most, prefix=0):
    n = fq.fq_kv4_attention_workspace_bytes(B, Hq, Hkv, most, prefix)
    assert n % (B * Hq * 520) == 0
    return n // (B * Hq * 520)


def _own(table_rows, lens, page, width, first):
    """A table whose sequences take pages one behind the other from `first` on."""
    table = np.full((table_rows, width), -3, np.int32)
    for b, n in enumerate(lens):
        need = -(-n // page)
        table[b, :need] = first + np.arange(need)
        first += need
    return table, first


@pytest.mark.parametrize("B, Hq, Hkv, prefix, longest, parts", [
    (40, 1, 1, 9700, 1000, 38 + 4),                       # the joining kernel by a workgroup a row, prefix parts and own ones
    (33, 32, 8, 8000, 3000, 11 + 3), (200, 16, 4, 520, 2200, 3 + 2),          # (by a wave a row)
    (32, 1, 1, 20000, 30, 79 + 1)])                       # one own part, and more of the prefix than its kernel adds
def test_a_grouped_prefix_and_own_tokens_that_are_joined(fq, B, Hq, Hkv, prefix, longest, parts):
    rng = np.random.default_rng(B)
    page = 32
    lens = [min(longest, int(n)) for n in rng.integers(0, 40, B)]
    lens[:4] = [longest, 0, longest // 2, min(longest, 17)]
    assert _parts(fq, B, Hq, Hkv, longest, prefix) == parts       # (the path that is meant, on 256 compute units)
    shared = -(-prefix // page)
    table, pages = _own(B, lens, page, -(-longest // page) + 3, shared)
    ref = _random_cache(rng, pages, Hkv, page)
    pre = rng.permutation(shared).astype(np.int32)
    q, qs = _queries(rng, B, Hq, 1.5)
    Q, S, C, P, T, L = _gpu(q, qs, ref.b, pre, table, np.array(lens, np.int32))
    got = fq.fq_kv4_attention_prefix(Q, S, C, P, prefix, T, L, 0.1, max_len=longest)
    rows = [(b, r) for b in {0, 1, 2, 3, B - 1, *rng.integers(0, B, 4).tolist()} for r in sorted({0, Hq - 1, int(rng.integers(0, Hq))})]
    _check_rows(ref, table, lens, q, qs, Hkv, got, 0.1, rows, pre, prefix)
    again = fq.fq_kv4_attention_prefix(Q, S, C, P, prefix, T, L, 0.1, max_len=longest)
    assert torch.equal(got.view(torch.int16), again.view(torch.int16))
    # one sequence with a bad page, one that is too long: NaN, and the others as they were
    table[2, 3] = pages
    lens[5] = longest + 1
    T, L = _gpu(table, np.array(lens, np.int32))
    bad = fq.fq_kv4_attention_prefix(Q, S, C, P, prefix, T, L, 0.1, max_len=longest)
    off = [5] + ([2] if longest // 2 > 3 * page else [])
    on = [b for b in range(B) if b not in off]
    assert bool(torch.isnan(bad[off].float()).all()) and torch.equal(bad[on].view(torch.int16), got[on].view(torch.int16))


def test_waves_over_more_pages_than_a_register_holds(fq):
    """Parts of 1024 tiles, 256 a wave, each tile a page: page numbers are fetched four times and more."""
    rng = np.random.default_rng(31)
    B, Hq, Hkv, page, bound = 2, 3, 1, 16, 1 << 20
    lens = [17003, 5000]
    assert _parts(fq, B, Hq, Hkv, bound) == 64
    table, pages = _own(B, lens, page, bound // page, 0)
    order = rng.permutation(pages)
    table = np.where(table >= 0, order[np.maximum(table, 0)], table).astype(np.int32)
    ref = _random_cache(rng, pages, Hkv, page)
    q, qs = _queries(rng, B, Hq, 1.5)
    Q, S, C, T, L = _gpu(q, qs, ref.b, table, np.array(lens, np.int32))
    got = fq.fq_kv4_attention(Q, S, C, T, L, 0.1)
    _check_rows(ref, table, lens, q, qs, Hkv, got, 0.1, [(b, r) for b in range(B) for r in range(Hq)])
    for at in (70, 300, 17003 // 16):                      # a page number outside the cache, behind a wave's first 64
        for number in (-1, pages):
            T[0, at], was = number, int(T[0, at])
            bad = fq.fq_kv4_attention(Q, S, C, T, L, 0.1)
            T[0, at] = was
            assert bool(torch.isnan(bad[0].float()).all()) and torch.equal(bad[1].view(torch.int16), got[1].view(torch.int16)), at
    T[0, 17003 // 16 + 1] = pages                          # ... and behind the length
    assert torch.equal(fq.fq_kv4_attention(Q, S, C, T, L, 0.1).view(torch.int16), got.view(torch.int16))


def test_prefix_waves_over_more_pages_than_a_register_holds(fq):
    """The same for the prefix's kernel: two parts of 632 tiles for 256 groups of rows, 158 pages a wave."""
    rng = np.random.default_rng(32)
    B, H, page, prefix = 1024, 8, 16, 20000
    lens = [int(n) for n in rng.integers(0, 4, B)]
    assert _parts(fq, B, H, H, 3, prefix) == 2
    shared = prefix // page
    table, pages = _own(B, lens, page, 1, shared)
    ref = _random_cache(rng, pages, H, page)
    pre = rng.permutation(shared).astype(np.int32)
    q, qs = _queries(rng, B, H, 1.5)
    Q, S, C, P, T, L = _gpu(q, qs, ref.b, pre, table, np.array(lens, np.int32))
    got = fq.fq_kv4_attention_prefix(Q, S, C, P, prefix, T, L, 0.1, max_len=3)
    _check_rows(ref, table, lens, q, qs, H, got, 0.1, [(0, 0), (1, 7), (31, 3), (32, 3), (1023, 7), (700, 5)], pre, prefix)
    P[200] = -1
    assert bool(torch.isnan(fq.fq_kv4_attention_prefix(Q, S, C, P, prefix, T, L, 0.1, max_len=3).float()).all())


@pytest.mark.parametrize("B, Hq, Hkv, longest, parts", [(17, 8, 8, 4000, 2), (32, 8, 8, 2100, 2), (20, 32, 8, 33000, 17), (3, 40, 2, 30000, 20)])
def test_uneven_batches_of_129_to_256_heads_and_fewer(fq, B, Hq, Hkv, longest, parts):
    """One long sequence among short ones, in parts."""
    rng = np.random.default_rng(B)
    page = 48
    lens = [int(n) for n in rng.integers(0, 70, B)]
    lens[B // 2] = longest
    assert _parts(fq, B, Hq, Hkv, longest) == parts
    table, pages = _own(B, lens, page, -(-longest // page) + 1, 0)
    ref = _random_cache(rng, pages, Hkv, page)
    q, qs = _queries(rng, B, Hq, 1.5)
    got = fq.fq_kv4_attention(*_gpu(q, qs, ref.b, table, np.array(lens, np.int32)), 0.1, max_len=longest)
    rows = [(b, r) for b in sorted({0, B // 2, B - 1}) for r in sorted({0, Hq - 1, Hq // 2})]
    _check_rows(ref, table, lens, q, qs, Hkv, got, 0.1, rows)
