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


@pytest.mark.parametrize("seqs, Hq, Hkv", [([(4, 300)], 4, 2), ([(4, 1500), (3, 900)], 4, 1), ([(9, 300)], 4, 2), ([(70, 400)], 4, 2)])
@pytest.mark.parametrize("at", [40, 100, 140, 200])
@pytest.mark.parametrize("scale", [1e5, 1e7, 1e30])
def test_rows_beside_those_whose_scores_pass_the_range(fq, seqs, Hq, Hkv, at, scale):  # noqa: F811
    """Scores of 10^8 to 10^36: no other row of the wave is the worse for them."""
    b = Batch(seqs, Hq, Hkv, 16, 83)
    odd = np.arange(b.T) % 3 == 0
    b.qs[odd] = scale
    for early in (odd, ~odd):
        first = np.where(early, 0, at).astype(np.int32)
        end = np.concatenate([np.full(k, n) for k, n in seqs]).astype(np.int32)
        rows = [i for i in range(b.T) if (i % 13 < 2 or i == b.T - 1) and not odd[i]]
        for cap, bias in ((0.0, False), (1e20, False), (0.0, True), (1e10, True)):
            slopes = np.linspace(0.5, 0.0, Hq).astype(np.float32) if bias else None
            out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, first=torch.as_tensor(first).cuda(), end=torch.as_tensor(end).cuda(), cap=cap,
                                            slopes=None if slopes is None else torch.as_tensor(slopes).cuda())
            b.check(out, first=first, end=end, rows=rows, cap=cap, slopes=slopes)


@pytest.mark.parametrize("seqs", [[(4, 1)], [(20, 9), (4, 1)], [(70, 30)]])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 5, 2 ** 30])
def test_the_longest_windows_of_rows_before_the_first_token(fq, seqs, window):  # noqa: F811
    """Fewer cached than new tokens and an end of their own: rows whose place is negative see what a window leaves, which is all."""
    b = Batch(seqs, 4, 2, 16, 89)
    end = np.concatenate([np.full(k, n) for k, n in seqs]).astype(np.int32)
    out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, end=torch.as_tensor(end).cuda(), window=window)
    b.check(out, end=end, window=window)
    b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, window=window), window=window)


def test_rows_past_the_threads_of_a_grid_in_parts(fq):  # noqa: F811
    """2^24 rows, of which one sequence has a few, in more parts than a wave joins."""
    b = Batch([(1, 2310)], 32, 1, 32, 101)
    q, qs, cache, table, starts, lens = b.gpu()
    want = fq.fq_kv4_attention_chunk(q, qs, cache, table, starts, lens, SCALE, max_new=1, max_len=2310)
    T = 1 << 19
    need = fq.fq_kv4_attention_chunk_workspace_bytes(T, 1, 32, 1, 1, 2310)
    assert need // (T * 32 * 520) > 8
    far = torch.empty((T, 32, 128), dtype=torch.uint8, device="cuda"), torch.empty((T, 32), device="cuda")
    out = torch.full((T, 32, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    try:
        for at in (0, 123457, T - 1):
            far[0][at], far[1][at] = q[0], qs[0]
            fq.fq_kv4_attention_chunk(*far, cache, table, starts + at, lens, SCALE, max_new=1, max_len=2310, out=out)
            assert torch.equal(out[at].view(torch.int16), want[0].view(torch.int16))
            out[at] = 7.0
            assert all(bool((x == 7.0).all()) for x in out.split(1 << 17))   # rows of no sequence
    finally:
        del far, out
        torch.cuda.empty_cache()


@pytest.mark.parametrize("seqs", [[(1, 60), (9, 120)], [(70, 150)]])
@pytest.mark.parametrize("cap", [2.0 ** 99, 2.0 ** 100, 1e35, 1e38, 2e38, 3.4e38])
def test_caps_up_to_the_largest_number(fq, seqs, cap):  # noqa: F811
    b = Batch(seqs, 4, 2, 16, 97)
    b.qs[::2] *= 1e-3
    b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, cap=cap), cap=cap)


@pytest.mark.parametrize("seqs, Hq, Hkv", [([(64, 2600)], 4, 1), ([(40, 1500)], 4, 2), ([(90, 1900), (45, 700)], 2, 1)])
@pytest.mark.parametrize("cap, bias", [(25.0, False), (0.0, True), (25.0, True)])
def test_capped_and_biased_chunks_in_parts(fq, seqs, Hq, Hkv, cap, bias):  # noqa: F811
    """A few query tiles over some thousand tokens: as many parts as fill the device once or twice."""
    b = Batch(seqs, Hq, Hkv, 32, 107)
    slopes = np.linspace(0.3, 0.0, Hq).astype(np.float32) if bias else None
    rows = [i for i in range(b.T) if i % 17 < 2 or i == b.T - 1]
    for max_len in (max(n for _, n in seqs), 9000):
        out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, max_new=max(k for k, _ in seqs), max_len=max_len, cap=cap, slopes=None if slopes is None else torch.as_tensor(slopes).cuda())
        b.check(out, cap=cap, slopes=slopes, rows=rows)


@pytest.mark.parametrize("cap, bias, window", [(0.0, False, 0), (20.0, False, 300), (0.0, True, 0)])
def test_a_chunk_beside_single_tokens_of_long_caches(fq, cap, bias, window):  # noqa: F811
    """One sequence brings more rows than a query tile holds, the others one token each at lengths from one to some thousand."""
    b = Batch([(1, 2600), (200, 700), (1, 1), (1, 1300), (0, 500), (2, 1900)], 4, 2, 32, 103)
    slopes = np.float32([0.5, 0.05, 0.005, 0.0]) if bias else None
    rows = [i for i in range(b.T) if i % 29 < 2 or i > 200]
    shape = dict(cap=cap, window=window, slopes=None if slopes is None else torch.as_tensor(slopes).cuda())
    for kw in ({}, {"max_new": 200, "max_len": 2600}, {"max_new": 1}):
        b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, **shape, **kw), cap=cap, window=window, slopes=slopes, rows=rows)
    # a call for each run of sequences of one kind, into the same rows
    q, qs, cache, table, starts, lens = b.gpu()
    out = torch.full((b.T, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    for lo, hi, new in ((0, 1, 1), (1, 2, 200), (2, 6, 1)):
        fq.fq_kv4_attention_chunk(q, qs, cache, table[lo:hi], starts[lo:hi + 1], lens[lo:hi], SCALE, max_new=new, out=out, **shape)
    b.check(out, cap=cap, window=window, slopes=slopes, rows=rows)
