"""Attention of new tokens (fireq_chunk.h) against 64-bit arithmetic: row counts of every variant, masks, windows, caps, biases, broken tokens."""
import numpy as np
import pytest
import torch

import chunk_util as cu
import paged_util as pu

pytestmark = pytest.mark.gpu
SCALE = 128 ** -0.5


@pytest.fixture(scope="module")
def fq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: torch.cuda.is_available() is False")
    from paper_2505_20839_amd import binding
    return binding


class Batch:
    """Sequences of (new rows, cached tokens) in a pool of pages in any order; what was never cached has NaN scales."""

    def __init__(self, seqs, Hq, Hkv, page, seed, before=0, behind=0):
        rng = np.random.default_rng(seed)
        self.seqs, self.Hq, self.Hkv, self.page = seqs, Hq, Hkv, page
        width = max(1, max(-(-max(n, 0) // page) for _, n in seqs))
        self.cache = pu.Cache(len(seqs) * width + 1, Hkv, page, rng)
        self.table = rng.permutation(len(seqs) * width + 1)[: len(seqs) * width].reshape(len(seqs), width).astype(np.int32)
        for b, (_, n) in enumerate(seqs):
            for t in range(max(n, 0)):
                for h in range(Hkv):
                    for value in (False, True):
                        self.cache.put(int(self.table[b, t // page]) * page + t % page, h, value, np.clip(np.rint(2.7 * rng.standard_normal(128)), -8, 7),
                                       int(pu.to_e4m3(0.37 * np.exp(0.3 * rng.standard_normal()))))
        self.starts = np.concatenate([[before], before + np.cumsum([k for k, _ in seqs])]).astype(np.int32)
        self.T = int(self.starts[-1]) + behind
        x = 2.0 * rng.standard_normal((self.T, Hq, 128)) * np.exp(0.5 * rng.standard_normal((self.T, Hq, 1)))
        self.qs = (np.abs(x).max(-1) / 448).astype(np.float32)
        self.q = pu.to_e4m3(x / self.qs[..., None])
        self.lens = np.array([n for _, n in seqs], np.int32)

    def gpu(self):
        t = lambda x: torch.as_tensor(x).cuda()           # noqa: E731
        return t(self.q), t(self.qs), t(self.cache.b), t(self.table), t(self.starts), t(self.lens)

    def check(self, out, first=None, end=None, window=0, cap=0.0, slopes=None, rows=None):
        """Every row of every sequence (or those of `rows`) within its tolerance."""
        out = out.float().cpu().numpy().reshape(self.T, self.Hq, 128)
        G = self.Hq // self.Hkv
        for b, (k, n) in enumerate(self.seqs):
            a = int(self.starts[b])
            cut = lambda x: None if x is None else x[a:a + k]     # noqa: E731
            want = cu.ranges(k, n, cut(first), cut(end), window)
            slots = [int(self.table[b, t // self.page]) * self.page + t % self.page for t in range(max(n, 0))]
            for h in range(self.Hkv):
                tokens = [x for x in self.cache.tokens(slots, h)]
                for i, (lo, hi) in enumerate(want):
                    if rows is not None and a + i not in rows:
                        continue
                    for j in range(h * G, h * G + G):
                        o, tol = cu.attention(self.q[a + i, j], self.qs[a + i, j], tokens, n - k + i, lo, hi, SCALE, cap, 0.0 if slopes is None else float(slopes[j]))
                        err = np.abs(out[a + i, j] - o)
                        assert (err <= tol).all(), (b, i, j, lo, hi, float((err - tol).max()), float(err.max()))


SHAPES = [
    # (new rows, cached tokens) of each sequence, Hq, Hkv, page
    ([(1, 1)], 1, 1, 16),
    ([(1, 37), (1, 0), (1, 160), (1, 5)], 8, 2, 16),                      # single tokens, one sequence empty
    ([(1, 700)], 20, 1, 32),                                              # more than 16 query heads of a key/value head
    ([(2, 33), (0, 20), (3, 3), (1, 90)], 12, 4, 48),                     # 3 heads each, no rows in one
    ([(5, 200), (4, 64)], 14, 2, 32),                                     # 7 heads: tiles end inside a token
    ([(13, 13), (6, 100)], 4, 2, 16),
    ([(31, 31), (1, 17), (20, 150)], 5, 1, 64),
    ([(70, 300)], 8, 2, 128),
    ([(65, 65), (3, 40), (64, 64)], 4, 4, 16),                            # a head each
    ([(3, 2), (2, -4), (4, 1)], 4, 1, 16),                                # fewer cached than new
    ([(2, 20 + b % 7) for b in range(130)], 8, 8, 16),                    # many sequences
    ([(34, 34 + b % 5) for b in range(33)], 8, 8, 16),                    # as many tiles as fill the device
]


@pytest.mark.parametrize("seqs, Hq, Hkv, page", SHAPES, ids=lambda v: str(len(v)) if isinstance(v, list) else str(v))
@pytest.mark.parametrize("cap, bias, window", [(0.0, False, 0), (2.0, False, 0), (0.0, True, 0), (30.0, True, 9), (0.0, False, 20)])
def test_rows(fq, seqs, Hq, Hkv, page, cap, bias, window):
    b = Batch(seqs, Hq, Hkv, page, 1000 * Hq + page, before=2, behind=3)
    slopes = (2.0 ** (-8.0 * np.arange(1, Hq + 1) / Hq)).astype(np.float32) if bias else None
    out = torch.full((b.T, Hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    r = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, max_new=max(k for k, _ in seqs), max_len=max(max(n for _, n in seqs), 0), window=window, cap=cap,
                                  slopes=None if slopes is None else torch.as_tensor(slopes).cuda(), out=out)
    assert r.data_ptr() == out.data_ptr()
    b.check(out, window=window, cap=cap, slopes=slopes)
    assert (out[: b.starts[0]] == 7.0).all() and (out[b.starts[-1]:] == 7.0).all()        # rows of no sequence


@pytest.mark.parametrize("seqs, Hq, Hkv", [([(40, 70), (1, 9), (33, 33)], 4, 2), ([(4, 50), (3, 3)], 4, 1), ([(1, 90), (1, 40)], 4, 2),
                                           ([(34, 40) for _ in range(33)], 8, 8)])
@pytest.mark.parametrize("kind", ["documents", "prefix", "any"])
@pytest.mark.parametrize("cap, bias, window", [(0.0, False, 0), (1.5, True, 0), (0.0, True, 11)])
def test_ranges(fq, seqs, Hq, Hkv, kind, cap, bias, window):
    """Ranges of rows: documents with padding rows, a prefix seen whole, and any ranges, empty, inverted and past both ends among them."""
    b = Batch(seqs, Hq, Hkv, 16, 7)
    rng = np.random.default_rng(5)
    first, end = np.zeros(b.T, np.int32), np.zeros(b.T, np.int32)
    for s, (k, n) in enumerate(seqs):
        for i in range(k):
            at, pos = int(b.starts[s]) + i, n - k + i
            if kind == "documents":
                pad = pos % 7 == 3
                first[at], end[at] = (pos if pad else pos // 13 * 13), (pos if pad else pos + 1)
            elif kind == "prefix":
                first[at], end[at] = 0, max(pos + 1, n // 2)
            else:
                first[at], end[at] = rng.integers(-20, n + 5), rng.integers(-5, n + 20)
    slopes = np.linspace(0.9, -0.1, Hq).astype(np.float32) if bias else None
    out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, first=torch.as_tensor(first).cuda(), end=torch.as_tensor(end).cuda(), window=window, cap=cap,
                                    slopes=None if slopes is None else torch.as_tensor(slopes).cuda())
    b.check(out, first, end, window, cap, slopes)


@pytest.mark.parametrize("max_new", [1, 5, 40, 1000])
@pytest.mark.parametrize("max_len", [None, 900, 1 << 30])
def test_bounds_that_are_far_off(fq, max_new, max_len):
    """max_new may be anything, and max_len far above the lengths."""
    b = Batch([(20, 300), (1, 900), (7, 7)], 8, 2, 32, 3)
    b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, max_new=max_new, max_len=max_len, cap=20.0), cap=20.0)


def test_long_cache_in_parts(fq):
    """One token and a few over some thousand tokens, in parts joined through memory; window and ranges inside one part."""
    b = Batch([(1, 4001)], 4, 1, 64, 11)
    b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, max_new=1))
    b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, max_new=1, window=33), window=33)
    slopes = np.float32([0.5, 0.05, 0.005, 0.0])
    b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, slopes=torch.as_tensor(slopes).cuda()), slopes=slopes)
    b = Batch([(3, 2500), (2, 17)], 8, 1, 16, 12)
    b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, max_new=3, cap=5.0), cap=5.0)


def test_bias_far_from_the_row(fq):
    """A row whose tokens all lie far away: distances differ by one, and their common part is no error."""
    b = Batch([(2, 400)], 2, 1, 16, 13)
    starts, lens = b.starts.copy(), b.lens.copy()
    first, end = np.int32([0, 3]), np.int32([64, 90])
    slopes = np.float32([0.03, 2.0 ** 10])
    out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, first=torch.as_tensor(first).cuda(), end=torch.as_tensor(end).cuda(), slopes=torch.as_tensor(slopes).cuda())
    assert (starts == b.starts).all() and (lens == b.lens).all()
    b.check(out, first, end, slopes=slopes)


@pytest.mark.parametrize("cap", [1e-3, 0.3, 1e4, 1e20])
def test_caps_of_every_size(fq, cap):
    """Scores far above their cap, about it, and far below (tanh's series, and a capped score that is the score)."""
    b = Batch([(9, 120), (1, 60)], 4, 2, 16, 17)
    b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, cap=cap), cap=cap)


@pytest.mark.parametrize("seqs, Hq, Hkv", [([(24, 24)], 2, 1), ([(4, 40)], 4, 1), ([(80, 80)], 4, 4), ([(34, 34) for _ in range(33)], 8, 8)])
@pytest.mark.parametrize("value", [False, True])
def test_a_broken_token_reaches_only_the_rows_that_see_it(fq, seqs, Hq, Hkv, value):
    b = Batch(seqs, Hq, Hkv, 16, 19)
    k, n = seqs[0]
    bad = n - k // 2                                      # seen by the rows from here on
    slot = int(b.table[0, bad // 16]) * 16 + bad % 16
    b.cache.flat(slot // 16, 0)[pu.scale_place(slot % 16, value)] = 0xFF if value else 0x7F
    out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE)
    sees = [i for i in range(k) if n - k + i >= bad]
    G = Hq // Hkv
    assert sees and len(sees) < k
    assert torch.isnan(out[sees][:, :G]).all() and not torch.isnan(out[sees][:, G:]).any()
    assert not torch.isnan(out[[i for i in range(out.shape[0]) if i not in sees]]).any()
    b.check(out, rows=[i for i in range(k) if i not in sees])


def test_a_page_outside_the_cache(fq):
    """It makes NaN those rows only that attend to its tokens."""
    b = Batch([(50, 50), (1, 40)], 4, 2, 16, 23)
    for page in (-1, 10 ** 6):
        b.table[0, 1] = page                              # tokens 16 .. 31
        out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, window=8)
        sees = [i for i in range(50) if i >= 16 and i - 7 <= 31]
        assert torch.isnan(out[sees]).all()
        assert not torch.isnan(out[[i for i in range(51) if i not in sees]]).any()


def test_lengths_past_the_bounds(fq):
    b = Batch([(3, 30), (3, 64)], 4, 2, 16, 29)
    args = list(b.gpu())
    out = fq.fq_kv4_attention_chunk(*args, SCALE, max_len=40)
    assert not torch.isnan(out[:3]).any() and torch.isnan(out[3:]).all()
    args[3] = args[3][:, :3].contiguous()                 # room for 48
    out = fq.fq_kv4_attention_chunk(*args, SCALE, max_len=64)
    assert not torch.isnan(out[:3]).any() and torch.isnan(out[3:]).all()


def test_starts_outside_the_rows(fq):
    """Starts that run past the rows, or backwards, write nothing outside them."""
    b = Batch([(3, 30), (3, 64), (2, 20)], 4, 2, 16, 31)
    args = list(b.gpu())
    for starts in ([-5, 3, 6, 100], [8, 8, 8, 8], [6, 3, 6, 8], [2 ** 31 - 1, -2 ** 31, 5, 7]):
        args[4] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        pool = torch.full((3 * b.T, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        fq.fq_kv4_attention_chunk(*args, SCALE, out=pool[b.T: 2 * b.T])
        torch.cuda.synchronize()
        assert (pool[: b.T] == 7.0).all() and (pool[2 * b.T:] == 7.0).all()


def test_one_token_agrees_with_the_decode_attention(fq):
    """Single tokens, plain scores: fq_kv4_attention's results but for the order of sums."""
    b = Batch([(1, n) for n in (1, 33, 400, 777, 0)], 8, 2, 32, 37)
    q, qs, cache, table, starts, lens = b.gpu()
    x = fq.fq_kv4_attention(q, qs, cache, table, lens, SCALE).float()
    y = fq.fq_kv4_attention_chunk(q, qs, cache, table, starts, lens, SCALE).float()
    assert ((x - y).abs() <= 2.0 ** -6 * x.abs() + 1e-3).all()


def test_a_slice_of_a_pool_of_layers(fq):
    b = Batch([(20, 50), (1, 33)], 4, 2, 16, 41)
    q, qs, cache, table, starts, lens = b.gpu()
    pool = torch.full((cache.shape[0], 3, 2) + tuple(cache.shape[2:]), 0x7F, dtype=torch.uint8, device="cuda")
    pool[:, 1] = cache
    b.check(fq.fq_kv4_attention_chunk(q, qs, pool[:, 1], table, starts, lens, SCALE))


@pytest.mark.parametrize("seqs, max_new", [([(1, 2000), (1, 30)], 1), ([(40, 600), (5, 5)], 40), ([(34, 40) for _ in range(33)], 34)])
def test_captured_and_on_another_stream(fq, seqs, max_new):
    """Replays with other lengths, rows and codes in the same arrays, eager work of other sizes between them."""
    b = Batch(seqs, 8, 8 if len(seqs) > 9 else 1, 16, 43)
    args = list(b.gpu())
    other = Batch([(3, 100)], 8, 1, 16, 44)
    other_args = other.gpu()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        want = fq.fq_kv4_attention_chunk(*args, SCALE, max_new=max_new, cap=10.0)
    s.synchronize()
    b.check(want, cap=10.0, rows=set(range(0, b.T, 7)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = fq.fq_kv4_attention_chunk(*args, SCALE, max_new=max_new, cap=10.0)
    for i in range(3):
        out.zero_()
        graph.replay()
        fq.fq_kv4_attention_chunk(*other_args, SCALE)
        torch.cuda.synchronize()
        want = fq.fq_kv4_attention_chunk(*args, SCALE, max_new=max_new, cap=10.0)
        assert torch.equal(out, want), i
        args[1].mul_(0.5)
        args[5].sub_(1)


def test_results_are_the_same_every_time(fq):
    b = Batch([(50, 500), (1, 900)], 8, 2, 32, 47)
    args = b.gpu()
    want = fq.fq_kv4_attention_chunk(*args, SCALE)
    for _ in range(5):
        assert torch.equal(fq.fq_kv4_attention_chunk(*args, SCALE), want)


def test_workspace_is_the_callers(fq):
    b = Batch([(1, 3000)], 8, 1, 32, 53)
    need = fq.fq_kv4_attention_chunk_workspace_bytes(1, 1, 8, 1, 1, 3000)
    assert need > 0
    pool = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, max_new=1, max_len=3000, workspace=pool[16: 16 + need])
    b.check(out)
    assert (pool[:16] == 0xFF).all() and (pool[16 + need:] == 0xFF).all()
    with pytest.raises(fq.FireqError):
        fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, max_new=1, max_len=3000, workspace=pool[16: need])


@pytest.mark.parametrize("seqs, Hq, Hkv", [([(1, 30), (1, 1)], 4, 2), ([(1, 700)], 4, 2), ([(9, 40), (2, 90)], 4, 2), ([(80, 90), (3, 70)], 4, 2), ([(40, 900)], 8, 1)])
@pytest.mark.parametrize("kw", [{}, {"cap": 5.0}, {"slopes": True}, {"cap": 5.0, "slopes": True}, {"window": 9}])
@pytest.mark.parametrize("code", [False, True])
def test_a_query_that_is_not_a_number(fq, seqs, Hq, Hkv, kw, code):
    """A NaN scale, or a NaN among the codes: NaN to that row's head, and to nothing else."""
    b = Batch(seqs, Hq, Hkv, 16, 43)
    row = b.T // 2
    if code:
        b.q[row, 1, 77] = 0x7F
    else:
        b.qs[row, 1] = np.nan
    if kw.get("slopes"):
        kw = dict(kw, slopes=torch.full((Hq,), 0.1, device="cuda"))
    out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, **kw).view(b.T, Hq, 128)
    assert torch.isnan(out[row, 1]).all()
    out[row, 1] = 0
    assert not torch.isnan(out).any()


@pytest.mark.parametrize("seqs", [[(1, 200)], [(20, 100)], [(70, 150)]])
@pytest.mark.parametrize("forward", [False, True])
def test_slopes_of_any_size(fq, seqs, forward):
    """Up to the largest finite number, with which the nearest tokens alone count."""
    b = Batch(seqs, 4, 2, 16, 47)
    slopes = np.array([0.0, 1e-30, 1e10, 3.4e38], np.float32)
    end = np.full(b.T, 120 if forward else 90, np.int32)  # (rows whose nearest token lies before them, at them, or behind)
    first = np.full(b.T, 35, np.int32)
    out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, first=torch.as_tensor(first).cuda(), end=torch.as_tensor(end).cuda(), slopes=torch.as_tensor(slopes).cuda())
    b.check(out, first=first, end=end, slopes=slopes)


@pytest.mark.parametrize("starts", [[0, 900, 1000, 0, 0], [0, 1000, 1000, 0, 3], [900, 0, 1000, 10, 1000], [0, 500, 400, 1000, 2], [1000, 900, 0, 1000, 0]])
@pytest.mark.parametrize("max_new", [1, 16, 1000])
def test_starts_that_decrease_far(fq, starts, max_new):
    b = Batch([(1000, 40)] + [(0, 40)] * 3, 4, 2, 16, 53)
    args = list(b.gpu())
    args[4] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    pool = torch.full((3 * b.T, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    fq.fq_kv4_attention_chunk(*args, SCALE, max_new=max_new, out=pool[b.T: 2 * b.T])
    torch.cuda.synchronize()
    assert (pool[: b.T] == 7.0).all() and (pool[2 * b.T:] == 7.0).all()


@pytest.mark.parametrize("seqs, Hq, Hkv", [([(1, 2100)], 4, 2), ([(1, 1500), (1, 90), (1, 2000)], 2, 1), ([(6, 1700)], 4, 1), ([(70, 1900)], 2, 1), ([(45, 1500), (60, 700)], 4, 1)])
@pytest.mark.parametrize("window", [1, 15, 16, 17, 129, 600])
def test_windows_in_parts(fq, seqs, Hq, Hkv, window):
    """Windows far shorter than the sequences, whose tokens are cut into parts by the window's length; a bound that is far off; an end of their own."""
    b = Batch(seqs, Hq, Hkv, 32, 59 + window)
    rows = [i for i in range(b.T) if i % 13 in (0, 5) or i == b.T - 1]
    for max_len in (None, 4096):
        kw = {} if max_len is None else {"max_len": max_len}
        b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, window=window, **kw), window=window, rows=rows)
    end = np.concatenate([np.full(k, n) for k, n in seqs]).astype(np.int32)
    out = fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, window=window, end=torch.as_tensor(end).cuda(), max_new=1, cap=3.0)
    b.check(out, window=window, end=end, cap=3.0, rows=rows)


@pytest.mark.parametrize("seqs", [[(5, 40), (0, 30), (0, 20), (0, 0), (0, 1)], [(0, 9), (33, 60)] + [(0, 5)] * 31, [(1, 40)] * 3])
def test_rows_that_no_bound_is_given_for(fq, seqs):
    """No more rows than sequences are taken for single tokens, whosever they are."""
    b = Batch(seqs, 8, 2, 16, 61)
    b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE))
    b.check(fq.fq_kv4_attention_chunk(*b.gpu(), SCALE, max_len=2000, window=11), window=11)


@pytest.mark.parametrize("seqs", [[(1, 50), (3, 40)], [(60, 90), (9, 33)]])
def test_pages_past_four_gigabytes(fq, seqs):
    """The same tokens in near pages and behind 4 GiB of cache: the same output."""
    b = Batch(seqs, 4, 2, 16, 67)
    q, qs, cache, table, starts, lens = b.gpu()
    pages = (1 << 32) // cache[0].numel() + cache.shape[0] + 3
    far = torch.empty((pages,) + tuple(cache.shape[1:]), dtype=torch.uint8, device="cuda")
    far[-cache.shape[0]:].copy_(cache)
    near = fq.fq_kv4_attention_chunk(q, qs, cache, table, starts, lens, SCALE)
    out = fq.fq_kv4_attention_chunk(q, qs, far, (table + (pages - cache.shape[0])).to(torch.int32), starts, lens, SCALE)
    assert torch.equal(out.view(torch.int16), near.view(torch.int16))


def test_two_calls_at_once(fq):
    """On two streams, each with scratch of its own: what each gives alone."""
    a, b = Batch([(1, 1500), (1, 900)], 8, 2, 32, 71), Batch([(80, 700)], 8, 2, 32, 73)
    args = [a.gpu(), b.gpu()]
    want = [fq.fq_kv4_attention_chunk(*x, SCALE) for x in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = [None, None]
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                for _ in range(4):
                    got[i] = fq.fq_kv4_attention_chunk(*args[i], SCALE)
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))
