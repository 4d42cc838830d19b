"""Norms, paged cache and attention on the GPU against the plain 64-bit forms of paged_util.py.

Tolerances are counted from the roundings of the definition before anything ran; codes and cached bytes are compared bit for bit."""
import numpy as np
import pytest

import paged_util as pu

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def fq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: torch.cuda.is_available() is False")
    from paper_2505_20839_amd import binding
    return binding


# ---- norms ----

def _norm_inputs(M, K, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, K), generator=g) * scale
    x[:, :: max(1, K // 7)] *= 20
    r = 16 * scale * torch.randn((M, K), generator=g)
    w = 1 + 0.1 * torch.randn(K, generator=g)
    return x.bfloat16(), r.bfloat16(), w.bfloat16()


def _check_norm(fq, x, r, w, eps, got, quant):
    """`got`: the call's outputs on the CPU.  FP32 sums of K squares in chains of at most 64 numbers and a tree: the mean is off by
    less than 2^-17, its root by half of that; y takes three more roundings."""
    h = x.double() if r is None else (x.float() + r.float()).bfloat16().double()
    if r is not None:
        assert torch.equal(got[-1].view(torch.int16), (x.float() + r.float()).bfloat16().view(torch.int16))
    y = h * w.double() / torch.sqrt(h.square().mean(-1, keepdim=True) + eps)
    rel = 2.0 ** -17
    if not quant:
        assert bool(((got[0].double() - y).abs() <= (2.0 ** -8 + rel) * y.abs() + 1e-38).all())
        return
    codes, s = got[0], got[1].double()
    amax = y.abs().amax(-1)
    want = torch.where(amax > 0, amax / 448, torch.ones_like(amax))
    assert bool(((s - want).abs() <= rel * want).all())
    val = torch.from_numpy(pu.E4M3[codes.numpy()])
    assert not bool(((codes & 0x7F) == 0x7F).any())
    q = y / want[:, None]
    # half an E4M3 step: 2^-4 relative, 2^-10 below the smallest normal number
    assert bool(((val - q).abs() <= torch.maximum(2.0 ** -4 * q.abs(), torch.tensor(2.0 ** -10, dtype=torch.float64)) + 2 * rel * q.abs()).all())


@pytest.mark.parametrize("K", [8, 64, 520, 1024, 2048, 2056, 4096, 4104, 5120, 8200, 11008, 16384, 16392, 32768, 33000, 65536, 65544, 70000])
@pytest.mark.parametrize("quant", [True, False])
def test_norm_sizes(fq, K, quant):
    for M, with_r in ((1, True), (5, False), (3, True)):
        x, r, w = _norm_inputs(M, K, K + M)
        r = r if with_r else None
        call = fq.fq_rmsnorm_quant if quant else fq.fq_rmsnorm
        got = call(x.cuda(), w.cuda(), 1e-5, residual=None if r is None else r.cuda())
        got = got if isinstance(got, tuple) else (got,)
        _check_norm(fq, x, r, w, 1e-5, [t.cpu() for t in got], quant)


@pytest.mark.parametrize("M, K", [(2, 4096), (64, 4096), (65, 128), (300, 4096), (700, 1024), (1600, 2048), (1537, 1920), (513, 11008), (70, 16384)])
def test_norm_many_rows_and_prepared_workspace(fq, M, K):
    """With the GEMM's workspace: the same codes and scales, and the workspace as the quantiser leaves it for them."""
    x, r, w = _norm_inputs(M, K, M + K)
    A, s, H = fq.fq_rmsnorm_quant(x.cuda(), w.cuda(), 1e-6, residual=r.cuda())
    _check_norm(fq, x, r, w, 1e-6, [A.cpu(), s.cpu(), H.cpu()], True)
    y = fq.fq_rmsnorm(x.cuda(), w.cuda(), 1e-6)
    _check_norm(fq, x, None, w, 1e-6, [y.cpu()], False)
    if K % 128 == 0:
        N = 256
        need = fq.fq_w4a8_gemm_workspace_bytes(M, N, K)
        ws = torch.full((max(need, 16),), 0xA5, dtype=torch.uint8, device="cuda")
        A2, s2, H2 = fq.fq_rmsnorm_quant(x.cuda(), w.cuda(), 1e-6, residual=r.cuda(), workspace=ws)
        assert torch.equal(A, A2) and torch.equal(s, s2) and torch.equal(H, H2)
        q = torch.randint(-8, 8, (N, K), dtype=torch.int8, device="cuda")
        gs = torch.full((N, K // 128), 0x20, dtype=torch.uint8, device="cuda")
        packed = fq.fq_pack_weights(q)
        one = fq.fq_w4a8_gemm(A, s, packed, gs, 1.0, N)
        two = fq.fq_w4a8_gemm(A2, s2, packed, gs, 1.0, N, workspace=ws, workspace_prepared=need > 0)
        assert torch.equal(one, two)


def test_norm_in_place_and_zero_rows(fq):
    x, r, w = _norm_inputs(6, 4096, 1)
    x[2] = 0
    r[2] = 0
    x[3] = -r[3]
    want = fq.fq_rmsnorm_quant(x.cuda(), w.cuda(), 1e-5, residual=r.cuda())
    res = r.cuda()
    got = fq.fq_rmsnorm_quant(x.cuda(), w.cuda(), 1e-5, residual=res, out=res)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert got[2].data_ptr() == res.data_ptr()
    assert float(got[1][2]) == 1.0 and not bool((got[0][2] & 0x7F).any())
    xs = x.cuda()
    got = fq.fq_rmsnorm(xs, w.cuda(), 1e-5, residual=r.cuda(), out=xs)
    assert torch.equal(got[1], want[2]) and got[1].data_ptr() == xs.data_ptr()
    assert not bool(got[0][2].float().any())
    long, rl, wl = _norm_inputs(2, 70000, 2)               # rows that are read twice
    res = rl.cuda()
    got = fq.fq_rmsnorm_quant(long.cuda(), wl.cuda(), 1e-5, residual=res, out=res)
    _check_norm(fq, long, rl, wl, 1e-5, [t.cpu() for t in got], True)


@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e-3, 1e15])
def test_norm_magnitudes(fq, scale):
    """Rows far from 1: eps decides, or does not, and the codes use their whole range."""
    x, _, w = _norm_inputs(3, 512, 9, scale)
    A, s = fq.fq_rmsnorm_quant(x.cuda(), w.cuda(), 1e-12)
    _check_norm(fq, x, None, w, 1e-12, [A.cpu(), s.cpu()], True)


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan"), 3e38])
def test_norm_rows_that_are_not_finite(fq, bad):
    for K in (1024, 70000):
        x, r, w = _norm_inputs(4, K, 3)
        x[1, 77] = bad
        A, s = fq.fq_rmsnorm_quant(x.cuda(), w.cuda(), 1e-5)
        assert torch.isnan(s[1]) and not bool(A[1].any())
        ok = [0, 2, 3]
        _check_norm(fq, x[ok], None, w, 1e-5, [A.cpu()[ok], s.cpu()[ok]], True)
        assert bool(torch.isnan(fq.fq_rmsnorm(x.cuda(), w.cuda(), 1e-5)[1]).all())
    w[5] = float("nan")
    A, s = fq.fq_rmsnorm_quant(r.cuda(), w.cuda(), 1e-5)
    assert bool(torch.isnan(s).all()) and not bool(A.any())


@pytest.mark.parametrize("K", [1024, 4096, 70000])
def test_norm_results_past_the_range(fq, K):
    """h w fits FP32 and y does not: a row with one number is brought to sqrt(K) times the weight."""
    x, w = torch.zeros((3, K)), torch.ones(K)
    x[:, 9], w[9] = 1.0, 1e38
    x[1, 9], x[1, 10], x[2, 9] = 0.0, 1.0, 0.0
    x, w = x.bfloat16(), w.bfloat16()
    A, s = fq.fq_rmsnorm_quant(x.cuda(), w.cuda(), 1e-5)
    assert torch.isnan(s[0]) and not bool(A[0].any())
    _check_norm(fq, x[1:], None, w, 1e-5, [A.cpu()[1:], s.cpu()[1:]], True)
    y = fq.fq_rmsnorm(x.cuda(), w.cuda(), 1e-5).cpu()
    assert float(y[0, 9]) == float("inf") and int((y[0] != 0).sum()) == 1


def test_norm_refusals(fq):
    x = torch.zeros((4, 512), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(512, dtype=torch.bfloat16, device="cuda")
    for call in (fq.fq_rmsnorm, fq.fq_rmsnorm_quant):
        with pytest.raises(TypeError):
            call(x.float(), w, 1e-5)
        with pytest.raises(TypeError):
            call(x, w.float(), 1e-5)
        with pytest.raises(ValueError):
            call(x[:, ::2], w[::2].contiguous(), 1e-5)
        for a, k in (((x, w[:256].contiguous(), 1e-5), {}), ((x, w, 0.0), {}), ((x, w, 1e-5), dict(residual=x[:2])), ((x, w, 1e-5), dict(out=x)),
                     ((x[:, :12].contiguous(), w[:12].contiguous(), 1e-5), {})):
            with pytest.raises(fq.FireqError):
                call(*a, **k)
    assert [tuple(t.shape) for t in fq.fq_rmsnorm_quant(x[:0], w, 1e-5)] == [(0, 512), (0,)]


# ---- append and read ----

def _rotation(n):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(64) / 64)
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


@pytest.mark.parametrize("T, Hq, Hkv, page, interleaved, ld", [
    (1, 1, 1, 16, False, 0), (1, 8, 2, 32, True, 0), (7, 4, 4, 48, False, 64), (37, 6, 2, 16, True, 8), (70, 5, 1, 64, False, 0), (65, 16, 1, 128, True, 128)])
def test_append_and_read(fq, T, Hq, Hkv, page, interleaved, ld):
    rng = np.random.default_rng(T * 100 + page)
    width = (Hq + 2 * Hkv) * 128
    pages = T // page + 3
    x = rng.standard_normal((T, width)) * np.exp(rng.standard_normal((T, 1)))
    x[:, ::97] *= 20
    full = torch.zeros((T, width + ld)).bfloat16()
    full[:, :width] = torch.from_numpy(x).bfloat16()
    full[0, :128] = 0                                     # a query of zeros
    full[T - 1, Hq * 128:(Hq + 1) * 128] = 0              # a key of zeros
    if T > 4:
        full[3, -ld - 128 if ld else -128:width] = full[3, -ld - 128 if ld else -128:width] * 2.0 ** -13   # sigma below E4M3's range
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    if T > 2:
        slots[1] = -1
        slots[T // 2:] = np.arange(T - T // 2) + page + 3  # a run that begins and ends inside a tile
    slots = np.array([s if i >= T // 2 or T <= 2 else (s if s not in range(page + 3, page + 3 + T) else -5) for i, s in enumerate(slots)])
    pos = rng.integers(0, 500, T).astype(np.int32)
    rot = _rotation(500)
    ref = pu.Cache(pages, Hkv, page, rng)
    cache = torch.from_numpy(ref.b.copy()).cuda()
    dev = full.cuda()[:, :width]
    Q, qs = fq.fq_kv4_append(dev, torch.from_numpy(rot).cuda(), torch.from_numpy(pos).cuda(), torch.from_numpy(slots).cuda(), cache, interleaved=interleaved)
    xf = full[:, :width].float().numpy().reshape(T, Hq + 2 * Hkv, 128)
    for i in range(T):
        for h in range(Hq):
            r = pu.rotate(xf[i, h], rot[pos[i]], interleaved)
            top = np.abs(r).max()
            s = np.float32(top) / np.float32(448) if top > 0 else np.float32(1)
            assert np.float32(qs[i, h].item()) == s
            assert np.array_equal(pu.E4M3[Q[i, h].cpu().numpy()], pu.E4M3[pu.to_e4m3(r / s)])
        if slots[i] >= 0:
            for h in range(Hkv):
                ref.put(int(slots[i]), h, False, *pu.int4(pu.rotate(xf[i, Hq + h], rot[pos[i]], interleaved)))
                ref.put(int(slots[i]), h, True, *pu.int4(xf[i, Hq + Hkv + h]))
    assert np.array_equal(cache.cpu().numpy(), ref.b)     # what was not appended is as it was
    K, V = fq.fq_kv4_read(cache, torch.from_numpy(slots).cuda())
    for i in range(T):
        for h in range(Hkv):
            if slots[i] < 0:
                assert not bool(K[i, h].float().any()) and not bool(V[i, h].float().any())
                continue
            for got, value in ((K, False), (V, True)):
                c, sc = ref.get(int(slots[i]), h, value)
                assert np.array_equal(got[i, h].double().cpu().numpy(), c * pu.E4M3[sc])


def test_append_what_cannot_be_done_shows(fq):
    Hq, Hkv, page, T = 4, 2, 16, 6
    x = torch.randn((T, (Hq + 2 * Hkv) * 128)).bfloat16()
    x[0, 5] = float("nan")                                # one query head
    x[1, Hq * 128 + 3] = float("inf")                     # one key head
    x[2, (Hq + Hkv) * 128 + 1] = float("nan")             # one value head
    pos = torch.tensor([0, 1, 2, 99, -1, 5], dtype=torch.int32)
    slots = torch.tensor([0, 1, 2, 3, 4, 48], dtype=torch.int64)
    cache = fq.fq_kv4_cache(3, Hkv, page)
    rot = torch.from_numpy(_rotation(50)).cuda()
    Q, qs = fq.fq_kv4_append(x.cuda(), rot, pos.cuda(), slots.cuda(), cache)
    nan = torch.isnan(qs).cpu()
    want = torch.zeros((T, Hq), dtype=torch.bool)
    want[0, 0] = True
    want[3:] = True                                       # positions outside the table, a slot behind the end
    assert torch.equal(nan, want) and not bool(Q[nan.cuda()].any())
    assert not bool(cache[1:].any())
    K, V = fq.fq_kv4_read(cache, slots.cuda())
    kn, vn = torch.isnan(K.float()).any(-1).cpu(), torch.isnan(V.float()).any(-1).cpu()
    both = torch.tensor([[False, False]] * 3 + [[True, True]] * 3)
    k, v = both.clone(), both.clone()
    k[1, 0] = True
    v[2, 0] = True
    assert torch.equal(kn, k) and torch.equal(vn, v)


def test_append_and_read_refusals(fq):
    cache = fq.fq_kv4_cache(2, 2, 16)
    x = torch.zeros((3, 8 * 128), dtype=torch.bfloat16, device="cuda")
    rot = torch.zeros((4, 64, 2), device="cuda")
    pos, slots = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    good = dict(QKV=x, cos_sin=rot, positions=pos, slots=slots, cache=cache)
    for change, e in ((dict(QKV=x.float()), TypeError), (dict(positions=slots), TypeError), (dict(slots=pos), TypeError), (dict(cos_sin=rot.double()), TypeError),
                      (dict(cache=cache.cpu()), TypeError), (dict(cache=cache.float()), TypeError), (dict(QKV=x.t()), ValueError),
                      (dict(cache=torch.zeros((2, 2, 2080, 2), dtype=torch.uint8, device="cuda").transpose(2, 3)), ValueError),
                      (dict(QKV=x[:, :1000]), fq.FireqError), (dict(QKV=x[:, :512]), fq.FireqError), (dict(QKV=x[:, : 5 * 128]), fq.FireqError),
                      (dict(cos_sin=rot[:, :32].contiguous()), fq.FireqError),
                      (dict(positions=pos[:2]), fq.FireqError), (dict(slots=slots[:2]), fq.FireqError), (dict(cache=cache[..., :2064]), fq.FireqError),
                      (dict(QKV=torch.zeros((3, 1030), dtype=torch.bfloat16, device="cuda")[:, :1024]), fq.FireqError)):
        with pytest.raises(e):
            fq.fq_kv4_append(**dict(good, **change))
    assert [tuple(t.shape) for t in fq.fq_kv4_append(x[:0], rot, pos[:0], slots[:0], cache)] == [(0, 4, 128), (0, 4)]
    assert tuple(fq.fq_kv4_read(cache, slots[:0])[0].shape) == (0, 2, 128)
    with pytest.raises(TypeError):
        fq.fq_kv4_read(cache, pos)
    K, V = fq.fq_kv4_read(cache, torch.tensor([32, -1], device="cuda"))    # behind the end; padding
    assert bool(torch.isnan(K[0]).all()) and bool(torch.isnan(V[0]).all()) and not bool(K[1].any())


# ---- attention ----

def _filled(rng, lens, Hkv, page, extra=2, prefix=0):
    """A cache with every sequence's tokens in pages of its own, its table (int32, with pages that do not exist behind a
    sequence's end), the prefix's pages and the free ones."""
    need = [-(-n // page) for n in lens]
    shared = -(-prefix // page)
    pages = sum(need) + shared + extra
    ref = pu.Cache(pages, Hkv, page, rng)
    order = list(rng.permutation(pages))
    table = np.full((len(lens), max(need + [0]) + 2), 1 << 30, np.int32)
    table[:, 1::2] = -7
    for b, n in enumerate(need):
        for i in range(n):
            table[b, i] = order.pop()
    pre = np.array([order.pop() for _ in range(shared)], np.int32)

    def fill(pages_of, n):
        for t in range(n):
            slot = int(pages_of[t // page]) * page + t % page
            for h in range(Hkv):
                for value in (False, True):
                    ref.put(slot, h, value, rng.integers(-8, 8, 128), int(pu.to_e4m3(np.float32(rng.uniform(0.05, 1.0) * (-1 if rng.random() < 0.1 else 1)))))

    for b, n in enumerate(lens):
        fill(table[b], n)
    fill(pre, prefix)
    return ref, table, pre


def _queries(rng, B, Hq, spread):
    x = rng.standard_normal((B, Hq, 128)) * spread
    s = (np.abs(x).max(-1) / 448).astype(np.float32)
    return pu.to_e4m3((x / s[..., None]).astype(np.float32)), s


def _check_attention(ref, table, lens, q, qs, Hkv, got, scale, pre=(), prefix=0, skip=(), only=None):
    B, Hq = q.shape[:2]
    page, G = ref.page, Hq // Hkv
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all() or skip
    for b in range(B) if only is None else only:
        if b in skip:
            assert np.isnan(got[b]).all(), b
            continue
        for h in range(Hkv):
            slots = [int(pre[t // page]) * page + t % page for t in range(prefix)] + [int(table[b, t // page]) * page + t % page for t in range(max(0, lens[b]))]
            kv = list(ref.tokens(slots, h))
            for r in range(h * G, (h + 1) * G):
                o, tol = pu.attention(q[b, r], qs[b, r], *kv, scale)
                assert (np.abs(got[b, r] - o) <= tol).all(), (b, r, float((np.abs(got[b, r] - o) / np.maximum(tol, 1e-30)).max()))


@pytest.mark.parametrize("Hq, Hkv, page, lens, spread", [
    (1, 1, 16, [1], 1), (4, 1, 16, [0], 1), (2, 2, 32, [0, 1, 2, 15, 16, 17, 31, 32, 33], 1), (8, 2, 16, [63, 64, 65, 0, 127], 3),
    (3, 1, 48, [47, 48, 49, 250], 1), (16, 1, 16, [300], 2), (17, 1, 64, [129, 5], 1), (40, 1, 128, [200], 1), (5, 5, 16, [1100], 4),
    (8, 1, 16, [2600, 3], 1), (4, 2, 128, [640], 30), (2, 1, 16, [700, 0, 1], 0.01)])
def test_attention_against_64_bits(fq, Hq, Hkv, page, lens, spread):
    rng = np.random.default_rng(sum(lens) + Hq)
    ref, table, _ = _filled(rng, lens, Hkv, page)
    q, qs = _queries(rng, len(lens), Hq, spread)
    lens_t = torch.tensor(lens, dtype=torch.int32).cuda()
    args = (torch.from_numpy(q).cuda(), torch.from_numpy(qs).cuda(), torch.from_numpy(ref.b).cuda(), torch.from_numpy(table).cuda(), lens_t, 0.1)
    for most in (None, max(lens), max(lens) + 40):        # (an upper bound decides how the work is split)
        got = fq.fq_kv4_attention(*args, max_len=most)
        _check_attention(ref, table, lens, q, qs, Hkv, got, 0.1)
        again = fq.fq_kv4_attention(*args, max_len=most)
        assert torch.equal(got.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("B, Hq, Hkv, page, prefix, longest", [
    (1, 1, 1, 16, 1, 0), (2, 4, 2, 16, 16, 20), (3, 8, 1, 32, 100, 5), (5, 3, 3, 48, 333, 70), (17, 8, 2, 16, 260, 40), (33, 16, 1, 64, 130, 3), (9, 20, 1, 128, 700, 30)])
def test_attention_behind_a_prefix(fq, B, Hq, Hkv, page, prefix, longest):
    rng = np.random.default_rng(B * prefix)
    lens = [int(n) for n in rng.integers(0, longest + 1, B)]
    lens[0] = 0
    ref, table, pre = _filled(rng, lens, Hkv, page, prefix=prefix)
    q, qs = _queries(rng, B, Hq, 1.5)
    args = (torch.from_numpy(q).cuda(), torch.from_numpy(qs).cuda(), torch.from_numpy(ref.b).cuda())
    own = (torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), 0.1)
    shared = torch.from_numpy(pre).cuda()
    for most in (None, longest):
        got = fq.fq_kv4_attention_prefix(*args, shared, prefix, *own, max_len=most)
        _check_attention(ref, table, lens, q, qs, Hkv, got, 0.1, pre, prefix)
    # no prefix: the plain call
    none = fq.fq_kv4_attention_prefix(*args, shared, 0, *own)
    assert torch.equal(none.view(torch.int16), fq.fq_kv4_attention(*args, *own).view(torch.int16))


def test_attention_with_a_bound_far_above_the_lengths(fq):
    """Parts are long then (a grid has 65535 of them at most): whole steps, nothing counted twice at their ends."""
    rng = np.random.default_rng(5)
    lens = [2500] + [0] * 258 + [17]
    ref, table, _ = _filled(rng, lens, 1, 32)
    q, qs = _queries(rng, len(lens), 1, 0.1)
    got = fq.fq_kv4_attention(torch.from_numpy(q).cuda(), torch.from_numpy(qs).cuda(), torch.from_numpy(ref.b).cuda(), torch.from_numpy(table).cuda(),
                              torch.tensor(lens, dtype=torch.int32).cuda(), 0.1, max_len=131072016)
    _check_attention(ref, table, lens, q, qs, 1, got, 0.1)


def test_attention_what_cannot_be_done_shows(fq):
    rng = np.random.default_rng(4)
    lens = [40, 40, 40, 70, 20, -3]
    ref, table, pre = _filled(rng, [max(n, 0) for n in lens], 2, 16, prefix=30)
    q, qs = _queries(rng, len(lens), 4, 1)
    qs[2, 1] = float("nan")
    bad = table.copy()
    bad[0, 1] = ref.b.shape[0]                            # pages outside the cache, within the length
    bad[4, 0] = -1
    Q, S, C = (torch.from_numpy(a).cuda() for a in (q, qs, ref.b))
    L = torch.tensor(lens, dtype=torch.int32).cuda()
    got = fq.fq_kv4_attention(Q, S, C, torch.from_numpy(bad).cuda(), L, 0.1, max_len=64)
    nan = torch.isnan(got.float()).all(-1).cpu()
    want = torch.zeros((6, 4), dtype=torch.bool)
    want[[0, 3, 4]] = True                                # 3: longer than max_len
    want[2, 1] = True
    assert torch.equal(nan, want) and not bool(got[5].float().any())
    ok = np.array([1])
    _check_attention(ref, bad[ok], [40], q[ok], qs[ok], 2, got[1:2], 0.1)
    # longer than the table
    got = fq.fq_kv4_attention(Q, S, C, torch.from_numpy(table[:, :3].copy()).cuda(), L, 0.1)
    nan = torch.isnan(got.float()).all(-1).cpu()
    assert bool(nan[3].all()) and not bool(nan[[0, 1, 4, 5]].any())
    # no room at all, and a prefix page that does not exist: for everybody
    got = fq.fq_kv4_attention(Q, S, C, torch.zeros((6, 0), dtype=torch.int32, device="cuda"), L, 0.1)
    assert bool(torch.isnan(got[:5].float()).all()) and not bool(got[5].float().any())
    pre[1] = -1
    got = fq.fq_kv4_attention_prefix(Q, S, C, torch.from_numpy(pre).cuda(), 30, torch.from_numpy(table).cuda(), L, 0.1)
    assert bool(torch.isnan(got.float()).all())


def test_attention_nan_scales_of_a_token(fq):
    """A cached key or value that is marked broken breaks its own sequence and head only."""
    rng = np.random.default_rng(5)
    lens = [50, 50, 50]
    ref, table, _ = _filled(rng, lens, 2, 16)
    ref.flat(table[0, 1], 0)[pu.scale_place(3, False)] = 0x7F
    ref.flat(table[1, 2], 1)[pu.scale_place(7, True)] = 0x7F
    q, qs = _queries(rng, 3, 4, 1)
    got = fq.fq_kv4_attention(torch.from_numpy(q).cuda(), torch.from_numpy(qs).cuda(), torch.from_numpy(ref.b).cuda(), torch.from_numpy(table).cuda(),
                              torch.tensor(lens, dtype=torch.int32).cuda(), 0.1)
    nan = torch.isnan(got.float()).any(-1).cpu()
    want = torch.zeros((3, 4), dtype=torch.bool)
    want[0, :2] = True
    want[1, 2:] = True
    assert torch.equal(nan, want)


def test_attention_of_a_layers_slice_and_far_pages(fq):
    """One layer's part of a larger pool (strided pages and heads), at byte offsets past 32 bits."""
    rng = np.random.default_rng(6)
    lens, page, Hkv = [90, 33], 32, 2
    ref, table, _ = _filled(rng, lens, Hkv, page)
    q, qs = _queries(rng, 2, 4, 1)
    n = ref.b.shape[0]
    layers, far = 3, (5 << 30) // (3 * Hkv * 2 * 2080)
    pool = torch.empty((far + n, layers, Hkv, page // 16, 2080), dtype=torch.uint8, device="cuda")
    cache = pool[:, 1]
    cache[far:] = torch.from_numpy(ref.b).cuda()
    used = table.copy()
    used[(table >= 0) & (table < n)] += far
    args = (torch.from_numpy(q).cuda(), torch.from_numpy(qs).cuda())
    L = torch.tensor(lens, dtype=torch.int32).cuda()
    got = fq.fq_kv4_attention(*args, cache, torch.from_numpy(used).cuda(), L, 0.1)
    _check_attention(ref, table, lens, q, qs, Hkv, got, 0.1)
    by_head = torch.empty((Hkv, n, page // 16, 2080), dtype=torch.uint8, device="cuda").transpose(0, 1)   # heads outside
    by_head.copy_(torch.from_numpy(ref.b))
    got2 = fq.fq_kv4_attention(*args, by_head, torch.from_numpy(table).cuda(), L, 0.1)
    assert torch.equal(got.view(torch.int16), got2.view(torch.int16))
    # append and read there too
    x = torch.randn((5, 8 * 128)).bfloat16().cuda()
    rot = torch.from_numpy(_rotation(9)).cuda()
    pos = torch.arange(5, dtype=torch.int32).cuda()
    at = torch.arange(5).cuda() + 70
    small = fq.fq_kv4_cache(n, Hkv, page)
    Q1, s1 = fq.fq_kv4_append(x, rot, pos, at, small)
    Q2, s2 = fq.fq_kv4_append(x, rot, pos, at + far * page, cache)
    assert torch.equal(Q1, Q2) and torch.equal(s1, s2)
    for a, b in zip(fq.fq_kv4_read(small, at), fq.fq_kv4_read(cache, at + far * page)):
        assert torch.equal(a, b)


def test_attention_refusals(fq):
    cache = fq.fq_kv4_cache(4, 2, 16)
    Q = torch.zeros((3, 4, 128), dtype=torch.uint8, device="cuda")
    qs = torch.ones((3, 4), device="cuda")
    table, lens = torch.zeros((3, 2), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    good = dict(Q=Q, q_scale=qs, cache=cache, block_table=table, seq_lens=lens, out_scale=0.1)
    for change, e in ((dict(Q=Q.float()), TypeError), (dict(q_scale=qs.half()), TypeError), (dict(block_table=table.long()), TypeError),
                      (dict(seq_lens=lens.long()), TypeError), (dict(cache=cache.cpu()), TypeError), (dict(block_table=table.t()), ValueError),
                      (dict(Q=Q[:, :3].contiguous()), fq.FireqError), (dict(q_scale=qs[:2]), fq.FireqError), (dict(seq_lens=lens[:2]), fq.FireqError),
                      (dict(block_table=table[:2]), fq.FireqError), (dict(out_scale=0.0), fq.FireqError), (dict(max_len=-1), fq.FireqError),
                      (dict(out=torch.empty((3, 4, 64), dtype=torch.bfloat16, device="cuda")), fq.FireqError),
                      (dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"), max_len=10 ** 6,
                            block_table=torch.zeros((3, 60000), dtype=torch.int32, device="cuda")), fq.FireqError)):
        with pytest.raises(e):
            fq.fq_kv4_attention(**dict(good, **change))
    shared = torch.zeros(2, dtype=torch.int32, device="cuda")
    for change, e in ((dict(prefix_len=33), fq.FireqError), (dict(prefix_len=-1), fq.FireqError), (dict(prefix_pages=shared.long()), TypeError)):
        with pytest.raises(e):
            fq.fq_kv4_attention_prefix(**dict(dict(good, prefix_pages=shared, prefix_len=5), **change))
    empty = fq.fq_kv4_attention(Q[:0], qs[:0], cache, table[:0], lens[:0], 0.1)
    assert tuple(empty.shape) == (0, 4, 128)
    flat = torch.empty((3, 512), dtype=torch.bfloat16, device="cuda")
    assert fq.fq_kv4_attention(**good, out=flat).data_ptr() == flat.data_ptr() and not bool(flat.any())


@pytest.mark.parametrize("more", [1 << 32, (1 << 32) + 5, (1 << 33) + (1 << 20), (1 << 30) + 1])
def test_attention_refuses_bounds_past_its_integers(fq, more):
    """Not taken for their low 32 bits."""
    cache = fq.fq_kv4_cache(2, 1, 16)
    Q, qs = torch.zeros((1, 1, 128), dtype=torch.uint8, device="cuda"), torch.ones((1, 1), device="cuda")
    table, lens = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(fq.FireqError):
        fq.fq_kv4_attention(Q, qs, cache, table, lens, 0.1, max_len=more)
    with pytest.raises(fq.FireqError):
        fq.fq_kv4_attention_prefix(Q, qs, cache, table[0], 3, table, lens, 0.1, max_len=more)
    with pytest.raises(fq.FireqError):
        fq.fq_kv4_attention_prefix(Q, qs, cache, table[0], more, table, lens, 0.1)


def test_workspaces_that_are_refused(fq):
    """Host memory, and a view whose numbers do not lie together."""
    x, w = torch.zeros((128, 512), dtype=torch.bfloat16, device="cuda"), torch.ones(512, dtype=torch.bfloat16, device="cuda")
    cache = fq.fq_kv4_cache(2, 1, 16)
    Q, qs = torch.zeros((1, 1, 128), dtype=torch.uint8, device="cuda"), torch.ones((1, 1), device="cuda")
    table, lens = torch.zeros((1, 2000), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    n = max(fq.fq_w4a8_gemm_workspace_bytes(128, 256, 512), fq.fq_kv4_attention_workspace_bytes(1, 1, 1, 32000, 20))
    for ws, e in ((torch.empty(n, dtype=torch.uint8), TypeError), (n, TypeError), (torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2], ValueError)):
        for call in (lambda: fq.fq_rmsnorm_quant(x, w, 1e-5, workspace=ws), lambda: fq.fq_kv4_attention(Q, qs, cache, table, lens, 0.1, workspace=ws),
                     lambda: fq.fq_kv4_attention_prefix(Q, qs, cache, table[0], 20, table, lens, 0.1, workspace=ws)):
            with pytest.raises(e, match="workspace"):
                call()


def test_a_decode_step_in_a_graph_and_on_another_stream(fq):
    """Norm, append and attention captured once, replayed on new inputs with eager work in between, and on a side stream."""
    torch.manual_seed(0)
    B, Hq, Hkv, page, width = 5, 8, 2, 16, 40
    cache = fq.fq_kv4_cache(B * width, Hkv, page)
    table = torch.randperm(B * width, device="cuda").to(torch.int32).reshape(B, width).contiguous()
    rot = torch.from_numpy(_rotation(700)).cuda()
    w = torch.ones(1024, dtype=torch.bfloat16, device="cuda")
    x = torch.randn((B, 1024), device="cuda").bfloat16()
    res = torch.randn((B, 1024), device="cuda").bfloat16()
    lens = torch.tensor([1, 20, 300, 555, 47], dtype=torch.int32, device="cuda")
    hist = torch.randn((600, 12 * 128), device="cuda").bfloat16()
    for b in range(B):
        t = torch.arange(600, device="cuda")
        fq.fq_kv4_append(hist, rot, t.to(torch.int32), table[b].long()[t // page] * page + t % page, cache)

    def step(qkv):
        A, s, H = fq.fq_rmsnorm_quant(x, w, 1e-5, residual=res)
        at = (lens - 1).long()
        slots = table.long().gather(1, (at // page)[:, None])[:, 0] * page + at % page
        Q, qs = fq.fq_kv4_append(qkv, rot, lens - 1, slots, cache)
        return A, s, H, Q, qs, fq.fq_kv4_attention(Q, qs, cache, table, lens, 0.0884, max_len=width * page)

    qkv = torch.randn((B, 12 * 128), device="cuda").bfloat16()
    step(qkv)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(qkv)
    side = torch.cuda.Stream()
    for i in range(4):
        qkv.copy_(torch.randn((B, 12 * 128), device="cuda"))
        x.copy_(torch.randn((B, 1024), device="cuda"))
        lens.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step(qkv)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = step(qkv)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for a, b, c in zip(got, want, other):
            assert torch.equal(a, b) and torch.equal(a, c)


def test_native_and_python_forms_agree(fq):
    """Every call through the native marshalling and through its Python form: the same outputs, the same refusals."""
    from test_gpu_marshal import _same
    x = torch.randn((5, 1024), device="cuda").bfloat16()
    r, w = torch.randn_like(x), torch.ones(1024, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    for name in ("fq_rmsnorm", "fq_rmsnorm_quant"):
        for kw in ({}, {"residual": r}, {"residual": r, "out": torch.empty_like(x)}):
            _same(fq, name, lambda: ((x, w, 1e-5), dict(kw)), native=True)
        for bad, exc in (((x.float(), w, 1e-5), TypeError), ((x, w[:-8], 1e-5), fq.FireqError), ((x, w, 0.0), fq.FireqError), ((x[:, ::2], w[::2].contiguous(), 1e-5), ValueError)):
            _same(fq, name, lambda: (bad, {}), exc)
        _same(fq, name, lambda: ((x, w, 1e-5), {"out": x}), fq.FireqError)
        _same(fq, name, lambda: ((x, w, 1e-5), {"residual": r[:4]}), fq.FireqError)
        _same(fq, name, lambda: ((x[:0], w, 1e-5), {}), native=False)
    _same(fq, "fq_rmsnorm_quant", lambda: ((x, w, 1e-5), {"workspace": ws}), native=True)
    Hq, Hkv, page = 4, 2, 32
    qkv = torch.randn((6, 8 * 128), device="cuda").bfloat16()
    rot = torch.from_numpy(_rotation(20)).cuda()
    pos, slots = torch.arange(6, dtype=torch.int32, device="cuda"), torch.arange(6, device="cuda") + 20
    cache = fq.fq_kv4_cache(3, Hkv, page)
    ok = (qkv, rot, pos, slots, cache)
    _same(fq, "fq_kv4_append", lambda: (ok, {}), native=True)
    _same(fq, "fq_kv4_append", lambda: (ok, {"interleaved": True}), native=True)
    _same(fq, "fq_kv4_append", lambda: ((qkv[:, :1024], rot, pos, slots, cache), {}), native=True)
    for bad, exc in (((qkv.float(),) + ok[1:], TypeError), ((qkv, rot, pos[:5], slots, cache), fq.FireqError), ((qkv, rot, pos, slots, cache[:, :, :, :2064]), fq.FireqError),
                     ((qkv[:, : 4 * 128], rot, pos, slots, cache), fq.FireqError)):
        _same(fq, "fq_kv4_append", lambda: (bad, {}), exc)
    _same(fq, "fq_kv4_read", lambda: ((cache, slots), {}), native=True)
    _same(fq, "fq_kv4_read", lambda: ((cache, pos), {}), TypeError)
    Q, qs = fq.fq_kv4_append(*ok)
    table = torch.arange(6, dtype=torch.int32, device="cuda").reshape(6, 1) % 3
    lens = torch.tensor([26, 0, 21, 26, 1, 22], dtype=torch.int32, device="cuda")
    slots2 = torch.arange(96, device="cuda")
    fq.fq_kv4_append(torch.randn((96, 8 * 128), device="cuda").bfloat16(), rot, (slots2 % 20).to(torch.int32), slots2, cache)
    args = (Q, qs, cache, table, lens, 0.1)
    need = fq.fq_kv4_attention_workspace_bytes(6, Hq, Hkv, 32)
    for kw in ({}, {"max_len": 30}, {"out": torch.empty((6, Hq * 128), dtype=torch.bfloat16, device="cuda")}, {"workspace": torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")}):
        _same(fq, "fq_kv4_attention", lambda: (args, dict(kw)), native=True)
    shared = torch.tensor([2, 1], dtype=torch.int32, device="cuda")
    _same(fq, "fq_kv4_attention_prefix", lambda: ((Q, qs, cache, shared, 50, table, lens, 0.1), {}), native=True)
    for bad, exc in (((Q, qs, cache, shared, 65, table, lens, 0.1), fq.FireqError), ((Q, qs, cache, shared, 50, table, lens, -0.1), fq.FireqError),
                     ((Q, qs, cache, shared.long(), 50, table, lens, 0.1), TypeError)):
        _same(fq, "fq_kv4_attention_prefix", lambda: (bad, {}), exc)
    for bad, exc in (((Q[:, :3].contiguous(), qs, cache, table, lens, 0.1), fq.FireqError), ((Q, qs, cache, table.long(), lens, 0.1), TypeError), ((Q, qs, cache, table, lens, 0.0), fq.FireqError)):
        _same(fq, "fq_kv4_attention", lambda: (bad, {}), exc)
    _same(fq, "fq_kv4_attention", lambda: (args, {"max_len": -1}), fq.FireqError)


def test_attention_negative_and_zero_query_scales(fq):
    """A query's scale of 0 weighs all tokens alike; a negative one turns its scores round."""
    rng = np.random.default_rng(8)
    lens = [77, 300]
    ref, table, _ = _filled(rng, lens, 1, 16)
    q, qs = _queries(rng, 2, 4, 2)
    qs[0, 1] = 0.0
    qs[1, 2] *= -1
    got = fq.fq_kv4_attention(torch.from_numpy(q).cuda(), torch.from_numpy(qs).cuda(), torch.from_numpy(ref.b).cuda(), torch.from_numpy(table).cuda(),
                              torch.tensor(lens, dtype=torch.int32).cuda(), 0.1)
    flipped, fs = q.copy(), np.abs(qs)
    flipped[1, 2] ^= 0x80
    _check_attention(ref, table, lens, flipped, fs, 1, got, 0.1)


@pytest.mark.parametrize("B, Hq, Hkv, page, prefix, longest", [
    (40, 4, 1, 16, 3000, 4), (130, 1, 1, 48, 1203, 1), (32, 8, 2, 128, 2047, 20), (65, 2, 1, 16, 17, 2), (100, 16, 8, 16, 130, 1),
    (200, 2, 1, 16, 3201, 3), (130, 12, 4, 48, 1303, 20), (20, 40, 8, 128, 4000, 9), (1000, 1, 1, 16, 700, 1), (300, 20, 1, 32, 999, 2)])
def test_attention_of_many_rows_behind_a_prefix(fq, B, Hq, Hkv, page, prefix, longest):
    """The prefix apart for each sequence (the first five) and together for groups of rows: last groups of few rows, chunks and waves without
    tokens, tiles that the prefix ends in.  A sample of the sequences is checked."""
    rng = np.random.default_rng(B + prefix)
    lens = [int(n) for n in rng.integers(0, longest + 1, B)]
    ref, table, pre = _filled(rng, lens, Hkv, page, prefix=prefix)
    q, qs = _queries(rng, B, Hq, 1.5)
    got = fq.fq_kv4_attention_prefix(torch.from_numpy(q).cuda(), torch.from_numpy(qs).cuda(), torch.from_numpy(ref.b).cuda(), torch.from_numpy(pre).cuda(), prefix,
                                     torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), 0.1, max_len=longest)
    _check_attention(ref, table, lens, q, qs, Hkv, got, 0.1, pre, prefix, only=sorted({0, B - 1} | set(rng.integers(0, B, 12).tolist())))


@pytest.mark.parametrize("B", [3, 30, 900])
def test_a_bad_prefix_page_is_everybodys(fq, B):
    rng = np.random.default_rng(B)
    ref, table, pre = _filled(rng, [5] * B, 1, 16, prefix=700)
    q, qs = _queries(rng, B, 4, 1)
    pre[17] = ref.b.shape[0] + 5
    got = fq.fq_kv4_attention_prefix(torch.from_numpy(q).cuda(), torch.from_numpy(qs).cuda(), torch.from_numpy(ref.b).cuda(), torch.from_numpy(pre).cuda(), 700,
                                     torch.from_numpy(table).cuda(), torch.full((B,), 5, dtype=torch.int32, device="cuda"), 0.1)
    assert bool(torch.isnan(got.float()).all())


def test_the_decoding_example(fq):
    """The blocks of examples/paged_decode.py: a prompt and tokens behind it, with the prefix shared and with a copy of it in every sequence's
    own pages; the same prompt decoded token by token; and the command itself, eager and from a graph."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")
    spec = importlib.util.spec_from_file_location("paged_decode", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    T, B, page = 70, 3, 16
    g = torch.Generator(device="cuda").manual_seed(3)
    prompt = torch.randn((T, 512), generator=g, device="cuda").bfloat16()
    tokens = torch.randn((4, B, 512), generator=g, device="cuda").bfloat16()

    def decoder():
        return ex.Decoder(blocks=2, hidden=512, ffn=768, Hq=4, Hkv=2, page=page, pages=64, positions=256)

    def pages(lo, n):
        return torch.arange(lo, lo + n, dtype=torch.int32, device="cuda")

    one, two = decoder(), decoder()
    one.prefill(prompt, pages(0, 5))
    table = torch.stack([pages(10 * (b + 1), 2) for b in range(B)])
    long = torch.stack([pages(10 * (b + 1), 6) for b in range(B)])
    for b in range(B):
        two.prefill(prompt, long[b])
    for i in range(4):
        shared = one.step(tokens[i], table, torch.full((B,), i + 1, dtype=torch.int32, device="cuda"), pages(0, 5), T, max_len=8)
        apart = two.step(tokens[i], long, torch.full((B,), T + i + 1, dtype=torch.int32, device="cuda"), None, 0, max_len=96)
        # both caches hold the same numbers; the sums are split otherwise, and a bf16 step in the first block can move codes behind it
        rel = (shared.float() - apart.float()).norm() / apart.float().norm()
        assert bool(torch.isfinite(shared.float()).all()) and float(rel) < 0.1, float(rel)
    three = decoder()
    last = None
    for t in range(T):
        last = three.step(prompt[t:t + 1], pages(0, 5)[None].contiguous(), torch.full((1,), t + 1, dtype=torch.int32, device="cuda"), None, 0, max_len=T)
    whole = decoder().prefill(prompt, pages(0, 5))[-1:]
    rel = (last.float() - whole.float()).norm() / whole.float().norm()
    assert float(rel) < 0.1, float(rel)
    a = ex.main(["--batch", "3", "--prefix", "100", "--steps", "5", "--blocks", "1"])
    b = ex.main(["--batch", "3", "--prefix", "100", "--steps", "5", "--blocks", "1", "--no-graph"])
    assert a.shape == b.shape and bool(torch.isfinite(a.float()).all())


@pytest.mark.parametrize("T, Hq, Hkv, page", [(300, 2, 1, 16), (129, 5, 1, 48), (3, 64, 16, 16), (2, 130, 2, 32)])
def test_append_of_many_rows_and_many_heads(fq, T, Hq, Hkv, page):
    """Rows that change places between the XCDs, and rows whose heads take more than one workgroup."""
    test_append_and_read(fq, T, Hq, Hkv, page, False, 0)


def test_read_of_many_tokens(fq):
    rng = np.random.default_rng(12)
    ref = pu.Cache(70, 2, 32, rng, stale_nan=False)
    ref.b[..., 2048:] = rng.integers(0, 0x7F, ref.b[..., 2048:].shape, dtype=np.uint8)
    slots = rng.integers(-1, 70 * 32, 2113)
    K, V = (t.double().cpu().numpy() for t in fq.fq_kv4_read(torch.from_numpy(ref.b).cuda(), torch.from_numpy(slots).cuda()))
    for i in list(range(0, 2113, 37)) + [2112]:
        for h in range(2):
            for got, value in ((K, False), (V, True)):
                if slots[i] < 0:
                    assert not got[i, h].any()
                    continue
                c, sc = ref.get(int(slots[i]), h, value)
                assert np.array_equal(got[i, h], c * pu.E4M3[sc])
    again = fq.fq_kv4_read(torch.from_numpy(ref.b).cuda(), torch.from_numpy(np.sort(slots)).cuda())
    order = np.argsort(slots, kind="stable")
    assert np.array_equal(again[0].double().cpu().numpy(), K[order]) and np.array_equal(again[1].double().cpu().numpy(), V[order])
