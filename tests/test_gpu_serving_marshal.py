"""The native argument marshalling of the operators of a serving step against the Python form: the same results, exceptions and messages."""
import numpy as np
import pytest

from test_gpu_marshal import _same, _Sub, fq  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _b(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


@pytest.mark.parametrize("M, K", [(1, 128), (37, 1024), (200, 512)])
@pytest.mark.parametrize("name", ["fq_rmsnorm_block", "fq_rmsnorm_block_quant"])
def test_norm_block_calls(fq, name, M, K):  # noqa: F811
    x, r, w, post = _b(M, K), _b(M, K, seed=1), _b(K, seed=2), _b(K, seed=3)
    rows = torch.randint(0, 3, (M,), device="cuda", dtype=torch.int32)
    for kw in ({}, {"post": post}, {"gate": post}, {"gate": _b(1, K)}, {"gate": _b(M, K)}, {"gate": _b(3, K), "gate_rows": rows}, {"scale": 2}, {"scale": 0.3}):
        _same(fq, name, lambda: ((x, w, 1e-5, r), kw), native=True)
    _same(fq, name, lambda: ((x, w, 1e-5, r), {"out": torch.empty_like(x)}), native=True)
    _same(fq, name, lambda: (lambda h: ((x, w, 1e-5, h), {"out": h}))(r.clone()), native=True)
    _same(fq, name, lambda: ((x, w, np.float32(1e-5), r), {}), native=False)
    _same(fq, name, lambda: ((x.as_subclass(_Sub), w, 1e-5, r), {}), native=False)
    for bad, kw, exc in [((x.float(), w, 1e-5, r), {}, TypeError), ((x, w, 1e-5, None), {}, TypeError), ((x, w[:-8], 1e-5, r), {}, fq.FireqError),
                         ((x, w, 1e-5, r[:, :-8].contiguous()), {}, fq.FireqError), ((x, w, -1.0, r), {}, fq.FireqError), ((x, w, 1e-5, r), {"scale": float("inf")}, fq.FireqError),
                         ((x, w, 1e-5, r), {"post": post[:-8]}, fq.FireqError), ((x, w, 1e-5, r), {"gate": _b(M + 3, K)}, fq.FireqError),
                         ((x, w, 1e-5, r), {"gate_rows": rows}, fq.FireqError), ((x, w, 1e-5, r), {"gate": _b(3, K), "gate_rows": rows.long()}, TypeError),
                         ((x, w, 1e-5, r), {"out": torch.empty_like(x).float()}, TypeError), ((x, w, 1e-5, r.cpu()), {}, TypeError)]:
        _same(fq, name, lambda: (bad, kw), exc)
    if name == "fq_rmsnorm_block_quant" and M > 64:
        need = fq.fq_w4a8_gemm_workspace_bytes(M, 256, K)
        _same(fq, name, lambda: ((x, w, 1e-5, r), {"workspace": torch.empty(need, dtype=torch.uint8, device="cuda")}), native=True)
        _same(fq, name, lambda: ((x, w, 1e-5, r), {"workspace": torch.empty(64, dtype=torch.uint8, device="cuda")}), fq.FireqError)


@pytest.mark.parametrize("T", [1, 20])
def test_append_axes_calls(fq, T):  # noqa: F811
    Hq, Hkv = 4, 2
    x, rot = _b(T, (Hq + 2 * Hkv) * 128), torch.rand((100, 64, 2), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    pos = torch.randint(0, 100, (3, T), device="cuda", dtype=torch.int32)
    slots = torch.arange(T, device="cuda")
    axis = [j % 3 for j in range(64)]
    cache = fq.fq_kv4_cache(2, Hkv, 16)
    for a in (axis, tuple(axis), [-1] * 64):
        _same(fq, "fq_kv4_append_axes", lambda: ((x, rot, pos, a, slots, cache), {}), native=True)
    _same(fq, "fq_kv4_append_axes", lambda: ((x, rot, pos, axis, slots, cache), {"interleaved": True}), native=True)
    _same(fq, "fq_kv4_append_axes", lambda: ((x, rot, pos, np.array(axis), slots, cache), {}), native=False)
    _same(fq, "fq_kv4_append_axes", lambda: ((x, rot, pos, torch.tensor(axis), slots, cache), {}), native=False)
    for bad, exc in [((x, rot, pos, axis[:-1], slots, cache), fq.FireqError), ((x, rot, pos, [3] * 64, slots, cache), fq.FireqError),
                     ((x, rot, pos, [-2] + axis[1:], slots, cache), fq.FireqError), ((x, rot, pos, [1 << 80] + axis[1:], slots, cache), fq.FireqError),
                     ((x, rot, pos[0], axis, slots, cache), fq.FireqError), ((x, rot, pos[:, :-1].contiguous(), axis, slots, cache), fq.FireqError),
                     ((x, rot, pos.long(), axis, slots, cache), TypeError), ((x, rot, None, axis, slots, cache), TypeError), ((x.float(), rot, pos, axis, slots, cache), TypeError),
                     ((x, rot, pos, None, slots, cache), TypeError), ((x, rot, pos, axis, slots.int(), cache), TypeError)]:
        _same(fq, "fq_kv4_append_axes", lambda: (bad, {}), exc)


@pytest.mark.parametrize("new, B", [(1, 3), (40, 2)])
def test_chunk_calls(fq, new, B):  # noqa: F811
    Hq, Hkv, page, n = 4, 2, 16, 60
    g = torch.Generator(device="cuda").manual_seed(new)
    cache = torch.randint(0, 0x70, (4 * B, Hkv, 1, 2080), generator=g, device="cuda", dtype=torch.uint8)
    T = B * new
    q, qs = torch.randint(0, 0x60, (T, Hq, 128), generator=g, device="cuda", dtype=torch.uint8), torch.rand((T, Hq), generator=g, device="cuda") * 0.01
    table = torch.arange(4 * B, device="cuda", dtype=torch.int32).reshape(B, 4)
    starts, lens = torch.arange(0, T + 1, new, device="cuda", dtype=torch.int32), torch.full((B,), n, device="cuda", dtype=torch.int32)
    ok = (q, qs, cache, table, starts, lens, 0.1)
    i32 = lambda v: torch.full((T,), v, device="cuda", dtype=torch.int32)     # noqa: E731
    slopes = torch.rand(Hq, generator=g, device="cuda")
    out = lambda: torch.empty((T, Hq, 128), dtype=torch.bfloat16, device="cuda")   # noqa: E731
    name = "fq_kv4_attention_chunk"
    for kw in ({}, {"max_new": new}, {"max_len": n}, {"max_new": 1, "max_len": 64}, {"first": i32(3)}, {"end": i32(20)}, {"window": 7}, {"cap": 5}, {"cap": 2.5}, {"slopes": slopes},
               {"first": i32(1), "end": i32(50), "window": 9, "cap": 1.0, "slopes": slopes}):
        _same(fq, name, lambda: (ok, kw), native=True)
    _same(fq, name, lambda: (ok, {"out": out()}), native=True)
    _same(fq, name, lambda: (ok, {"out": out().view(T, Hq * 128)}), native=True)
    _same(fq, name, lambda: (ok, {"window": np.int64(7)}), native=False)
    for bad, kw, exc in [((q.float(),) + ok[1:], {}, TypeError), (ok[:2] + (cache[..., :-16],) + ok[3:], {}, fq.FireqError), (ok[:4] + (starts[:-1],) + ok[5:], {}, fq.FireqError),
                         (ok[:5] + (lens[:-1],) + ok[6:], {}, fq.FireqError), (ok[:6] + (-1.0,), {}, fq.FireqError), (ok, {"cap": -1.0}, fq.FireqError), (ok, {"window": -1}, fq.FireqError),
                         (ok, {"first": i32(3)[:-1]}, fq.FireqError), (ok, {"end": i32(3).long()}, TypeError), (ok, {"slopes": slopes[:-1]}, fq.FireqError),
                         (ok, {"max_len": 1 << 40}, fq.FireqError), (ok, {"max_len": -1}, fq.FireqError), (ok, {"max_new": -3}, fq.FireqError), (ok, {"max_new": 1 << 40}, fq.FireqError),
                         (ok, {"out": out()[:-1]}, fq.FireqError), (ok, {"out": out().float()}, TypeError), (ok[:3] + (table.long(),) + ok[4:], {}, TypeError)]:
        _same(fq, name, lambda: (bad, kw), exc)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sample_calls(fq, dtype):  # noqa: F811
    B, V = 5, 33001
    x = _b(B, V).to(dtype)
    u, T, p = torch.rand(B, device="cuda"), torch.full((B,), 0.7, device="cuda"), torch.full((B,), 0.9, device="cuda")
    k = torch.full((B,), 20, dtype=torch.int32, device="cuda")
    for a, kw in (((x, u), {}), ((x, u, T), {}), ((x, u, T, k, p, p), {}), ((x, u), {"top_p": p}), ((x, u), {"min_p": p * 0.1}), ((x[:, 3:2000], u), {})):
        _same(fq, "fq_sample", lambda: (a, kw), native=True)
    need = fq.fq_sample_workspace_bytes(B, V)
    _same(fq, "fq_sample", lambda: ((x, u), {"workspace": torch.empty(need, dtype=torch.uint8, device="cuda")}), native=True)
    _same(fq, "fq_sample", lambda: ((x, u), {"workspace": torch.empty(need - 1, dtype=torch.uint8, device="cuda")}), fq.FireqError)
    _same(fq, "fq_sample", lambda: ((x.as_subclass(_Sub), u), {}), native=False)
    for bad, exc in [((x.half(), u), TypeError), ((x.cpu(), u), TypeError), ((x, u[:-1]), fq.FireqError), ((x, None), TypeError), ((x[0], u), fq.FireqError), ((x, u.double()), TypeError),
                     ((x, u, T, k.long()), TypeError), ((x, u, T[:-1]), fq.FireqError), ((x.t(), u), ValueError), ((x[:, ::2], u), ValueError),
                     ((torch.zeros((2, (1 << 20) + 1), dtype=dtype, device="cuda"), u[:2].contiguous()), fq.FireqError)]:
        _same(fq, "fq_sample", lambda: (bad, {}), exc)
    assert [t.numel() for t in fq.fq_sample(x[:0], u[:0])] == [0, 0]
