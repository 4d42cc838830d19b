"""Positions on several axes (fireq_chunk.h): codes and scales bit for bit against 64-bit arithmetic, and against the one-axis append."""
import numpy as np
import pytest
import torch

import paged_util as pu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: torch.cuda.is_available() is False")
    from paper_2505_20839_amd import binding
    return binding


def table(n):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(64) / 64)
    return np.stack((np.cos(a), np.sin(a)), axis=-1).astype(np.float32)


SECTIONS = [0] * 16 + [1] * 24 + [2] * 24
IN_TURN = [j % 3 for j in range(64)]
PARTIAL = [0] * 20 + [1] * 12 + [-1] * 32


@pytest.mark.parametrize("axis", [SECTIONS, IN_TURN, PARTIAL, [-1] * 64, [4, 0, 2, 1] * 16], ids=["sections", "in turn", "partial", "none", "any"])
@pytest.mark.parametrize("T, Hq, Hkv, page", [(1, 4, 1, 16), (37, 6, 2, 48), (5, 9, 3, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_against_the_definition(fq, axis, T, Hq, Hkv, page, interleaved):
    rng = np.random.default_rng(T + Hq)
    axes = max(max(axis) + 1, 1)
    rot = table(500)
    pos = rng.integers(0, 500, (axes, T)).astype(np.int32)
    x = torch.as_tensor(rng.standard_normal((T, (Hq + 2 * Hkv) * 128)).astype(np.float32)).bfloat16()
    cache = pu.Cache(T // page + 2, Hkv, page, rng)
    slots = rng.permutation(len(cache.b) * page)[:T].astype(np.int64)
    slots[T // 2] = -1
    dev = torch.as_tensor(cache.b).cuda()
    Q, qs = fq.fq_kv4_append_axes(x.cuda(), torch.as_tensor(rot).cuda(), torch.as_tensor(pos).cuda(), axis, torch.as_tensor(slots).cuda(), dev, interleaved=interleaved)
    Q, qs = Q.cpu().numpy(), qs.cpu().numpy()
    a = np.array(axis)
    heads = x.float().numpy().reshape(T, -1, 128)
    for i in range(T):
        cs = np.where((a >= 0)[:, None], rot[pos[np.maximum(a, 0), i], np.arange(64)], np.float32([1.0, 0.0]))
        for h in range(Hq + Hkv):
            y = pu.rotate(heads[i, h], cs, interleaved)
            if h < Hq:
                s = np.float32(np.abs(y).max()) / np.float32(448)
                assert qs[i, h] == s
                assert (pu.to_e4m3(y / s) == Q[i, h]).all()
            elif slots[i] >= 0:
                cache.put(int(slots[i]), h - Hq, False, *pu.int4(y))
        for h in range(Hkv):
            if slots[i] >= 0:
                cache.put(int(slots[i]), h, True, *pu.int4(heads[i, Hq + Hkv + h]))
    assert (dev.cpu().numpy() == cache.b).all()


@pytest.mark.parametrize("T, Hq, Hkv", [(1, 32, 8), (300, 32, 8), (700, 40, 40)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_axes_alike_are_one_axis(fq, T, Hq, Hkv, interleaved):
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, (Hq + 2 * Hkv) * 128 + 256), generator=g, device="cuda").bfloat16()[:, 128:-128]    # strided rows
    rot = torch.as_tensor(table(1000)).cuda()
    pos = torch.randint(0, 1000, (T,), generator=g, device="cuda", dtype=torch.int32)
    slots = torch.arange(T, device="cuda") + 5
    one, many = fq.fq_kv4_cache(T // 32 + 2, Hkv, 32), fq.fq_kv4_cache(T // 32 + 2, Hkv, 32)
    a = fq.fq_kv4_append(x, rot, pos, slots, one, interleaved=interleaved)
    b = fq.fq_kv4_append_axes(x, rot, pos[None].expand(3, T).contiguous(), SECTIONS, slots, many, interleaved=interleaved)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(one, many)


def test_positions_outside_the_table(fq):
    """On an axis that a pair turns by they spoil the row; on one that no pair turns by they do not."""
    T, Hq, Hkv = 6, 4, 2
    x = torch.randn((T, (Hq + 2 * Hkv) * 128), device="cuda").bfloat16()
    rot = torch.as_tensor(table(50)).cuda()
    pos = torch.full((3, T), 7, dtype=torch.int32, device="cuda")
    pos[0, 1], pos[1, 2], pos[2, 3], pos[2, 4] = 50, -1, 50, 2 ** 31 - 1
    slots = torch.arange(T, device="cuda")
    for axis, bad in ((SECTIONS, [1, 2, 3, 4]), ([0] * 32 + [1] * 32, [1, 2]), ([-1] * 63 + [2], [3, 4])):
        cache = fq.fq_kv4_cache(1, Hkv, 16)
        _, s = fq.fq_kv4_append_axes(x, rot, pos, axis, slots, cache)
        K, V = fq.fq_kv4_read(cache, slots)
        good = [i for i in range(T) if i not in bad]
        assert torch.isnan(s[bad]).all() and torch.isnan(K[bad]).all() and torch.isnan(V[bad]).all()
        assert torch.isfinite(s[good]).all() and torch.isfinite(K[good].float()).all()


def test_captured(fq):
    T, Hq, Hkv = 20, 8, 2
    x = torch.randn((T, (Hq + 2 * Hkv) * 128), device="cuda").bfloat16()
    rot = torch.as_tensor(table(500)).cuda()
    pos = torch.randint(0, 100, (3, T), device="cuda", dtype=torch.int32)
    slots, cache = torch.arange(T, device="cuda"), fq.fq_kv4_cache(2, Hkv, 16)
    axis = list(SECTIONS)
    fq.fq_kv4_append_axes(x, rot, pos, axis, slots, cache)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = fq.fq_kv4_append_axes(x, rot, pos, axis, slots, cache)
    axis[:] = [0] * 64                                    # (the axes were taken at the call)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        other = fq.fq_kv4_cache(2, Hkv, 16)
        want = fq.fq_kv4_append_axes(x, rot, pos, SECTIONS, slots, other)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
        assert torch.equal(fq.fq_kv4_read(cache, slots)[0], fq.fq_kv4_read(other, slots)[0])
        pos.add_(17)


@pytest.mark.parametrize("axis", [0, 2])
@pytest.mark.parametrize("interleaved", [False, True])
def test_all_pairs_by_one_axis(fq, axis, interleaved):
    """The one-axis append's queries and cache, whatever the other axes' positions are."""
    T, Hq, Hkv = 41, 6, 2
    g = torch.Generator(device="cuda").manual_seed(axis)
    x = torch.randn((T, (Hq + 2 * Hkv) * 128), generator=g, device="cuda").bfloat16()
    rot = torch.rand((50, 64, 2), generator=g, device="cuda")
    pos = torch.full((3, T), 1 << 30, device="cuda", dtype=torch.int32)
    pos[axis] = torch.randint(0, 50, (T,), generator=g, device="cuda", dtype=torch.int32)
    slots = torch.randperm(64, generator=g, device="cuda")[:T]
    a, b = fq.fq_kv4_cache(4, Hkv, 16), fq.fq_kv4_cache(4, Hkv, 16)
    got = fq.fq_kv4_append_axes(x, rot, pos, [axis] * 64, slots, a, interleaved)
    want = fq.fq_kv4_append(x, rot, pos[axis].contiguous(), slots, b, interleaved)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(a, b)
