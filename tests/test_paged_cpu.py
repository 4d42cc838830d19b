"""What fireq_norm.h and fireq_paged.h refuse, before any kernel is launched; the declared symbols; the reference's own pins."""
import ctypes
import os
import re
import subprocess
import sys

import numpy as np
import pytest
import torch

import paged_util as pu
from paper_2505_20839_amd import binding

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
P = 0x1000                                                # never dereferenced: validation fails first
ODD = 0x1008
F1, NAN = ctypes.c_float(1.0), ctypes.c_float(float("nan"))
OK, NULL, SHAPE, ALIGN, MEMORY = 0, -1, -2, -3, -5


def test_declared_symbols_are_exported():
    names = set()
    for h in ("fireq_norm.h", "fireq_paged.h"):
        src = re.sub(r"/\*.*?\*/", "", open(os.path.join(INCLUDE, h)).read(), flags=re.S)
        names |= set(re.findall(r"\b(fq_[a-z0-9_]+)\s*\(", src))
    assert names == {"fq_rmsnorm", "fq_rmsnorm_quant_ws", "fq_kv4_append", "fq_kv4_read", "fq_kv4_attention_workspace_bytes",
                     "fq_kv4_attention_ws", "fq_kv4_attention_prefix_ws"}
    for n in names:
        assert hasattr(binding.lib(), n)


@pytest.mark.parametrize("change, status", [
    (dict(M=0, X=0, w=0, Y=0), OK), (dict(M=-1), SHAPE), (dict(M=1 << 22), SHAPE), (dict(K=0), SHAPE), (dict(K=12), SHAPE), (dict(eps=0.0), SHAPE),
    (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE), (dict(X=0), NULL), (dict(w=0), NULL),
    (dict(Y=0), NULL), (dict(R=0x200000), NULL), (dict(H=0x200000), NULL), (dict(X=ODD), ALIGN), (dict(w=ODD), ALIGN), (dict(Y=0x300008), ALIGN),
    (dict(R=0x200008, H=0x400000), ALIGN),
    (dict(R=0x200000, H=0x200010), SHAPE), (dict(R=0x200000, H=0x1010), SHAPE),     # partly over an input
    (dict(R=0x200000, H=0x300000), SHAPE), (dict(Y=0x1010), SHAPE), (dict(w=0x300000), SHAPE)])
@pytest.mark.parametrize("quant", [False, True])
def test_norm_refusals(change, status, quant):
    a = dict(X=P, R=0, w=0x100000, eps=1e-5, H=0, Y=0x300000, M=4, K=512)
    a.update(change)
    L = binding.lib()
    if quant:
        rc = L.fq_rmsnorm_quant_ws(a["X"], a["R"], a["w"], ctypes.c_float(a["eps"]), a["H"], a["Y"], 0x500000, a["M"], a["K"], 0, 0, 0)
    else:
        rc = L.fq_rmsnorm(a["X"], a["R"], a["w"], ctypes.c_float(a["eps"]), a["H"], a["Y"], a["M"], a["K"], 0)
    assert rc == status


def test_norm_workspace_refusals():
    L = binding.lib()
    need = L.fq_w4a8_gemm_workspace_bytes(128, 256, 512)
    args = (P, 0, 0x100000, F1, 0, 0x300000)
    assert L.fq_rmsnorm_quant_ws(*args, 0, 128, 512, 0, 0, 0) == NULL
    assert L.fq_rmsnorm_quant_ws(*args, 0x500000, 128, 512, P, 64, 0) == MEMORY
    assert L.fq_rmsnorm_quant_ws(*args, 0x500000, 128, 512, ODD, need, 0) == ALIGN
    assert L.fq_rmsnorm_quant_ws(*args, 0x500000, 128, 520, P, 1 << 30, 0) == SHAPE       # groups of 128
    assert L.fq_rmsnorm_quant_ws(*args, 0x500000, 128, 16512, P, 1 << 30, 0) == SHAPE


PAGED = [(dict(page=0), SHAPE), (dict(page=24), SHAPE), (dict(pages=-1), SHAPE), (dict(page_stride=8), SHAPE), (dict(page_stride=0), SHAPE),
         (dict(head_stride=2064), SHAPE), (dict(page_stride=2064), SHAPE), (dict(head_stride=2088), SHAPE), (dict(cache=0), NULL), (dict(cache=ODD), ALIGN), (dict(Hkv=0), SHAPE)]


@pytest.mark.parametrize("change, status", PAGED + [
    (dict(T=0, QKV=0, slots=0, positions=0), OK), (dict(T=-1), SHAPE), (dict(Hq=0), SHAPE), (dict(Hq=5), SHAPE), (dict(ld=1016), SHAPE), (dict(ld=1028), SHAPE),
    (dict(max_positions=-1), SHAPE), (dict(T=1 << 28), SHAPE), (dict(QKV=0), NULL), (dict(slots=0), NULL), (dict(positions=0), NULL), (dict(cos_sin=0), NULL),
    (dict(Q=0), NULL), (dict(qs=0), NULL), (dict(QKV=ODD), ALIGN), (dict(cos_sin=ODD), ALIGN), (dict(Q=ODD), ALIGN)])
def test_append_refusals(change, status):
    a = dict(QKV=P, ld=1024, cos_sin=P, max_positions=8, positions=P, slots=P, Q=P, qs=P, cache=P, page_stride=4160, head_stride=2080, pages=4, page=16,
             T=3, Hq=4, Hkv=2)
    a.update(change)
    rc = binding.lib().fq_kv4_append(a["QKV"], a["ld"], a["cos_sin"], a["max_positions"], a["positions"], a["slots"], 0, a["Q"], a["qs"], a["cache"],
                                     a["page_stride"], a["head_stride"], a["pages"], a["page"], a["T"], a["Hq"], a["Hkv"], 0)
    assert rc == status


@pytest.mark.parametrize("change, status", PAGED + [
    (dict(n=0, slots=0, K=0, V=0), OK), (dict(n=-1), SHAPE), (dict(n=1 << 28), SHAPE), (dict(slots=0), NULL), (dict(K=0), NULL), (dict(V=0), NULL),
    (dict(K=ODD), ALIGN), (dict(V=ODD), ALIGN)])
def test_read_refusals(change, status):
    a = dict(cache=P, page_stride=4160, head_stride=2080, pages=4, page=16, slots=P, K=P, V=P, n=3, Hkv=2)
    a.update(change)
    rc = binding.lib().fq_kv4_read(a["cache"], a["page_stride"], a["head_stride"], a["pages"], a["page"], a["slots"], a["K"], a["V"], a["n"], a["Hkv"], 0)
    assert rc == status


@pytest.mark.parametrize("prefix", [False, True])
@pytest.mark.parametrize("change, status", PAGED + [
    (dict(B=0, Q=0, O=0), OK), (dict(B=-1), SHAPE), (dict(B=65536), SHAPE), (dict(Hq=5), SHAPE), (dict(B=65535, Hq=256), SHAPE), (dict(width=-1), SHAPE),
    (dict(max_len=-1), SHAPE), (dict(prefix_len=-1), SHAPE), (dict(max_len=(1 << 30) + 1), SHAPE), (dict(prefix_len=(1 << 30) + 1), SHAPE), (dict(scale=0.0), SHAPE), (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE),
    (dict(scale=float("inf")), SHAPE), (dict(pages=0), SHAPE), (dict(Q=0), NULL), (dict(qs=0), NULL), (dict(lens=0), NULL), (dict(table=0), NULL), (dict(O=0), NULL),
    (dict(shared=0), NULL), (dict(Q=ODD), ALIGN), (dict(O=ODD), ALIGN), (dict(ws=0), MEMORY), (dict(nbytes=64), MEMORY), (dict(ws=ODD), ALIGN)])
def test_attention_refusals(change, status, prefix):
    a = dict(Q=P, qs=P, cache=P, page_stride=4160, head_stride=2080, pages=4, page=16, shared=P, prefix_len=100, table=P, width=4000, lens=P, scale=0.1, O=P, B=2, Hq=4,
             Hkv=2, max_len=60000, ws=P, nbytes=1 << 40)
    a.update(change)
    if not prefix and ("prefix_len" in change or "shared" in change):
        return
    L = binding.lib()
    tail = (a["table"], a["width"], a["lens"], ctypes.c_float(a["scale"]), a["O"], a["B"], a["Hq"], a["Hkv"], a["max_len"], a["ws"], ctypes.c_size_t(a["nbytes"]), 0)
    head = (a["Q"], a["qs"], a["cache"], a["page_stride"], a["head_stride"], a["pages"], a["page"])
    rc = L.fq_kv4_attention_prefix_ws(*head, a["shared"], a["prefix_len"], *tail) if prefix else L.fq_kv4_attention_ws(*head, *tail)
    assert rc == status


def test_attention_workspace_sizes():
    size = binding.fq_kv4_attention_workspace_bytes
    assert size(0, 32, 8, 100) == 0 and size(4, 5, 2, 100) == 0 and size(4, 32, 8, -1) == 0
    # whole rows of 128 sums, a maximum and a sum in FP32 for each part of each query head
    assert size(4, 32, 8, 100000, 0) % (4 * 32 * 130 * 4) == 0 and size(4, 32, 8, 100000, 0) > 0
    assert size(4, 32, 8, 10, 5000) % (4 * 32 * 130 * 4) == 0 and size(4, 32, 8, 10, 5000) > 0


def test_no_workspace_for_sizes_that_are_refused():
    """In a process of its own: such sizes must not end the caller."""
    code = """from paper_2505_20839_amd import binding
for B, Hq, Hkv in ((2 ** 31 - 1, 64, 1), (65536, 8, 8), (1, 2 ** 31 - 1, 1), (65535, 256, 1), (2 ** 31 - 1, 2 ** 31 - 1, 1), (2 ** 30, 2 ** 30, 2 ** 30)):
    for prefix in (0, 1, 5000, 1 << 30):
        assert binding.fq_kv4_attention_workspace_bytes(B, Hq, Hkv, 100, prefix) == 0, (B, Hq, Hkv, prefix)
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=os.path.dirname(INCLUDE))
    assert r.returncode == 0, (r.returncode, r.stderr[-300:])


@pytest.mark.parametrize("max_len", [1 << 30, (1 << 30) - 5, 300000001, 131072000, 5000000])
@pytest.mark.parametrize("B, heads", [(8, 1), (1, 8), (64, 8), (600, 1)])
def test_parts_of_long_bounds_are_whole_steps(B, heads, max_len):
    """A step takes two tiles and may not pass the end of its part: some even number of tiles gives this number of parts."""
    parts, tiles = binding.fq_kv4_attention_workspace_bytes(B, heads, heads, max_len) // (B * heads * 130 * 4), (max_len + 15) // 16
    assert 1 < parts <= 60000
    assert any((tiles + n - 1) // n == parts for n in range(16, tiles + 16, 16) if abs(n * parts - tiles) <= n + 16 * parts)


def test_binding_wants_gpu_tensors():
    t = torch.zeros((2, 128))
    for call in (lambda: binding.fq_rmsnorm(t, t, 1e-5), lambda: binding.fq_rmsnorm_quant(t, t, 1e-5), lambda: binding.fq_kv4_read(t, t),
                 lambda: binding.fq_kv4_append(t, t, t, t, t), lambda: binding.fq_kv4_attention(t, t, t, t, t, 1.0),
                 lambda: binding.fq_kv4_attention_prefix(t, t, t, t, 1, t, t, 1.0), lambda: binding.fq_kv4_attention_prefix(t, t, t, None, 1, t, t, 1.0)):
        with pytest.raises(TypeError, match="GPU tensor"):
            call()
    with pytest.raises(TypeError, match="workspace must be a GPU tensor"):
        binding._scratch(t)
    with pytest.raises(binding.FireqError):
        binding.fq_kv4_cache(4, 2, 24, device="cpu")
    assert tuple(binding.fq_kv4_cache(4, 2, 48, device="cpu").shape) == (4, 2, 3, 2080)


# ---- the reference's own pins ----

def test_places_fill_a_tile_once():
    """Every nibble of a page belongs to one number, and the scales lie behind them."""
    for place in (pu.key_place, pu.value_place):
        seen = {(at, hi) for t in range(32) for d in range(128) for at, hi in [place(t, d)]}
        assert len(seen) == 32 * 128
    at = {pu.key_place(t, d)[0] for t in range(16) for d in range(128)}
    assert at == set(range(1024)) and {pu.value_place(t, d)[0] for t in range(16) for d in range(128)} == set(range(1024, 2048))
    assert sorted(pu.scale_place(t, v) for t in range(16) for v in (False, True)) == list(range(2048, 2080))
    assert pu.key_place(17, 49) == (2080 + 256 + 16 + 1, 1) and pu.value_place(5, 70) == (1024 + 256 + 96 + 8 + 2, 0)


def test_reference_attention_by_hand():
    one = np.full(128, 0x38, np.uint8)                    # 1.0
    K = np.zeros((2, 128)); V = np.stack([np.full(128, 1.0), np.full(128, 3.0)])
    kc, s = np.zeros((2, 128)), np.ones((2, 1))
    o, tol = pu.attention(one, 1.0, K, V, kc, s, s, 1.0)
    assert np.allclose(o, 2.0) and (tol < 0.1).all()
    K[1, 0] = np.log(3.0)
    assert np.allclose(pu.attention(one, 1.0, K, V, kc, s, s, 1.0)[0], 2.5)


def test_reference_rotation_and_int4():
    cs = np.stack([np.full(64, np.cos(0.5)), np.full(64, np.sin(0.5))], -1)
    x = np.zeros(128); x[3] = 1.0
    r = pu.rotate(x, cs, False)
    assert np.allclose([r[3], r[67]], [np.cos(0.5), np.sin(0.5)]) and np.count_nonzero(r) == 2
    r = pu.rotate(x, cs, True)
    assert np.allclose([r[2], r[3]], [-np.sin(0.5), np.cos(0.5)])
    x = np.zeros(128, np.float32); x[:3] = [7.0, -3.5, 2.5]
    assert list(pu.int4(x)[0][:3]) == [7, -4, 2] and pu.int4(x)[1] == 0x38
    assert pu.int4(np.zeros(128, np.float32)) [1] == 0
