"""What fireq_norm_block.h, fireq_chunk.h and fireq_sample.h refuse, before any kernel is launched; the declared symbols; workspace sizes."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import chunk_util as cu
import paged_util as pu
from paper_2505_20839_amd import binding

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
P = 0x1000                                                # never dereferenced: validation fails first
ODD = 0x1008
OK, NULL, SHAPE, ALIGN, MEMORY = 0, -1, -2, -3, -5
INF = float("inf")


def test_declared_symbols_are_exported():
    names = set()
    for h in ("fireq_norm_block.h", "fireq_chunk.h", "fireq_sample.h"):
        src = re.sub(r"/\*.*?\*/", "", open(os.path.join(INCLUDE, h)).read(), flags=re.S)
        names |= set(re.findall(r"\b(fq_[a-z0-9_]+)\s*\(", src))
    assert names == {"fq_rmsnorm_block", "fq_rmsnorm_block_quant_ws", "fq_kv4_append_axes", "fq_kv4_attention_chunk_workspace_bytes",
                     "fq_kv4_attention_chunk_ws", "fq_sample_workspace_bytes", "fq_sample_bf16_ws", "fq_sample_fp32_ws"}
    for n in names:
        assert hasattr(binding.lib(), n)


@pytest.mark.parametrize("change, status", [
    (dict(M=0, X=0, w=0, Y=0, R=0, H=0), OK), (dict(M=-1), SHAPE), (dict(M=1 << 22), SHAPE), (dict(K=0), SHAPE), (dict(K=12), SHAPE), (dict(eps=0.0), SHAPE),
    (dict(eps=float("nan")), SHAPE), (dict(scale=INF), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(X=0), NULL), (dict(w=0), NULL), (dict(Y=0), NULL),
    (dict(R=0), NULL), (dict(H=0), NULL), (dict(R=0, H=0), NULL), (dict(rows=0x700000), NULL), (dict(X=ODD), ALIGN), (dict(post=0x600008), ALIGN),
    (dict(gate=0x600008), ALIGN), (dict(gate=0x600000, gates=0), SHAPE), (dict(gate=0x600000, gates=3), SHAPE), (dict(gate=0x600000, gates=5), SHAPE),
    (dict(gate=0x600000, gates=0, rows=0x700000), SHAPE),
    (dict(H=0x1010), SHAPE), (dict(H=0x200010), SHAPE), (dict(Y=0x1010), SHAPE), (dict(H=0x300000), SHAPE),
    (dict(post=0x400000), SHAPE), (dict(post=0x300100), SHAPE), (dict(gate=0x400100), SHAPE), (dict(gate=0x600000, gates=9, rows=0x400000), SHAPE),
    (dict(gate=0x300000 - 8 * 1024, gates=9, rows=0x700000), SHAPE)])     # the last of nine gates
@pytest.mark.parametrize("quant", [False, True])
def test_norm_block_refusals(change, status, quant):
    a = dict(X=P, R=0x200000, w=0x100000, eps=1e-5, H=0x400000, Y=0x300000, M=4, K=512, post=0, gate=0, rows=0, gates=1, scale=1.0)
    a.update(change)
    head = (a["X"], a["post"], a["gate"], a["rows"], a["gates"], ctypes.c_float(a["scale"]), a["R"], a["w"], ctypes.c_float(a["eps"]), a["H"], a["Y"])
    L = binding.lib()
    rc = L.fq_rmsnorm_block_quant_ws(*head, 0x500000, a["M"], a["K"], 0, 0, 0) if quant else L.fq_rmsnorm_block(*head, a["M"], a["K"], 0)
    assert rc == status


def test_norm_block_scale_and_workspace_refusals():
    L = binding.lib()
    f = ctypes.c_float
    head = (P, 0, 0x600000, 0, 1, f(1.0), 0x200000, 0x100000, f(1e-5), 0x400000, 0x300000)
    need = L.fq_w4a8_gemm_workspace_bytes(128, 256, 512)
    assert L.fq_rmsnorm_block_quant_ws(*head, 0, 128, 512, 0, 0, 0) == NULL
    for scales in (P, 0x200000, 0x100000, 0x400000, 0x300000, 0x600000):
        assert L.fq_rmsnorm_block_quant_ws(*head, scales, 128, 512, 0, 0, 0) == SHAPE
    assert L.fq_rmsnorm_block_quant_ws(*head, 0x800000, 128, 512, 0x900000, 64, 0) == MEMORY
    assert L.fq_rmsnorm_block_quant_ws(*head, 0x800000, 128, 512, 0x900008, need, 0) == ALIGN
    assert L.fq_rmsnorm_block_quant_ws(*head, 0x800000, 128, 520, 0x900000, 1 << 30, 0) == SHAPE
    for ws in (P, 0x600000, 0x800000, 0x400000):
        assert L.fq_rmsnorm_block_quant_ws(*head, 0x800000, 128, 512, ws, need, 0) == SHAPE


PAIRS = [0] * 32 + [1] * 31 + [-1]


@pytest.mark.parametrize("change, status", [
    (dict(T=0, QKV=0, slots=0, positions=0), OK), (dict(T=-1), SHAPE), (dict(axes=0), SHAPE), (dict(axes=128), SHAPE), (dict(axes=1), SHAPE),
    (dict(pairs=[2] + PAIRS[1:]), SHAPE), (dict(pairs=PAIRS[:63] + [-2]), SHAPE), (dict(pairs=None), NULL), (dict(QKV=0), NULL), (dict(positions=0), NULL),
    (dict(Q=ODD), ALIGN), (dict(page=24), SHAPE), (dict(Hq=5), SHAPE), (dict(ld=1016), SHAPE),
    (dict(Q=0x20000 + 16), SHAPE), (dict(positions=0x30000 - 12), SHAPE)])      # Q over the second axis' positions, the last of them over the cache
def test_append_axes_refusals(change, status):
    a = dict(QKV=P, ld=1024, cos_sin=0x10000, max_positions=8, positions=0x20000, axes=2, pairs=PAIRS, slots=0x28000, Q=0x40000, qs=0x50000, cache=0x30000,
             page_stride=4160, head_stride=2080, pages=4, page=16, T=3, Hq=4, Hkv=2)
    a.update(change)
    pairs = 0 if a["pairs"] is None else (ctypes.c_int8 * 64)(*a["pairs"])
    rc = binding.lib().fq_kv4_append_axes(a["QKV"], a["ld"], a["cos_sin"], a["max_positions"], a["positions"], a["axes"], pairs, a["slots"], 0, a["Q"], a["qs"],
                                          a["cache"], a["page_stride"], a["head_stride"], a["pages"], a["page"], a["T"], a["Hq"], a["Hkv"], 0)
    assert rc == status


@pytest.mark.parametrize("change, status", [
    (dict(T=0, Q=0, O=0), OK), (dict(B=0, Q=0, O=0), OK), (dict(T=-1), SHAPE), (dict(B=-1), SHAPE), (dict(B=65536), SHAPE), (dict(T=1 << 23), SHAPE), (dict(Hq=5), SHAPE),
    (dict(Hkv=0), SHAPE), (dict(T=1 << 22, Hq=16), SHAPE), (dict(max_new=-1), SHAPE), (dict(max_len=-1), SHAPE), (dict(max_len=(1 << 30) + 1), SHAPE),
    (dict(window=-1), SHAPE), (dict(cap=-1.0), SHAPE), (dict(cap=INF), SHAPE), (dict(cap=float("nan")), SHAPE), (dict(cap=1e-30), SHAPE), (dict(out_scale=0.0), SHAPE),
    (dict(out_scale=INF), SHAPE), (dict(out_scale=1e30, cap=1e-10), SHAPE), (dict(width=-1), SHAPE), (dict(pages=0), SHAPE), (dict(page=24), SHAPE),
    (dict(head_stride=2064), SHAPE), (dict(Q=0), NULL), (dict(qs=0), NULL), (dict(table=0), NULL), (dict(starts=0), NULL), (dict(lens=0), NULL), (dict(O=0), NULL),
    (dict(cache=0), NULL), (dict(Q=ODD), ALIGN), (dict(O=0x60008), ALIGN), (dict(O=P), SHAPE), (dict(O=0x30000), SHAPE), (dict(first=0x60010), SHAPE),
    (dict(end=0x60010), SHAPE), (dict(slopes=0x60000), SHAPE), (dict(starts=0x60000 - 8), SHAPE), (dict(lens=0x60000), SHAPE), (dict(qs=0x60000), SHAPE)])
def test_chunk_refusals(change, status):
    a = dict(Q=P, qs=0x10000, cache=0x30000, page_stride=4160, head_stride=2080, pages=4, page=16, table=0x20000, width=2, starts=0x21000, lens=0x22000, first=0,
             end=0, window=0, cap=0.0, slopes=0, out_scale=1.0, O=0x60000, T=3, B=2, Hq=4, Hkv=2, max_new=3, max_len=30, ws=0, n=0)
    a.update(change)
    f = ctypes.c_float
    rc = binding.lib().fq_kv4_attention_chunk_ws(a["Q"], a["qs"], a["cache"], a["page_stride"], a["head_stride"], a["pages"], a["page"], a["table"], a["width"],
                                                 a["starts"], a["lens"], a["first"], a["end"], a["window"], f(a["cap"]), a["slopes"], f(a["out_scale"]), a["O"],
                                                 a["T"], a["B"], a["Hq"], a["Hkv"], a["max_new"], a["max_len"], a["ws"], a["n"], 0)
    assert rc == status


def test_chunk_workspace():
    """Scratch where a row's tokens are cut into parts (256 compute units assumed without a GPU): 130 FP32 numbers a part and row."""
    need = binding.fq_kv4_attention_chunk_workspace_bytes
    assert need(1, 1, 32, 8, 1, 40) == 0
    n = need(1, 1, 32, 8, 1, 32001)
    assert n > 0 and n % (32 * 130 * 4) == 0
    for bad in ((0, 1, 32, 8, 1, 32001), (1, 0, 32, 8, 1, 32001), (1, 1, 30, 8, 1, 32001), (1, 1, 32, 8, -1, 32001), (1, 1, 32, 8, 1, -5), (1, 1, 32, 8, 1, 1 << 31),
                (1 << 40, 1, 32, 8, 1, 100)):
        assert need(*bad) == 0
    f, L = ctypes.c_float, binding.lib()
    call = lambda ws, size, O=0x6000000: L.fq_kv4_attention_chunk_ws(P, 0x10000, 0x300000, 8320 * 8, 8320, 4, 64, 0x20000, 600, 0x21000, 0x22000, 0, 0, 0, f(0.0), 0,  # noqa: E731
                                                                     f(1.0), O, 1, 1, 32, 8, 1, 32001, ws, size, 0)
    assert call(0, 0) == MEMORY and call(0x4000000, n - 1) == MEMORY and call(0x4000008, n) == ALIGN
    assert call(0x6000000 - n + 16, n) == SHAPE and call(P, n) == SHAPE and call(0x300000, n) == SHAPE


@pytest.mark.parametrize("change, status", [
    (dict(B=0, x=0, u=0, token=0), OK), (dict(B=-1), SHAPE), (dict(B=65536), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 20) + 1, ld=1 << 21), SHAPE), (dict(ld=39999), SHAPE),
    (dict(ld=(1 << 40) + 1), SHAPE), (dict(x=0), NULL), (dict(u=0), NULL), (dict(token=0), NULL), (dict(x=P + 1), ALIGN), (dict(ws=0), MEMORY), (dict(n=100), MEMORY),
    (dict(ws=0x900008), ALIGN), (dict(token=P + 64), SHAPE), (dict(logprob=P + 64), SHAPE), (dict(token=0x100000), SHAPE), (dict(token=0x110000), SHAPE),
    (dict(logprob=0x120000), SHAPE), (dict(logprob=0x150000), SHAPE), (dict(ws=P), SHAPE), (dict(ws=0x150000), SHAPE), (dict(ws=0x140000), SHAPE)])
@pytest.mark.parametrize("wide", [False, True])
def test_sample_refusals(change, status, wide):
    a = dict(x=P, ld=40000, u=0x100000, T=0x110000, k=0x120000, p=0x130000, m=0x140000, token=0x150000, logprob=0x160000, B=3, V=40000, ws=0x900000, n=1 << 24)
    a.update(change)
    call = binding.lib().fq_sample_fp32_ws if wide else binding.lib().fq_sample_bf16_ws
    assert call(a["x"], a["ld"], a["u"], a["T"], a["k"], a["p"], a["m"], a["token"], a["logprob"], a["B"], a["V"], a["ws"], a["n"], 0) == status


def test_sample_workspace_sizes():
    need = binding.fq_sample_workspace_bytes
    assert need(1, 1) == need(64, 32761) == 0 and need(64, 131072) > need(1, 131072) > need(1, 32762) > 0 and need(65535, 1 << 20) > 0
    for bad in ((0, 5), (-1, 5), (5, 0), (65536, 5), (1, (1 << 20) + 1), (1, 1 << 40)):
        assert need(*bad) == 0


def test_python_forms_refuse_tensors_that_are_not_on_a_gpu():
    x = torch.zeros((2, 128), dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="residual"):
        binding.fq_rmsnorm_block(x, x[0], 1e-5, None)
    with pytest.raises(TypeError, match="X must be a GPU tensor"):
        binding.fq_rmsnorm_block_quant(x, x[0], 1e-5, x)
    with pytest.raises(TypeError, match="positions must be a GPU tensor"):
        binding.fq_kv4_append_axes(x, x, x, [0] * 64, x, x)
    with pytest.raises(TypeError, match="Q must be a GPU tensor"):
        binding.fq_kv4_attention_chunk(x, x, x, x, x, x, 1.0)
    with pytest.raises(TypeError, match="logits must be a GPU tensor"):
        binding.fq_sample(x, x)


def test_reference_ranges_and_scores():
    """The oracle's own pins: hand-made ranges, and scores whose softmax is known."""
    assert cu.ranges(3, 5) == [(0, 3), (0, 4), (0, 5)]
    assert cu.ranges(2, 5, window=2) == [(2, 4), (3, 5)]
    assert cu.ranges(2, 1) == [(0, 0), (0, 1)]
    assert cu.ranges(2, 4, first=[1, 7], end=[9, 9]) == [(1, 4), (7, 4)]
    n = 4
    K, V = np.zeros((n, 128)), np.eye(n, 128)
    tokens = (K, V, K, np.zeros((n, 1)), np.ones((n, 1)))
    q = pu.to_e4m3(np.ones(128))
    o, _ = cu.attention(q, 1.0, tokens, 3, 0, 4, 1.0, 0.0, 0.0)
    assert np.allclose(o[:4], 0.25)
    o, _ = cu.attention(q, 1.0, tokens, 3, 0, 4, 1.0, 0.0, np.log(2.0))
    assert np.allclose(o[:4], np.array([1, 2, 4, 8]) / 15)
    K = K.copy()
    K[2, 0] = 1e6                                         # capped at 3: e^3 against 1
    o, _ = cu.attention(q, 1.0, (K, V, K, np.zeros((n, 1)), np.ones((n, 1))), 3, 0, 4, 1.0, 3.0, 0.0)
    assert np.allclose(o[:4], np.array([1, 1, np.exp(3), 1]) / (3 + np.exp(3)))


def test_gates_of_another_shape(monkeypatch):
    """K numbers in two dimensions are gates of fewer numbers each, of which rows would be read behind the tensor."""
    monkeypatch.setattr(binding, "_dev", lambda t, dtype, name: t)
    monkeypatch.setattr(binding, "_here", lambda *tensors: None)
    b = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)     # noqa: E731
    K = 16
    rows = torch.zeros(2, dtype=torch.int32)
    for gate, gate_rows in ((b(2, K // 2), None), (b(2, K // 2), rows), (b(K, 1), rows), (b(K, 1), None), (b(2, K + 1), None), (b(2 * K), None), (b(2, 2, K), rows)):
        with pytest.raises(binding.FireqError):
            binding._block_arguments("x", b(2, K), b(K), b(2, K), None, gate, gate_rows, 1.0, None)
    for gate, gate_rows, gates in ((b(K), None, 1), (b(1, K), None, 1), (b(1, 1, K), None, 1), (b(2, K), None, 2), (b(5, K), rows, 5)):
        assert binding._block_arguments("x", b(2, K), b(K), b(2, K), None, gate, gate_rows, 1.0, None)[2][4] == gates


@pytest.mark.parametrize("rows", [None, torch.zeros(2, dtype=torch.int32)])
def test_a_gate_of_no_rows(monkeypatch, rows):
    """A table without a gate is refused, and not taken for no gate (its data are NULL)."""
    monkeypatch.setattr(binding, "_dev", lambda t, dtype, name: t)
    monkeypatch.setattr(binding, "_here", lambda *tensors: None)
    x = torch.zeros((2, 16), dtype=torch.bfloat16)
    with pytest.raises(binding.FireqError):
        binding._block_arguments("x", x, x[0], x, None, x[:0], rows, 1.0, None)
