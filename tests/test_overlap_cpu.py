"""Outputs and workspaces that lie over what a call still reads are refused, and what lies between a cache's tiles is not.

The addresses are made up and nothing is launched on them: without a GPU a call that is not refused ends in FQ_ERR_LAUNCH."""
import ctypes
import random

import pytest
import torch

from paper_2505_20839_amd import binding

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="a call that is not refused would run on made-up addresses")

SHAPE, LAUNCH = -2, -4
MB = 1 << 20
TILE = 2080
# pages of 32 tokens of 2 heads, in a pool of 3 layers of which this cache is the middle one
PER, HEAD, PAGE, PAGES = 2 * TILE, 2 * TILE, 3 * 2 * 2 * TILE, 5
CACHE = 64 * MB + 2 * 2 * TILE
END = CACHE + 4 * PAGE + HEAD + PER


def attention(prefix=False, **change):
    a = dict(Q=1 * MB, qs=2 * MB, cache=CACHE, page_stride=PAGE, head_stride=HEAD, shared=3 * MB, table=4 * MB, lens=5 * MB, O=6 * MB, ws=16 * MB)
    a.update(change)
    B, Hq, Hkv, width, most = 3, 8, 2, 100, 3000
    L = binding.lib()
    need = L.fq_kv4_attention_workspace_bytes(B, Hq, Hkv, most, 70 if prefix else 0)
    assert 0 < need < 16 * MB
    tail = (a["table"], width, a["lens"], ctypes.c_float(0.1), a["O"], B, Hq, Hkv, most, a["ws"], ctypes.c_size_t(need), 0)
    head = (a["Q"], a["qs"], a["cache"], a["page_stride"], a["head_stride"], PAGES, 32)
    return (L.fq_kv4_attention_prefix_ws(*head, a["shared"], 70, *tail) if prefix else L.fq_kv4_attention_ws(*head, *tail)), need


def append(**change):
    a = dict(QKV=1 * MB, ld=1856, cos_sin=2 * MB, positions=3 * MB, slots=4 * MB, Q=5 * MB, qs=6 * MB, cache=CACHE, page_stride=PAGE, head_stride=HEAD)
    a.update(change)
    return binding.lib().fq_kv4_append(a["QKV"], a["ld"], a["cos_sin"], 40, a["positions"], a["slots"], 0, a["Q"], a["qs"], a["cache"], a["page_stride"],
                                       a["head_stride"], PAGES, 32, 6, 10, 2, 0)


def read(**change):
    a = dict(cache=CACHE, page_stride=PAGE, head_stride=HEAD, slots=1 * MB, K=2 * MB, V=3 * MB)
    a.update(change)
    return binding.lib().fq_kv4_read(a["cache"], a["page_stride"], a["head_stride"], PAGES, 32, a["slots"], a["K"], a["V"], 7, 2, 0)


def test_what_lies_apart_is_taken():
    assert attention()[0] == attention(True)[0] == append() == read() == LAUNCH


@pytest.mark.parametrize("prefix", [False, True])
def test_attention_outputs_over_inputs(prefix):
    out = 3 * 8 * 256
    _, need = attention(prefix)
    inputs = dict(Q=3 * 8 * 128, qs=3 * 8 * 4, table=3 * 100 * 4, lens=12, **(dict(shared=12) if prefix else {}))
    for name, n in inputs.items():
        n16 = (n + 15) // 16 * 16
        for at in (0, n16 - 16, 16 - out):                # the output's first, last and only common bytes
            assert attention(prefix, **{"O": 32 * MB, name: 32 * MB - at})[0] == SHAPE, (name, at)
        for at in (n16, -out):
            assert attention(prefix, **{"O": 32 * MB, name: 32 * MB - at})[0] == LAUNCH, (name, at)
        for at in (0, n16 - 16, 16 - need):
            assert attention(prefix, **{"ws": 32 * MB, name: 32 * MB - at})[0] == SHAPE, (name, at)
    for at in (0, out - 16, 16 - need):
        assert attention(prefix, ws=32 * MB, O=32 * MB - at)[0] == SHAPE
    assert attention(prefix, ws=32 * MB, O=32 * MB - out)[0] == attention(prefix, ws=32 * MB, O=32 * MB + need)[0] == LAUNCH
    for at in (CACHE, CACHE + HEAD, CACHE + HEAD + PER - 16, CACHE + PAGE - out + 16, END - 16, CACHE - out + 16):
        assert attention(prefix, O=at)[0] == SHAPE, at
    for at in (CACHE - out, CACHE + HEAD + PER, CACHE + PAGE - out, CACHE + 2 * PAGE + HEAD + PER, END):   # before, behind, other layers' tiles
        assert attention(prefix, O=at)[0] == LAUNCH, at
    for at in (CACHE, CACHE - need + 16, END - 16):
        assert attention(prefix, ws=at)[0] == SHAPE
    assert attention(prefix, ws=CACHE - need)[0] == attention(prefix, ws=(END + 15) // 16 * 16)[0] == LAUNCH


def test_append_outputs_over_inputs():
    q, s, rows = 6 * 10 * 128, 6 * 10 * 4, 14 * 256
    for name, n in dict(cos_sin=40 * 512, positions=24, slots=48).items():
        n16 = (n + 15) // 16 * 16
        for out, no in (("Q", q), ("qs", s)):
            for at in (0, n16 - 16, 16 - no):
                assert append(**{out: 32 * MB, name: 32 * MB - at}) == SHAPE, (name, out, at)
            assert append(**{out: 32 * MB, name: 32 * MB - n16}) == append(**{out: 32 * MB, name: 32 * MB + no}) == LAUNCH
    assert append(Q=32 * MB, qs=32 * MB + 16) == append(Q=32 * MB, qs=32 * MB + q - 16) == SHAPE
    X = 32 * MB
    for i in (0, 1, 5):                                   # strided rows of 14 heads: Q over a row
        for at in (X + i * 3712, X + i * 3712 + rows - 16):
            assert append(QKV=X, Q=at) == append(QKV=X, qs=at) == SHAPE
    assert append(QKV=X, qs=X + 3 * 3712 - 64) == SHAPE
    assert append(QKV=X, ld=16384, Q=X + 2 * 32768 + rows) == LAUNCH     # between two rows
    assert append(QKV=X, Q=X + 5 * 3712 + rows) == append(QKV=X, Q=X - q) == LAUNCH
    for name in ("QKV", "cos_sin", "positions", "slots", "Q", "qs"):
        for at in (CACHE, CACHE + HEAD, CACHE + 3 * PAGE, END - 16):
            assert append(**{name: at}) == SHAPE, (name, at)
        assert append(**{name: END}) == LAUNCH


def test_read_outputs_over_inputs():
    n = 7 * 2 * 256
    assert read(K=32 * MB, V=32 * MB) == read(K=32 * MB, V=32 * MB + n - 16) == read(K=32 * MB, V=32 * MB - n + 16) == SHAPE
    assert read(K=32 * MB, V=32 * MB + n) == LAUNCH
    for out in ("K", "V"):
        assert read(**{out: 32 * MB, "slots": 32 * MB + 64}) == read(**{out: 32 * MB, "slots": 32 * MB - 40}) == SHAPE
        assert read(**{out: CACHE}) == read(**{out: CACHE + 4 * PAGE - 16}) == read(**{out: END - 16}) == SHAPE
        assert read(**{out: CACHE + HEAD + PER}) == read(**{out: END}) == LAUNCH


def test_gaps_of_any_layout():
    """Against every block of random layouts (heads inside pages, and outside) one by one."""
    rng = random.Random(1)
    n = 7 * 2 * 256
    for _ in range(3000):
        inner = PER + 16 * rng.choice([0, 0, 1, 300, 700])
        if rng.random() < 0.5:
            head, page = inner, inner + PER + 16 * rng.choice([0, 3, 250, 2000])
        else:
            page, head = inner, 4 * inner + PER + 16 * rng.choice([0, 3, 250, 2000])
        at = CACHE + 16 * rng.randrange(-n // 16 - 2, (4 * page + head + PER) // 16 + 2)
        meets = any(at < CACHE + p * page + h * head + PER and CACHE + p * page + h * head < at + n for p in range(PAGES) for h in range(2))
        assert read(page_stride=page, head_stride=head, K=at) == (SHAPE if meets else LAUNCH), (page, head, at - CACHE)


def norm(residual=False, **change):
    M, K = 100, 256
    need = binding.lib().fq_w4a8_gemm_workspace_bytes(M, 256, K)
    a = dict(X=1 * MB, R=2 * MB, w=3 * MB, H=4 * MB, A=5 * MB, s=6 * MB, ws=7 * MB)
    a.update(change)
    return binding.lib().fq_rmsnorm_quant_ws(a["X"], a["R"] if residual else 0, a["w"], ctypes.c_float(1e-5), a["H"] if residual else 0, a["A"], a["s"], M, K,
                                             a["ws"], need, 0), need


@pytest.mark.parametrize("residual", [False, True])
def test_norm_scales_and_workspace_over_the_rest(residual):
    rc, need = norm(residual)
    assert rc == LAUNCH and need > 0 and need % 16 == 0
    arrays = dict(X=100 * 512, w=512, A=100 * 256, **(dict(R=100 * 512, H=100 * 512) if residual else {}))
    for out, no in (("s", 400), ("ws", need)):
        for name, n in arrays.items():
            for at in (0, n - 16, 16 - no):
                assert norm(residual, **{out: 32 * MB, name: 32 * MB - at})[0] == SHAPE, (out, name, at)
            for at in (n, -no):
                assert norm(residual, **{out: 32 * MB, name: 32 * MB - at})[0] == LAUNCH, (out, name, at)
    assert norm(residual, s=32 * MB, ws=32 * MB)[0] == norm(residual, s=32 * MB + need - 4, ws=32 * MB)[0] == SHAPE
    if residual:                                          # the stream in place is still taken
        assert norm(True, H=1 * MB)[0] == norm(True, H=2 * MB)[0] == LAUNCH
