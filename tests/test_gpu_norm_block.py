"""The norm between two blocks (fireq_norm_block.h): its stream against 64-bit arithmetic, its norm bit for bit against the norm of that stream."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def fq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: torch.cuda.is_available() is False")
    from paper_2505_20839_amd import binding
    return binding


def make(M, K, seed=0, gates=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")     # noqa: E731
    x = n(M, K)
    x[:, :: 97] *= 20
    return (x.bfloat16(), (16 * n(M, K)).bfloat16(), (1 + 0.1 * n(K)).bfloat16(), (1 + 0.1 * n(K)).bfloat16(),
            torch.tanh(n(gates, K)).bfloat16() if gates else None)


def stream(x, r, post, gate, scale):
    """The exact stream and the bound of a bf16 one: half a step, and FP32's roundings (the sum of K squares, square root, quotient and four
    products) of the branch, and of the addition."""
    p = x.double()
    if post is not None:
        p = p / torch.sqrt(p.square().mean(-1, keepdim=True) + EPS) * post.double()
    if gate is not None:
        p = p * gate.double()
    b = float(np.float32(scale)) * p
    h = r.double() + b
    return h, 2.0 ** -8 * h.abs() + 2.0 ** -19 * (b.abs() + r.double().abs()) + 1e-38


CASES = [(1, 8), (1, 4096), (3, 128), (37, 2048), (2000, 1024), (5, 4104), (300, 5120), (7, 6144), (3, 6152), (9, 8192), (2, 8200), (64, 11008), (5, 12288), (3, 12296), (3, 16384), (4, 20000), (2, 32768), (3, 40000)]


@pytest.mark.parametrize("M, K", CASES)
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("kind", ["none", "one", "own", "rows"])
def test_stream_and_norm(fq, M, K, post, kind):
    gates = {"none": 0, "one": 1, "own": M, "rows": 5}[kind]
    x, r, w, pw, gate = make(M, K, M + K, gates)
    pw = pw if post else None
    rows = torch.randint(0, 5, (M,), device="cuda", dtype=torch.int32) if kind == "rows" else None
    scale = {"none": 1.0, "one": 0.3, "own": -2.0, "rows": 1.0}[kind]
    g = None if gate is None else gate[rows.long()] if rows is not None else gate
    want, tol = stream(x, r, pw, g, scale)
    keep = [t.clone() for t in (x, r)]
    Y, H = fq.fq_rmsnorm_block(x, w, EPS, r, post=pw, gate=gate, gate_rows=rows, scale=scale)
    assert ((H.double() - want).abs() <= tol).all()
    assert torch.equal(x, keep[0]) and torch.equal(r, keep[1])
    A, s, H2 = fq.fq_rmsnorm_block_quant(x, w, EPS, r, post=pw, gate=gate, gate_rows=rows, scale=scale)
    assert torch.equal(H, H2)
    # the norm behind it is that of the stream
    assert torch.equal(Y, fq.fq_rmsnorm(H, w, EPS))
    A1, s1 = fq.fq_rmsnorm_quant(H, w, EPS)
    assert torch.equal(A, A1) and torch.equal(s, s1)


def test_without_norm_gate_and_factor_it_is_the_residual_norm(fq):
    x, r, w, _, _ = make(40, 4096)
    Y, H = fq.fq_rmsnorm_block(x, w, EPS, r)
    Y1, H1 = fq.fq_rmsnorm(x, w, EPS, residual=r)
    assert torch.equal(H, H1) and torch.equal(Y, Y1)
    for kw in (dict(scale=0.0), dict(gate=torch.zeros(4096, dtype=torch.bfloat16, device="cuda"))):
        assert torch.equal(fq.fq_rmsnorm_block(x, w, EPS, r, post=w, **kw)[1], r)


@pytest.mark.parametrize("M, K", [(7, 4096), (3, 40000), (2000, 1024)])
def test_in_place(fq, M, K):
    x, r, w, pw, gate = make(M, K, 3, 1)
    want = fq.fq_rmsnorm_block_quant(x, w, EPS, r, post=pw, gate=gate)
    for over in (x, r):
        a, b = x.clone(), r.clone()
        out = a if over is x else b
        got = fq.fq_rmsnorm_block_quant(a, w, EPS, b, post=pw, gate=gate, out=out)
        assert got[2].data_ptr() == out.data_ptr()
        for u, v in zip(got, want):
            assert torch.equal(u, v)


@pytest.mark.parametrize("M", [100, 600])
def test_prepared_workspace(fq, M):
    """The GEMM behind it gives the same from the workspace that the norm has prepared."""
    N, K = 256, 1024
    x, r, w, pw, _ = make(M, K, 5)
    q = torch.randint(-8, 8, (N, K), device="cuda", dtype=torch.int8)
    packed, gs = fq.fq_pack_weights(q), torch.full((N, K // 128), 0.02, device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)
    ws = torch.full((fq.fq_w4a8_gemm_workspace_bytes(M, N, K),), 0xFF, dtype=torch.uint8, device="cuda")
    A, s, H = fq.fq_rmsnorm_block_quant(x, w, EPS, r, post=pw, workspace=ws)
    assert torch.equal(fq.fq_w4a8_gemm(A, s, packed, gs, 1.0, N, workspace=ws, workspace_prepared=True), fq.fq_w4a8_gemm(A, s, packed, gs, 1.0, N))


def test_rows_that_have_no_value(fq):
    """NaN, infinity, squares past FP32's range and a gate outside the gates spoil their rows and no other."""
    x, r, w, pw, gate = make(8, 512, 7, 3)
    x[1, 5], x[2, 9], x[3] = float("nan"), float("inf"), 2e25
    rows = torch.tensor([0, 1, 2, 0, -1, 3, 1, 2], dtype=torch.int32, device="cuda")
    A, s, H = fq.fq_rmsnorm_block_quant(x, w, EPS, r, post=pw, gate=gate, gate_rows=rows)
    Y, _ = fq.fq_rmsnorm_block(x, w, EPS, r, post=pw, gate=gate, gate_rows=rows)
    bad, good = [1, 2, 3, 4, 5], [0, 6, 7]
    assert torch.isnan(s[bad]).all() and (A[bad] == 0).all() and torch.isnan(Y[bad]).all() and torch.isnan(H[bad]).all()
    assert torch.isfinite(s[good]).all() and torch.isfinite(Y[good].float()).all() and torch.isfinite(H[good].float()).all()
    want, tol = stream(x, r, pw, gate[rows.long().clamp(0, 2)], 1.0)
    assert ((H.double() - want).abs() <= tol)[good].all()


def test_captured(fq):
    x, r, w, pw, gate = make(33, 4096, 9, 33)
    graph = torch.cuda.CUDAGraph()
    fq.fq_rmsnorm_block_quant(x, w, EPS, r, post=pw, gate=gate)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = fq.fq_rmsnorm_block_quant(x, w, EPS, r, post=pw, gate=gate)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, fq.fq_rmsnorm_block_quant(x, w, EPS, r, post=pw, gate=gate)):
            assert torch.equal(a, b)
        x.add_(0.5)
        r.copy_(out[2])
