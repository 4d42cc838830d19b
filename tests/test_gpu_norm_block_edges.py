"""The norm between two blocks (fireq_norm_block.h): gates of shapes that it refuses, and rows that have no norm."""
import pytest
import torch

from test_gpu_norm_block import EPS, fq, make  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["fq_rmsnorm_block", "fq_rmsnorm_block_quant"])
def test_gates_of_another_shape(fq, name):  # noqa: F811
    """K numbers in two dimensions are no gate of K numbers, with rows named or not."""
    M, K = 2, 512
    x, r, w, _, gate = make(M, K, 3, 1)
    rows = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for shape in ((2, K // 2), (K // 8, 8), (K, 1)):
        for kw in ({}, {"gate_rows": rows}):
            with pytest.raises(fq.FireqError):
                getattr(fq, name)(x, w, EPS, r, gate=gate.reshape(shape), **kw)
    want = getattr(fq, name)(x, w, EPS, r, gate=gate)
    for got in (getattr(fq, name)(x, w, EPS, r, gate=gate.reshape(K)), getattr(fq, name)(x, w, EPS, r, gate=gate.reshape(1, 1, K))):
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("name", ["fq_rmsnorm_block", "fq_rmsnorm_block_quant"])
def test_a_gate_of_no_rows(fq, name):  # noqa: F811
    x, r, w, _, gate = make(3, 512, 5, 3)
    rows = torch.zeros(3, dtype=torch.int32, device="cuda")
    for kw in ({}, {"gate_rows": rows}):
        with pytest.raises(fq.FireqError):
            getattr(fq, name)(x, w, EPS, r, gate=gate[:0], **kw)


@pytest.mark.parametrize("M, K", [(6, 512), (6, 40000)])
def test_numbers_that_are_not_finite_without_a_norm_of_their_own(fq, M, K):  # noqa: F811
    """Without `post` they reach their own place in the stream alone, and the norm behind it as any stream's do; a gate outside the gates spoils the row."""
    x, r, w, _, gate = make(M, K, 11, 2)
    x[1, 5], x[2, 9], x[3, 7] = float("nan"), float("inf"), 3e38
    rows = torch.tensor([0, 1, 0, 1, 2, -1], dtype=torch.int32, device="cuda")
    for kw, g in (({}, torch.ones((M, K), device="cuda").bfloat16()), ({"gate": gate, "gate_rows": rows}, gate[rows.long().clamp(0, 1)])):
        Y, H = fq.fq_rmsnorm_block(x, w, EPS, r, scale=0.5, **kw)
        A, s, H2 = fq.fq_rmsnorm_block_quant(x, w, EPS, r, scale=0.5, **kw)
        # FP32 and one rounding: half a step of bf16, and 2^-22 of the terms for a product and a sum
        want = r.double() + 0.5 * g.double() * x.double()
        tol = 2.0 ** -8 * want.abs() + 2.0 ** -22 * (r.double().abs() + x.double().abs()) + 1e-38
        lost = torch.zeros(M, dtype=torch.bool, device="cuda")
        if kw:
            lost[4:] = True
        fine = torch.isfinite(want) & ~lost[:, None]
        assert ((H.double() - want).abs() <= tol)[fine].all() and int((~fine).sum()) == 2 + (2 * K if kw else 0)
        assert torch.isnan(H[lost].float()).all() and torch.isnan(H[1, 5].float()) and torch.isinf(H[2, 9].float())
        assert torch.equal(H.view(torch.int16), H2.view(torch.int16))
        A1, s1 = fq.fq_rmsnorm_quant(H, w, EPS)
        assert torch.equal(A, A1) and torch.equal(s.isnan(), s1.isnan()) and torch.equal(s[~s.isnan()], s1[~s.isnan()])
        assert torch.equal(torch.isnan(Y.float()), torch.isnan(fq.fq_rmsnorm(H, w, EPS).float()))
