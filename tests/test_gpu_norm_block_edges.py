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
