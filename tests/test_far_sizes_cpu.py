"""Sizes past a C int are refused by the Python forms of the norms and the paged calls, not taken for their low 32 bits.

The tensors have shapes and no memory; nothing is launched (a call that got through would be refused for its null pointers)."""
import pytest
import torch

from paper_2505_20839_amd import binding

FAR = 1 << 32
SHAPE = -2


class Shape(torch.Tensor):
    is_cuda = property(lambda self: True)


def shape(*size, dtype=torch.bfloat16):
    return torch.empty(size, dtype=dtype, device="meta").as_subclass(Shape)


@pytest.fixture(autouse=True)
def without_a_stream(monkeypatch):
    monkeypatch.setattr(binding, "_stream", lambda: 0)


def refused(call, *a, **k):
    with pytest.raises(binding.FireqError) as e:
        call(*a, **k)
    assert e.value.status == SHAPE


@pytest.mark.parametrize("M, K", [(FAR + 3, 8), (1, FAR + 8), (2, 1 << 31), (1 << 31, 8)])
def test_norm(M, K):
    for call in (binding.fq_rmsnorm, binding.fq_rmsnorm_quant):
        refused(call, shape(M, K), shape(K), 1e-5)
        refused(call, shape(M, K), shape(K), 1e-5, residual=shape(M, K))


def test_cache_and_its_calls():
    i32, i64, u8 = torch.int32, torch.int64, torch.uint8
    rot, x = shape(4, 64, 2, dtype=torch.float32), shape(3, 1024)
    pos, slots = shape(3, dtype=i32), shape(3, dtype=i64)
    Q, qs = shape(3, 4, 128, dtype=u8), shape(3, 4, dtype=torch.float32)
    table, lens = shape(3, 5, dtype=i32), shape(3, dtype=i32)
    for size in ((FAR + 4, 2, 1, 2080), (4, 2, FAR + 1, 2080), (4, 2, 1 << 27, 2080), (1 << 31, 2, 1, 2080)):
        cache = shape(*size, dtype=u8)
        refused(binding.fq_kv4_read, cache, slots)
        refused(binding.fq_kv4_append, x, rot, pos, slots, cache)
        refused(binding.fq_kv4_attention, Q, qs, cache, table, lens, 0.1, max_len=9)
    cache = shape(4, 2, 1, 2080, dtype=u8)
    refused(binding.fq_kv4_read, cache, shape(FAR + 3, dtype=i64))
    refused(binding.fq_kv4_append, x, shape(FAR + 4, 64, 2, dtype=torch.float32), pos, slots, cache)
    refused(binding.fq_kv4_append, shape(FAR + 3, 1024), rot, shape(FAR + 3, dtype=i32), shape(FAR + 3, dtype=i64), cache)
    refused(binding.fq_kv4_append, shape(3, (FAR + 8) * 128), rot, pos, slots, cache)
    refused(binding.fq_kv4_attention, Q, qs, cache, shape(3, FAR + 5, dtype=i32), lens, 0.1, max_len=9)
    refused(binding.fq_kv4_attention_prefix, Q, qs, cache, shape(9, dtype=i32), 5, shape(3, FAR + 5, dtype=i32), lens, 0.1, max_len=9)
    far = [shape(FAR + 3, *t, dtype=d) for t, d in (((4, 128), u8), ((4,), torch.float32), ((5,), i32), ((), i32))]
    refused(binding.fq_kv4_attention, far[0], far[1], cache, far[2], far[3], 0.1, max_len=9)
    refused(binding.fq_kv4_attention, shape(1, FAR + 4, 128, dtype=u8), shape(1, FAR + 4, dtype=torch.float32), cache, shape(1, 5, dtype=i32), shape(1, dtype=i32), 0.1)


@pytest.mark.parametrize("at", range(5))
@pytest.mark.parametrize("far", [FAR, FAR + 100, 1 << 31, (1 << 33) + 4, -FAR + 4])
def test_workspace_of_far_sizes(at, far):
    a = [4, 32, 8, 60000, 5000]
    assert binding.fq_kv4_attention_workspace_bytes(*a) > 0
    a[at] = far
    assert binding.fq_kv4_attention_workspace_bytes(*a) == 0
