"""How the attention cuts sequences into parts, read from the workspace it asks for (256 compute units, the plan's default without a GPU)."""
import pytest
import torch

from paper_2505_20839_amd import binding

pytestmark = pytest.mark.skipif(torch.cuda.is_available() and torch.cuda.get_device_properties(0).multi_processor_count != 256, reason="256 compute units")


def parts(B, Hq, Hkv, max_len, prefix=0):
    """Parts of a row that go through memory; 0 where a sequence's own tokens are one part that leaves the output."""
    n = binding.fq_kv4_attention_workspace_bytes(B, Hq, Hkv, max_len, prefix)
    assert n % (B * Hq * 130 * 4) == 0
    return n // (B * Hq * 130 * 4)


@pytest.mark.parametrize("Hq, Hkv", [(32, 8), (8, 1), (64, 8), (5, 5), (40, 2)])
@pytest.mark.parametrize("max_len", [2050, 4000, 8000, 32001, 131072, 1 << 20])
def test_no_sequence_of_a_batch_is_left_to_a_few_long_parts(Hq, Hkv, max_len):
    """Lengths of a batch differ.  Whatever the number of heads, a part has at most 128 tiles, or a sixteenth of the longest sequence."""
    tiles = (max_len + 15) // 16
    for B in list(range(2, 40)) + [51, 64, 100, 128, 200, 256, 300]:
        n = max(1, parts(B, Hq, Hkv, max_len))
        assert -(-tiles // n) <= max(128, tiles // 16 + 16), (B, n)


def test_one_sequence_fills_the_compute_units_once():
    assert parts(1, 32, 8, 32001) == 32 and parts(1, 8, 1, 32001) == 63 and parts(1, 32, 8, 8000) == 32


def test_short_sequences_are_one_part():
    assert parts(1, 32, 8, 600) == 0 and parts(16, 32, 8, 1000) == 0 and parts(64, 32, 8, 1000) == 0
