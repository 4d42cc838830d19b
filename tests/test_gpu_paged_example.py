"""examples/paged_decode.py: what the command returns and reports."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: torch.cuda.is_available() is False")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")
    spec = importlib.util.spec_from_file_location("paged_decode", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_eager_and_graph_end_alike(example):
    """The same seeds and the same number of steps: the last step's output, bit for bit; and other steps end elsewhere."""
    args = ["--batch", "3", "--prefix", "100", "--blocks", "1", "--steps"]
    graph, eager = example.main(args + ["5"]), example.main(args + ["5", "--no-graph"])
    assert bool(torch.isfinite(eager.float()).all()) and torch.equal(graph.view(torch.int16), eager.view(torch.int16))
    assert not torch.equal(eager.view(torch.int16), example.main(args + ["4", "--no-graph"]).view(torch.int16))


def test_without_a_shared_prompt(example):
    args = ["--batch", "2", "--prefix", "0", "--steps", "2", "--blocks", "1"]
    graph, eager = example.main(args), example.main(args + ["--no-graph"])
    assert bool(torch.isfinite(eager.float()).all()) and torch.equal(graph.view(torch.int16), eager.view(torch.int16))
