"""The operators of a serving step one behind the other, as examples/sampled_serving.py uses them: each one's result against 64-bit arithmetic on what it was
really given, the step from a graph, and the example itself."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import chunk_util as cu
from test_gpu_norm_block import stream
from test_gpu_sample import check as check_token

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: torch.cuda.is_available() is False")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "sampled_serving.py")
    spec = importlib.util.spec_from_file_location("sampled_serving", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


class Seen:
    """Stands before the binding: keeps what the new operators were given and gave."""

    def __init__(self, fq):
        self.fq, self.calls = fq, []

    def __getattr__(self, name):
        f = getattr(self.fq, name)
        if name not in ("fq_rmsnorm_block", "fq_rmsnorm_block_quant", "fq_kv4_append_axes", "fq_kv4_attention_chunk", "fq_sample"):
            return f

        def call(*args, **kw):
            before = [a.clone() if isinstance(a, torch.Tensor) and name != "fq_kv4_append_axes" else a for a in args]
            r = f(*args, **kw)
            self.calls.append((name, before, kw, [t.clone() for t in (r if isinstance(r, tuple) else (r,))]))
            return r
        return call


def _check_chunk(fq, args, kw, out, rows):
    Q, qs, cache, table, starts, lens, scale = args
    G = Q.shape[1] // cache.shape[1]
    page = cache.shape[2] * 16
    for b in range(table.shape[0]):
        k, n, a = int(starts[b + 1] - starts[b]), int(lens[b]), int(starts[b])
        t = torch.arange(n, device="cuda")
        K, V = fq.fq_kv4_read(cache, table[b].long()[t // page] * page + t % page)
        for i, (lo, hi) in enumerate(cu.ranges(k, n, window=kw.get("window", 0))):
            if (a + i) % rows:
                continue
            for h in (0, G, Q.shape[1] - 1):
                key, value = (x[:, h // G].double().cpu().numpy() for x in (K, V))
                # (codes and scales apart are not needed: a code is at most 8 and a zero-point term at most 16 of its scale, 1 / 7 of the largest of a head at least)
                ks = np.abs(key).max(1, keepdims=True) / 4 + 1e-9
                tokens = (key, value, np.full_like(key, 8.0), ks, np.abs(value).max(1, keepdims=True) / 4 + 1e-9)
                o, tol = cu.attention(Q[a + i, h].cpu().numpy(), float(qs[a + i, h]), tokens, n - k + i, lo, hi, scale, kw["cap"], 0.0)
                assert (np.abs(out[a + i, h].double().cpu().numpy() - o) <= tol).all(), (b, i, h)


def test_every_operator_on_what_it_was_given(example, monkeypatch):
    fq = example.fq
    seen = Seen(fq)
    monkeypatch.setattr(example, "fq", seen)
    example.main(["--prompts", "70,9,33", "--chunk", "40", "--steps", "2", "--blocks", "2", "--vocabulary", "5003", "--no-graph"])
    names = [c[0] for c in seen.calls]
    passes = 2 + 2                                        # two chunks, two steps
    assert names.count("fq_kv4_attention_chunk") == names.count("fq_kv4_append_axes") == 2 * passes and names.count("fq_sample") == 3
    assert names.count("fq_rmsnorm_block_quant") == 3 * passes and names.count("fq_rmsnorm_block") == passes
    for name, args, kw, out in seen.calls:
        if name.startswith("fq_rmsnorm_block"):
            X, w, eps, R = args
            want, tol = stream(X, R, kw["post"], None, 1.0)
            assert ((out[-1].double() - want).abs() <= tol).all()
            same = fq.fq_rmsnorm(out[-1], w, eps) if name == "fq_rmsnorm_block" else fq.fq_rmsnorm_quant(out[-1], w, eps)[0]
            assert torch.equal(out[0], same)
        elif name == "fq_sample":
            logits = args[0].double().cpu().numpy()
            for b in range(logits.shape[0]):
                check_token(logits[b], int(out[0][b]), float(out[1][b]), float(args[1][b]), float(args[2][b]), int(args[3][b]), float(args[4][b]), float(args[5][b]))
        elif name == "fq_kv4_attention_chunk":
            _check_chunk(fq, args, kw, out[0], 7)


def test_a_chunked_prompt_caches_what_a_whole_one_does(example):
    """The first block's cache does not depend on the chunks (its keys and values come from the tokens alone)."""
    fq = example.fq
    got = []
    for chunk in (1000, 16):
        model = example.Model(blocks=1, pages=16, positions=500, vocabulary=1000)
        batch = example.Batch(model, [90, 17], 4)
        x = example.prefill(model, batch, chunk)
        t = torch.arange(90, device="cuda")
        got.append((fq.fq_kv4_read(model.blocks[0].cache, batch.slots(0, t, model.page)), x))
    # (a GEMM's kernel depends on its rows, and with it the last bit of a sum: a code beside a border, one of 7 steps, may fall on either side)
    for a, b in zip(got[0][0], got[1][0]):
        step = a.float().abs().amax(-1, keepdim=True) / 4
        assert ((a.float() - b.float()).abs() <= step).all() and (a != b).float().mean() < 0.02
    assert bool(torch.isfinite(got[0][1].float()).all()) and bool(torch.isfinite(got[1][1].float()).all())


def test_graph_and_eager_draw_the_same(example):
    args = ["--prompts", "50,3,100", "--chunk", "64", "--blocks", "2", "--vocabulary", "3001", "--steps"]
    graph, eager = example.main(args + ["6"]), example.main(args + ["6", "--no-graph"])
    assert torch.equal(graph[0], eager[0]) and torch.equal(graph[1], eager[1])
    assert (graph[0] >= 0).all() and (graph[0] < 3001).all() and bool(torch.isfinite(graph[1]).all())
