"""Serving prompts and sampled tokens with W4A8-FP layers: chunks of prompts, decoding and the choice of the next token, from one paged INT4 cache.

A batch of sequences, text with an image in it (positions on three axes: time, height, width), goes through a few decoder blocks with random weights.  A
block has a norm on both sides of its attention and of its feed-forward part, capped scores, and a window in every other block.  Prompts are cached and
attended to chunk by chunk; then every step takes one token of each sequence through the blocks and draws the next from its logits.  The step is
captured once into a HIP graph and replayed; tokens, lengths, slots and positions live on the GPU and move on by themselves.

    python examples/sampled_serving.py [--prompts 300,41,120] [--chunk 128] [--steps 32] [--blocks 2] [--vocabulary 32000] [--no-graph]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_20839_amd import binding as fq  # noqa: E402

EPS, CAP, WINDOW = 1e-5, 30.0, 256
AXES = [0] * 16 + [1] * 24 + [2] * 24                     # the axis that each pair of dimensions turns by


def rotation(positions, theta=500000.0):
    """float32 [positions, 64, 2]: cosine and sine of position * theta^(-2 i / 128), the angles in 64 bits."""
    a = torch.arange(positions, dtype=torch.float64)[:, None] * theta ** (-torch.arange(64, dtype=torch.float64) / 64)
    return torch.stack((a.cos(), a.sin()), dim=-1).float().contiguous().cuda()


def layer(g, N, K):
    """(packed INT4 weights, E4M3 group scales, per-tensor factor, N) of a random layer whose outputs are about as large as its inputs."""
    q = torch.randint(-8, 8, (N, K), generator=g, device="cuda", dtype=torch.int8)
    s = torch.full((N, K // 128), 0.25 / K ** 0.5, device="cuda") * (0.8 + 0.4 * torch.rand((N, K // 128), generator=g, device="cuda"))
    t = 2.0 ** -5                                          # keeps the group scales inside E4M3's range
    return fq.fq_pack_weights(q), (s / t).to(torch.float8_e4m3fn).view(torch.uint8), t, N


def places(length, image=(4, 6)):
    """int32 [3, length]: text, then an image of rows and columns, then text again."""
    i = torch.arange(length)
    rows, cols = image
    before, n = min(8, length), rows * cols
    j = (i - before).clamp(0, n - 1)
    inside = (i >= before) & (i < before + n)
    after = i - n + max(rows, cols)                       # text goes on behind the image's largest position
    text = torch.where(i < before, i, after)
    return torch.stack([torch.where(inside, before + v, text) for v in (0 * j, j // cols, j % cols)]).to(torch.int32)


class Block:
    def __init__(self, g, hidden, ffn, Hq, Hkv, pages, page, window):
        self.qkv, self.o = layer(g, (Hq + 2 * Hkv) * 128, hidden), layer(g, hidden, Hq * 128)
        self.gate_up, self.down = layer(g, 2 * ffn, hidden), layer(g, hidden, ffn)
        norm = lambda: (1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).bfloat16()   # noqa: E731
        self.norm1, self.post1, self.norm2, self.post2 = norm(), norm(), norm(), norm()
        self.cache, self.window = fq.fq_kv4_cache(pages, Hkv, page), window


class Model:
    def __init__(self, blocks=2, hidden=4096, ffn=11008, Hq=32, Hkv=8, page=32, pages=512, positions=32768, vocabulary=32000, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.Hq, self.Hkv, self.page = Hq, Hkv, page
        self.blocks = [Block(g, hidden, ffn, Hq, Hkv, pages, page, WINDOW if i % 2 else 0) for i in range(blocks)]
        self.rotation = rotation(positions)
        self.final = (1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).bfloat16()
        self.embedding = torch.randn((vocabulary, hidden), generator=g, device="cuda").bfloat16()
        self.head = layer(g, vocabulary, hidden)

    def forward(self, tokens, positions, slots, table, starts, lens, max_new, max_len):
        """bf16 [T, hidden] of the new tokens of all sequences (rows starts[b] .. starts[b + 1] - 1), which are cached on the way."""
        h = self.embedding[tokens]
        out = last = None
        for b in self.blocks:
            if out is None:
                A, s = fq.fq_rmsnorm_quant(h, b.norm1, EPS)
            else:                                         # the last block's output, its norm, the residual and this block's norm
                A, s, h = fq.fq_rmsnorm_block_quant(out, b.norm1, EPS, h, post=last.post2)
            Q, qs = fq.fq_kv4_append_axes(fq.fq_w4a8_gemm(A, s, *b.qkv), self.rotation, positions, AXES, slots, b.cache)
            O = fq.fq_kv4_attention_chunk(Q, qs, b.cache, table, starts, lens, 128 ** -0.5, max_new=max_new, max_len=max_len, cap=CAP, window=b.window)
            A, s = fq.fq_quantize_act(O.view(O.shape[0], -1))
            A, s, h = fq.fq_rmsnorm_block_quant(fq.fq_w4a8_gemm(A, s, *b.o), b.norm2, EPS, h, post=b.post1)
            _, A, s = fq.fq_w4a8_gemm_swiglu_quant(A, s, *b.gate_up)
            out, last = fq.fq_w4a8_gemm(A, s, *b.down), b
        return fq.fq_rmsnorm_block(out, self.final, EPS, h, post=last.post2)[0]

    def draw(self, x, u, sampling):
        """(int32 [B] tokens, float32 [B] log-probabilities) from the last rows' hidden states."""
        A, s = fq.fq_quantize_act(x)
        return fq.fq_sample(fq.fq_w4a8_gemm(A, s, *self.head), u, *sampling)


class Batch:
    """Sequences with their pages, lengths and sampling parameters."""

    def __init__(self, model, prompts, steps, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.B, self.prompts, page = len(prompts), prompts, model.page
        self.width = -(-(max(prompts) + steps) // page)
        self.table = torch.randperm(self.B * self.width, generator=g, device="cuda").to(torch.int32).reshape(self.B, self.width).contiguous()
        vocabulary = model.embedding.shape[0]
        self.tokens = [torch.randint(0, vocabulary, (n,), generator=g, device="cuda") for n in prompts]
        self.places = [places(n + steps).cuda() for n in prompts]
        self.u = torch.rand((steps + 1, self.B), generator=g, device="cuda")
        pick = lambda values, dtype: torch.tensor([values[i % len(values)] for i in range(self.B)], dtype=dtype, device="cuda")   # noqa: E731
        self.sampling = (pick([0.8, 1.0, 0.0], torch.float32), pick([50, 0, 0], torch.int32), pick([0.95, 0.9, 1.0], torch.float32), pick([0.0, 0.02], torch.float32))

    def slots(self, b, t, page):
        """int64 slots of sequence b's tokens t."""
        return self.table[b].long()[t // page] * page + t % page


def prefill(model, batch, chunk):
    """Prompts into the cache, `chunk` tokens of each at a time; the hidden states of their last tokens, bf16 [B, hidden]."""
    last = [None] * batch.B
    for lo in range(0, max(batch.prompts), chunk):
        new = [max(0, min(n, lo + chunk) - lo) for n in batch.prompts]
        t = [torch.arange(lo, lo + k, device="cuda") for k in new]
        rows = torch.tensor([0] + new).cumsum(0)
        x = model.forward(torch.cat([batch.tokens[b][lo:lo + k] for b, k in enumerate(new)]),
                          torch.cat([batch.places[b][:, lo:lo + k] for b, k in enumerate(new)], dim=1).contiguous(),
                          torch.cat([batch.slots(b, t[b], model.page) for b in range(batch.B)]), batch.table, rows.to(torch.int32).cuda(),
                          torch.tensor([min(n, lo + chunk) for n in batch.prompts], dtype=torch.int32, device="cuda"), max(new), lo + chunk)
        for b, k in enumerate(new):
            if k > 0 and lo + k == batch.prompts[b]:
                last[b] = x[rows[b + 1] - 1]
    return torch.stack(last)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompts", default="300,41,120,7")
    ap.add_argument("--chunk", type=int, default=128)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--vocabulary", type=int, default=32000)
    ap.add_argument("--no-graph", action="store_true")
    a = ap.parse_args(argv)
    prompts = [int(x) for x in a.prompts.split(",")]
    page = 32
    width = -(-(max(prompts) + a.steps) // page)
    model = Model(blocks=a.blocks, pages=len(prompts) * width, page=page, positions=max(prompts) + a.steps + 64, vocabulary=a.vocabulary)
    batch = Batch(model, prompts, a.steps)
    B = batch.B
    token, logprob = model.draw(prefill(model, batch, a.chunk), batch.u[0], batch.sampling)
    lens = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    every = torch.stack([p[:, : max(prompts) + a.steps] if p.shape[1] >= max(prompts) + a.steps else
                         torch.cat([p, p[:, -1:].expand(3, max(prompts) + a.steps - p.shape[1])], dim=1) for p in batch.places])   # [B, 3, tokens]
    step_of, u = torch.zeros(1, dtype=torch.long, device="cuda"), batch.u
    tokens = torch.zeros((a.steps + 1, B), dtype=torch.int32, device="cuda")
    logs = torch.zeros((a.steps + 1, B), device="cuda")
    tokens[0], logs[0] = token, logprob

    def step():
        """One token of every sequence: it is cached, attended from, and the next one drawn."""
        at = lens.long()
        now = tokens.index_select(0, step_of)[0].long()
        slots = batch.table.long().gather(1, (at // page)[:, None])[:, 0] * page + at % page
        positions = every.gather(2, at[:, None, None].expand(B, 3, 1))[:, :, 0].t().contiguous()
        lens.add_(1)
        step_of.add_(1)
        x = model.forward(now, positions, slots, batch.table, starts, lens, 1, width * page)
        t, p = model.draw(x, u.index_select(0, step_of)[0], batch.sampling)
        tokens.index_copy_(0, step_of, t[None])
        logs.index_copy_(0, step_of, p[None])

    run = step
    if not a.no_graph and a.steps > 1:
        kept = [v.clone() for v in (lens, step_of, tokens, logs)]
        step()                                            # (a first pass outside the graph; its token is drawn again)
        torch.cuda.synchronize()
        for v, k in zip((lens, step_of, tokens, logs), kept):
            v.copy_(k)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        run = graph.replay
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(a.steps):
        run()
    torch.cuda.synchronize()
    took = (time.perf_counter() - began) / max(1, a.steps)
    print("%d sequences of %s tokens, %d blocks: %.1f us a step, %.0f tokens/s; mean log-probability %.3f"
          % (B, a.prompts, a.blocks, took * 1e6, B / took, float(logs.mean())))
    return tokens, logs


if __name__ == "__main__":
    main()
