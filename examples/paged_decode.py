"""Decoding with W4A8-FP layers from a paged INT4 key/value cache: the library's operators together, as a serving loop uses them.

A batch of sequences shares a prompt prefix (a system prompt) and decodes token by token through a few decoder blocks with random
weights.  Per block and step: residual + norm to FP8 -> QKV layer -> rotation, FP8 queries, INT4 keys and values into the cache ->
attention over the shared and the own pages -> output layer + residual -> norm to FP8 -> gate/up layer with SiLU -> down layer +
residual.  The step is captured once into a HIP graph and replayed; lengths, slots and positions live on the GPU and move on by themselves.

    python examples/paged_decode.py [--batch 16] [--prefix 1000] [--steps 64] [--blocks 2] [--no-graph]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_20839_amd import binding as fq  # noqa: E402

EPS = 1e-5


def rotation(positions, theta=500000.0):
    """float32 [positions, 64, 2]: cosine and sine of position * theta^(-2 i / 128), the angles in 64 bits."""
    freq = theta ** (-torch.arange(64, dtype=torch.float64) / 64)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * freq
    return torch.stack((a.cos(), a.sin()), dim=-1).float().contiguous().cuda()


def layer(g, N, K):
    """(packed INT4 weights, E4M3 group scales, N) of a random layer whose outputs are about as large as its inputs."""
    q = torch.randint(-8, 8, (N, K), generator=g, device="cuda", dtype=torch.int8)
    s = torch.full((N, K // 128), 0.25 / K ** 0.5, device="cuda") * (0.8 + 0.4 * torch.rand((N, K // 128), generator=g, device="cuda"))
    t = 2.0 ** -5                                          # per-tensor factor: keeps the group scales inside E4M3's range
    return fq.fq_pack_weights(q), (s / t).to(torch.float8_e4m3fn).view(torch.uint8), t, N


class Block:
    def __init__(self, g, hidden, ffn, Hq, Hkv, pages, page):
        self.qkv, self.o = layer(g, (Hq + 2 * Hkv) * 128, hidden), layer(g, hidden, Hq * 128)
        self.gate_up, self.down = layer(g, 2 * ffn, hidden), layer(g, hidden, ffn)
        self.norm1, self.norm2 = ((1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).bfloat16() for _ in range(2))
        self.cache = fq.fq_kv4_cache(pages, Hkv, page)


def gemm(A, s, w, **kw):
    return fq.fq_w4a8_gemm(A, s, w[0], w[1], w[2], w[3], **kw)


class Decoder:
    """`blocks` decoder blocks over a pool of pages; sequences own their rows of `table`, the prefix its pages."""

    def __init__(self, blocks=2, hidden=4096, ffn=11008, Hq=32, Hkv=8, page=32, pages=512, positions=32768, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.Hq, self.Hkv, self.page = Hq, Hkv, page
        self.blocks = [Block(g, hidden, ffn, Hq, Hkv, pages, page) for _ in range(blocks)]
        self.rotation = rotation(positions)
        self.final = (1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).bfloat16()

    def forward(self, x, positions, slots, attend):
        """bf16 [T, hidden] through all blocks.  `attend(block, Q, q_scale)` -> bf16 [T, Hq * 128]; the new tokens are cached before it."""
        h, out = x, None
        for b in self.blocks:
            if out is None:
                A, s = fq.fq_rmsnorm_quant(h, b.norm1, EPS)
            else:                                         # the stream takes the last block's output on the way into the norm
                A, s, h = fq.fq_rmsnorm_quant(out, b.norm1, EPS, residual=h)
            Q, qs = fq.fq_kv4_append(gemm(A, s, b.qkv), self.rotation, positions, slots, b.cache)
            A, s = fq.fq_quantize_act(attend(b, Q, qs))
            h = fq.fq_w4a8_gemm_add(A, s, *b.o, h)
            A, s = fq.fq_rmsnorm_quant(h, b.norm2, EPS)
            _, A, s = fq.fq_w4a8_gemm_swiglu_quant(A, s, *b.gate_up)
            out = gemm(A, s, b.down)
        return fq.fq_rmsnorm(out, self.final, EPS, residual=h)[0]

    def prefill(self, x, pages_of):
        """A prompt of T tokens into the cache, in pages `pages_of`; its own attention over the keys and values as the cache holds them."""
        T = x.shape[0]
        t = torch.arange(T, device="cuda")
        slots = pages_of.long()[t // self.page] * self.page + t % self.page

        def attend(b, Q, qs):
            K, V = (v.float().repeat_interleave(self.Hq // self.Hkv, dim=1).transpose(0, 1).contiguous() for v in fq.fq_kv4_read(b.cache, slots))
            q = (Q.view(torch.float8_e4m3fn).float() * qs[..., None]).transpose(0, 1).contiguous()
            score = torch.matmul(q, K.transpose(1, 2).contiguous()) * 128 ** -0.5
            score.masked_fill_(t[None, :] > t[:, None], float("-inf"))
            return torch.matmul(torch.softmax(score, dim=-1), V).transpose(0, 1).reshape(T, -1).bfloat16()

        return self.forward(x, t.to(torch.int32), slots, attend)

    def step(self, x, table, lens, prefix_pages, prefix, max_len):
        """One token of every sequence: x bf16 [B, hidden]; lens int32 [B] counts the tokens of its own that a sequence has with this one."""
        last = (lens - 1).long()
        slots = table.long().gather(1, (last // self.page)[:, None])[:, 0] * self.page + last % self.page

        def attend(b, Q, qs):
            if prefix_pages is None:
                O = fq.fq_kv4_attention(Q, qs, b.cache, table, lens, 128 ** -0.5, max_len=max_len)
            else:
                O = fq.fq_kv4_attention_prefix(Q, qs, b.cache, prefix_pages, prefix, table, lens, 128 ** -0.5, max_len=max_len)
            return O.view(O.shape[0], -1)

        return self.forward(x, lens - 1 + prefix, slots, attend)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--prefix", type=int, default=1000)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--no-graph", action="store_true")
    a = ap.parse_args(argv)
    B, page, steps = a.batch, 32, a.steps
    width, shared = -(-(steps + 4) // page), -(-a.prefix // page)
    d = Decoder(blocks=a.blocks, pages=B * width + shared, page=page, positions=a.prefix + steps + 2)
    g = torch.Generator(device="cuda").manual_seed(1)
    order = torch.randperm(B * width + shared, generator=g, device="cuda").to(torch.int32)
    table, prefix_pages = order[: B * width].reshape(B, width).contiguous(), order[B * width:].contiguous()
    if a.prefix:
        d.prefill(torch.randn((a.prefix, 4096), generator=g, device="cuda").bfloat16(), prefix_pages)
    x = torch.randn((B, 4096), generator=g, device="cuda").bfloat16()
    lens = torch.ones(B, dtype=torch.int32, device="cuda")

    def step():
        y = d.step(x, table, lens, prefix_pages, a.prefix, max_len=width * page)
        x.copy_(y)                                        # (the next token's embedding, in a model with a vocabulary)
        lens.add_(1)
        return y

    step()
    torch.cuda.synchronize()
    run = step
    if not a.no_graph:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = step()

        def run():
            graph.replay()
            return y

    last = run()
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(steps):
        last = run()
    torch.cuda.synchronize()
    took = (time.perf_counter() - began) / steps
    print("%d sequences behind %d shared tokens, %d blocks: %.1f us a step, %.0f tokens/s; finite: %s"
          % (B, a.prefix, a.blocks, took * 1e6, B / took, bool(torch.isfinite(last.float()).all())))
    return last


if __name__ == "__main__":
    main()
