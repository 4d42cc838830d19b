"""Operators of a serving step beside those of ``perf/operators.py``, for timing and comparison: prompts and chunks of prompts over
the paged INT4 cache with shaped scores, positions on several axes, blocks with norms on both sides, and the choice of the next token,
through ``paper_2505_20839_amd.binding``.

Sizes are those of the repository's workloads (hidden 4096 and 5120, 32 query heads over 8 key/value heads of 128) at token counts from
one decode row to a prompt of 8192, uneven ones among them, caches of one token to some ten thousands per sequence in pages of 16 to
128 tokens, and vocabularies of 32000 to 131072.

Kinds of case:
  block   what stands between two blocks with a norm on both sides: norm of the block's output, its gate and scale, the residual, the
          next block's norm to E4M3 codes and row scales (form "quant") or bf16; fq_rmsnorm_block_quant, fq_rmsnorm_block
  axes    the QKV layer's output into the cache with positions on several axes (time, height, width), a pair of dimensions turning with
          one of them or not at all, then the tokens read back; fq_kv4_append_axes, fq_kv4_read
  chunk   one or many new tokens per sequence against their cached tokens: a range of tokens for each row (causal, documents, a
          prefix that is seen whole), a window, scores capped by a tanh, a bias that grows with the distance; fq_kv4_attention_chunk
  sample  a token for each row of logits by temperature, min-p, top-k and top-p, from given uniform numbers, and its
          log-probability; fq_sample

A cache is uint8 [pages, heads, page / 16, 2080]: per 16 tokens of a head 1024 bytes of key codes, 1024 bytes of value codes
and 32 bytes of scales.  A code is the INT4 number + 8.
  keys    byte 256 g + 16 t + j (token t): dimension 32 g + j in the low nibble, 32 g + 16 + j in the high one
  values  byte 1024 + 256 p + 16 n + 4 m + b: token 4 p + (0, 2, 1, 3)[b], channel n + 32 m low, n + 32 m + 16 high
  scales  byte 2048 + 8 p + i: E4M3 scale of the key of token 4 p + i; 2048 + 8 p + 4 + i: of its value
Slot s is token s % page of page s // page.
"""
import math

import torch

own = False

D = 128                                                   # head width
TILE = 2080                                               # bytes of 16 tokens of a head
EPS = 1e-5
SCALE = D ** -0.5


def listed():
    return [
        # one token between two blocks: launch and host latency
        {"name": "block_token", "kind": "block", "form": "quant", "M": 1, "K": 4096, "post": True, "gates": 0, "scale": 1.0},
        # seven sequences with a gate each, an uneven prompt batch; bf16 for a layer that is not quantised
        {"name": "block_1000_gated", "kind": "block", "form": "bf16", "M": 1000, "K": 5120, "post": True, "gates": 7, "scale": 1.0},
        # a prefill of 8192 tokens, scaled residual branch
        {"name": "block_8192", "kind": "block", "form": "quant", "M": 8192, "K": 4096, "post": True, "gates": 0, "scale": 0.25},
        # a decode batch of 37 sequences behind images
        {"name": "axes_batch_37", "kind": "axes", "T": 37, "Hq": 32, "Hkv": 8, "page": 16, "axes": 3, "mixed": False, "still": 0, "interleaved": False},
        # text and a large image, uneven
        {"name": "axes_6001", "kind": "axes", "T": 6001, "Hq": 32, "Hkv": 8, "page": 64, "axes": 3, "mixed": False, "still": 0, "interleaved": False},
        # a decode batch at all lengths, empty rows among them, capped scores
        {"name": "decode_capped_37", "kind": "chunk", "B": 37, "new": 1, "longest": 6000, "Hq": 32, "Hkv": 8, "page": 16, "ragged": True,
         "cap": 30.0, "bias": False, "window": 0, "mask": "causal"},
        # one long sequence, one token, biased by distance
        {"name": "decode_biased_long", "kind": "chunk", "B": 1, "new": 1, "longest": 32001, "Hq": 32, "Hkv": 8, "page": 64, "ragged": False,
         "cap": 0.0, "bias": True, "window": 0, "mask": "causal"},
        # a chunk of a prompt behind what is cached already, in a window
        {"name": "chunk_200_window", "kind": "chunk", "B": 1, "new": 200, "longest": 16201, "Hq": 32, "Hkv": 8, "page": 32, "ragged": False,
         "cap": 50.0, "bias": False, "window": 4096, "mask": "causal"},
        # prompts packed of documents, padding rows among them
        {"name": "prompt_documents_5", "kind": "chunk", "B": 5, "new": 2100, "longest": 2100, "Hq": 32, "Hkv": 8, "page": 64, "ragged": True,
         "cap": 0.0, "bias": False, "window": 0, "mask": "documents"},
        # one long prompt, capped, whose first part is seen whole
        {"name": "prompt_8192", "kind": "chunk", "B": 1, "new": 8192, "longest": 8192, "Hq": 32, "Hkv": 8, "page": 64, "ragged": False,
         "cap": 30.0, "bias": False, "window": 0, "mask": "prefix"},
        # one row of logits: latency
        {"name": "sample_one", "kind": "sample", "B": 1, "V": 32000, "wide": False, "spread": 2.5},
        # a decode batch, each row with its own parameters
        {"name": "sample_64", "kind": "sample", "B": 64, "V": 131072, "wide": False, "spread": 2.5},
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(hi, max(lo, round(v / step) * step)))


def _heads(rng):
    Hkv = rng.choice([1, 2, 4, 8, 8, 8, 16, 32])
    return Hkv * rng.choice([g for g in (1, 2, 3, 4, 4, 5, 7, 8, 16) if g * Hkv <= 64]), Hkv


def draw(rng):
    kind = rng.choice(["block", "block", "axes", "axes", "chunk", "chunk", "chunk", "chunk", "sample", "sample"])
    if kind == "block":
        K = _log_int(rng, 512, 16384, 8)
        M = _log_int(rng, 1, min(8192, 8192 * 4096 // K))
        return {"kind": kind, "form": rng.choice(["quant", "quant", "bf16"]), "M": M, "K": K, "post": rng.random() < 0.75,
                "gates": rng.choice([0, 0, 1, min(M, 5), M]), "scale": rng.choice([1.0, 0.25, 0.7])}
    if kind == "sample":
        B = _log_int(rng, 1, 64)
        return {"kind": kind, "B": B, "V": _log_int(rng, 1000, 131072), "wide": rng.random() < 0.3, "spread": rng.uniform(1.0, 4.0)}
    Hq, Hkv = _heads(rng)
    page = rng.choice([16, 32, 48, 64, 128])
    if kind == "axes":
        return {"kind": kind, "T": _log_int(rng, 1, 6001 * 48 // max(48, Hq + 2 * Hkv)), "Hq": Hq, "Hkv": Hkv, "page": page,
                "axes": rng.choice([1, 2, 3, 3, 4]), "mixed": rng.random() < 0.3, "still": rng.choice([0, 0, 16, 32]), "interleaved": rng.random() < 0.3}
    shape = {"Hq": Hq, "Hkv": Hkv, "page": page, "ragged": rng.random() < 0.6, "cap": rng.choice([0.0, 30.0, 50.0]), "bias": rng.random() < 0.3,
             "window": rng.choice([0, 0, _log_int(rng, 16, 4096)]), "mask": rng.choice(["causal", "causal", "documents", "prefix"])}
    if rng.random() < 0.4:                                # one token, or a few, of each sequence
        B, new = _log_int(rng, 1, 64), rng.choice([1, 1, 2, 5])
        longest = _log_int(rng, new, max(64, min(40000, (32 * 6000 * 8) // (B * max(4, Hkv, new * Hq // 4)))))
    else:
        B = _log_int(rng, 1, 8)
        new = _log_int(rng, 6, 4096)
        longest = _log_int(rng, new, max(new, min(20000, 4096 * 8192 * 32 // (B * new * Hq))))
        new = max(6, min(new, 4096 * 8192 * 32 // (B * longest * Hq)))
    return dict({"kind": kind, "B": B, "new": new, "longest": longest}, **shape)


def _lengths(case):
    """(new tokens, cached tokens with them) of each sequence: by the case alone, so that work() knows them."""
    B, new, n = case["B"], case["new"], case["longest"]
    if not case["ragged"]:
        return [(new, n)] * B
    out = []
    for b in range(B):                                    # the first has them all, every eleventh none
        x = (b * 2654435761 >> 7)
        if b == 0:
            out.append((new, n))
        elif b % 11 == 10:
            out.append((1 if new == 1 else 0, 0))
        else:
            k = 1 + x % new
            out.append((k, k + (x >> 3) % (n - new + 1) if new > 1 else 1 + x % n))
    return out


def _ranges(case, b):
    """The tokens first <= t < end of each new row of sequence b, before the window: lists, by the case alone."""
    k, n = _lengths(case)[b]
    first, end = [], []
    step = max(8, n // 5)
    for i in range(k):
        pos = n - k + i
        if case["mask"] == "documents":                   # documents of different lengths, every 97th row is padding
            j = pos // step
            start = j * step + (0 if j == 0 else (j * 7919) % max(1, step // 3))
            if pos < start:
                j -= 1
                start = j * step + (0 if j == 0 else (j * 7919) % max(1, step // 3))
            pad = pos % 97 == 50
            first.append(pos if pad else start)
            end.append(pos if pad else pos + 1)
        elif case["mask"] == "prefix":                    # the first quarter is seen whole
            first.append(0)
            end.append(min(max(pos + 1, n // 4), max(n, 0)))
        else:
            first.append(0)
            end.append(min(pos + 1, max(n, 0)))
    if case["window"]:
        first = [max(f, n - k + i - case["window"] + 1) for i, f in enumerate(first)]
    return first, end


# ---- inputs ----

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7417 + 523)


def _acts(g, M, K, scale=1.0):
    """bf16 activations: N(0,1), 1 % of the columns x 20."""
    x = torch.randn((M, K), generator=g, device="cuda")
    x[:, torch.randperm(K, generator=g, device="cuda")[: max(1, K // 100)]] *= 20.0
    return (x * scale).to(torch.bfloat16)


def _cache(g, pages, heads, page):
    """A pool in use: codes as the quantiser leaves normal values (spread 2.7 steps, at most 7), scales around 0.37."""
    cache = torch.empty((pages, heads, page // 16, TILE), dtype=torch.uint8, device="cuda")
    for lo in range(0, pages, 1024):                      # (a slice at a time: the float draws are many times the cache)
        part = cache[lo:lo + 1024]
        q = torch.randn(part.shape[:3] + (2, 2048), generator=g, device="cuda").mul_(2.7).round_().clamp_(-7, 7).add_(8).to(torch.uint8)
        part[..., :2048] = q[..., 0, :] | (q[..., 1, :] << 4)
        s = torch.exp(0.2 * torch.randn(part.shape[:3] + (32,), generator=g, device="cuda")) * 0.37
        part[..., 2048:] = s.to(torch.float8_e4m3fn).view(torch.uint8)
    return cache


def _rotation(positions):
    """float32 [positions, 64, 2]: cosine and sine of position * 500000^(-2i/128)."""
    freq = 500000.0 ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack((a.cos(), a.sin()), dim=-1).to(torch.float32).contiguous()


def _axis_of(case):
    """The axis that each of the 64 pairs turns with: sections one after the other, or axes in turn; the last `still` pairs do not turn."""
    turning, A = 64 - case["still"], case["axes"]
    axes = [j % A for j in range(turning)] if case["mixed"] else [min(A - 1, (j * A + A // 2) // turning) for j in range(turning)]
    return axes + [-1] * case["still"]


def prepare(case, seed):
    g, kind, s = _gen(seed), case["kind"], {"case": case}
    if kind == "block":
        M, K = case["M"], case["K"]
        s["x"] = _acts(g, M, K)
        s["res"] = _acts(g, M, K, 16.0)
        s["w"] = (1.0 + 0.1 * torch.randn(K, generator=g, device="cuda")).to(torch.bfloat16)
        s["post"] = (1.0 + 0.1 * torch.randn(K, generator=g, device="cuda")).to(torch.bfloat16) if case["post"] else None
        n = case["gates"]
        s["gate"] = torch.tanh(torch.randn((n, K), generator=g, device="cuda")).to(torch.bfloat16) if n else None
        # (a gate for all rows, for each row, or for each sequence of a batch)
        s["rows"] = torch.sort(torch.randint(0, n, (M,), generator=g, device="cuda", dtype=torch.int32))[0] if n not in (0, 1, M) else None
        return s
    if kind == "sample":
        B, V = case["B"], case["V"]
        x = case["spread"] * torch.randn((B, V), generator=g, device="cuda")
        s["logits"] = x if case["wide"] else x.to(torch.bfloat16)
        r = torch.rand((4, B), generator=g, device="cuda")
        pick = lambda values, k: torch.tensor(values, device="cuda")[(r[k] * len(values)).long().clamp(max=len(values) - 1)]   # noqa: E731
        s["temperature"] = pick([0.8] if B == 1 else [0.6, 0.8, 1.0, 1.3, 0.0], 0)
        s["top_k"] = pick([50] if B == 1 else [0, 0, 20, 50, 1000], 1).to(torch.int32)
        s["top_p"] = pick([0.95] if B == 1 else [1.0, 0.9, 0.95], 2)
        s["min_p"] = pick([0.0] if B == 1 else [0.0, 0.0, 0.05], 3)
        s["u"] = torch.rand((B,), generator=g, device="cuda")
        return s
    page = case["page"]
    if kind == "axes":
        T, Hkv = case["T"], case["Hkv"]
        pages = 2 * (T // page) + 2
        s["cache"] = _cache(g, pages, Hkv, page)
        order = torch.randperm(pages, generator=g, device="cuda")[: -(-T // page)]
        s["slots"] = (order[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)[:T].contiguous()
        s["slots"][torch.rand(T, generator=g, device="cuda") < 0.02] = -1
        s["qkv"] = _acts(g, T, (case["Hq"] + 2 * Hkv) * D)
        s["rot"] = _rotation(32768)
        # text, then an image: all axes alike, then the last three by frame, row and column
        start = int(torch.randint(0, 20000, (1,), generator=g, device="cuda"))
        text = T // 5
        wide = math.isqrt(max(1, T - text - 1)) + 1
        i = torch.arange(T, device="cuda")
        j = (i - text).clamp(min=0)
        cols = [torch.where(i < text, start + i, start + text + v) for v in (torch.zeros_like(j), j // wide, j % wide, j % 7)]
        s["pos"] = torch.stack(cols[: case["axes"]]).to(torch.int32).contiguous()
        s["axis_of"] = _axis_of(case)
        return s
    lengths = _lengths(case)
    B = case["B"]
    width = max(1, max(-(-n // page) for _, n in lengths))
    s["cache"] = _cache(g, B * width, case["Hkv"], page)
    T = sum(k for k, _ in lengths)
    x = 2.0 * torch.randn((T, case["Hq"], D), generator=g, device="cuda")
    s["qs"] = x.abs().amax(-1) / 448.0
    s["q"] = (x / s["qs"][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    s["table"] = torch.randperm(B * width, generator=g, device="cuda").to(torch.int32).reshape(B, width).contiguous()
    starts = [0]
    for k, _ in lengths:
        starts.append(starts[-1] + k)
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["lens"] = torch.tensor([n for _, n in lengths], dtype=torch.int32, device="cuda")
    s["most"], s["most_new"] = max(n for _, n in lengths), max(k for k, _ in lengths)
    both = [_ranges(dict(case, window=0), b) for b in range(B)]
    flat = [torch.tensor([v for r in both for v in r[i]], dtype=torch.int32, device="cuda") for i in (0, 1)]
    s["first"] = flat[0] if case["mask"] == "documents" else None
    s["end"] = flat[1] if case["mask"] != "causal" else None
    # slopes 2^(-8 (h + 1) / heads), as biases by distance have them
    s["slopes"] = torch.exp2(-8.0 * torch.arange(1, case["Hq"] + 1, device="cuda", dtype=torch.float32) / case["Hq"]) if case["bias"] else None
    return s


# ---- the plain forms ----

def _over(x, n):
    """The quotients x / n: over a plain number torch multiplies by its reciprocal, and a quotient that is a border between two
    codes would fall beside it."""
    return x / torch.full_like(x, n)


def _quantise(y):
    """E4M3 codes and scales of float32 rows."""
    top = y.abs().amax(-1)
    s = torch.where(top > 0, _over(top, 448.0), torch.ones_like(top))
    return (y / s[..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), s


def _block(s):
    case = s["case"]
    p = s["x"].float()
    if s["post"] is not None:
        p = p * torch.rsqrt((p * p).mean(-1, keepdim=True) + EPS) * s["post"].float()
    if s["gate"] is not None:
        gate = s["gate"].float()
        p = p * (gate if s["rows"] is None else gate[s["rows"].long()])
    h = (s["res"].float() + case["scale"] * p).to(torch.bfloat16)
    f = h.float()
    y = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS) * s["w"].float()
    out = {"y": y.to(torch.bfloat16)} if case["form"] == "bf16" else dict(zip(("codes", "scale"), _quantise(y)))
    out["h"] = h
    return out


def _int4(x):
    """INT4 codes + 8 and E4M3 scales of float32 rows."""
    sigma = _over(x.abs().amax(-1), 7.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    f = sigma.float()[..., None]
    q = torch.where(f > 0, (x / f).round().clamp(-8, 7), torch.zeros_like(x))
    return (q + 8).to(torch.uint8), sigma.view(torch.uint8)


def _tokens(tiles):
    """float32 keys and values [..., 16, 128] of cache tiles [..., 2080]."""
    lead = tiles.shape[:-1]
    k = tiles[..., :1024].reshape(lead + (4, 16, 16))
    k = torch.stack((k & 15, k >> 4), dim=-2).movedim(-4, -3).reshape(lead + (16, D))
    v = tiles[..., 1024:2048].reshape(lead + (4, 16, 4, 4))[..., [0, 2, 1, 3]]
    v = torch.stack((v & 15, v >> 4), dim=-1)                                 # [quad, n, m, token, nibble]
    v = v.movedim(-2, -4).movedim(-3, -1).reshape(lead + (16, D))             # [quad, token, m, nibble, n]
    sc = tiles[..., 2048:].contiguous().view(torch.float8_e4m3fn).float().reshape(lead + (4, 2, 4))
    ks, vs = sc[..., 0, :].reshape(lead + (16, 1)), sc[..., 1, :].reshape(lead + (16, 1))
    return (k.float() - 8.0) * ks, (v.float() - 8.0) * vs


def _read(cache, slots):
    page = cache.shape[2] * 16
    at = slots.clamp(min=0)
    tiles = cache[at // page, :, at % page // 16]                              # [T, heads, 2080]
    k, v = _tokens(tiles)
    row = (at % 16)[:, None, None, None].expand(-1, k.shape[1], 1, D)
    there = (slots >= 0)[:, None, None]
    return {"k": (k.gather(2, row)[:, :, 0] * there).to(torch.bfloat16), "v": (v.gather(2, row)[:, :, 0] * there).to(torch.bfloat16)}


def _axes(s):
    case, cache, slots = s["case"], s["cache"], s["slots"]
    Hq, Hkv, page, T = case["Hq"], case["Hkv"], case["page"], case["T"]
    x = s["qkv"].reshape(T, Hq + 2 * Hkv, D)
    # in 64 bits: a rotated key next to the border between two codes has to fall on its own side of it
    axis = torch.tensor(s["axis_of"], device="cuda")
    pair = torch.arange(64, device="cuda")
    cs = s["rot"][s["pos"].long()[axis.clamp(min=0)].t(), pair].double()      # [T, 64, 2]
    c = torch.where(axis < 0, torch.ones_like(cs[..., 0]), cs[..., 0])[:, None]
    sn = torch.where(axis < 0, torch.zeros_like(cs[..., 1]), cs[..., 1])[:, None]
    h = x[:, : Hq + Hkv].double()
    if case["interleaved"]:
        a, b = h[..., 0::2], h[..., 1::2]
        r = torch.stack((a * c - b * sn, b * c + a * sn), dim=-1).reshape(h.shape).float()
    else:
        a, b = h[..., :64], h[..., 64:]
        r = torch.cat((a * c - b * sn, b * c + a * sn), dim=-1).float()
    codes, scale = _quantise(r[:, :Hq])
    kq, ks = _int4(r[:, Hq:])
    vq, vs = _int4(x[:, Hq + Hkv:].float())
    on = slots >= 0
    at, kq, ks, vq, vs = slots[on], kq[on], ks[on], vq[on], vs[on]
    pg, ti, t = at // page, at % page // 16, at % 16
    heads = torch.arange(Hkv, device="cuda")[None, :, None]
    pg, ti, t = pg[:, None, None], ti[:, None, None], t[:, None, None]
    e = torch.arange(64, device="cuda")
    kq = kq.reshape(-1, Hkv, 4, 2, 16)
    cache[pg, heads, ti, 256 * (e // 16) + 16 * t + e % 16] = (kq[..., 0, :] | (kq[..., 1, :] << 4)).reshape(-1, Hkv, 64)
    vq = vq.reshape(-1, Hkv, 4, 2, 16)                                        # [m, nibble, n]
    byte = torch.tensor([0, 2, 1, 3], device="cuda")[t % 4]
    cache[pg, heads, ti, 1024 + 256 * (t // 4) + 16 * (e % 16) + 4 * (e // 16) + byte] = (vq[..., 0, :] | (vq[..., 1, :] << 4)).reshape(-1, Hkv, 64)
    pg, ti, t, heads = pg[..., 0], ti[..., 0], t[..., 0], heads[..., 0]
    cache[pg, heads, ti, 2048 + 8 * (t // 4) + t % 4] = ks
    cache[pg, heads, ti, 2052 + 8 * (t // 4) + t % 4] = vs
    return dict(_read(cache, slots), codes=codes, scale=scale)


def _chunk(s):
    case = s["case"]
    Hq, Hkv, page = case["Hq"], case["Hkv"], case["page"]
    G, lo = Hq // Hkv, 0
    out = torch.empty((s["q"].shape[0], Hq, D), dtype=torch.bfloat16, device="cuda")
    for b, (k, n) in enumerate(_lengths(case)):
        if k == 0:
            continue
        row = slice(lo, lo + k)
        lo += k
        if n <= 0:
            out[row] = 0
            continue
        key, value = _tokens(s["cache"][s["table"][b, : -(-n // page)].long()].transpose(0, 1))
        key, value = key.reshape(Hkv, -1, D)[:, :n], value.reshape(Hkv, -1, D)[:, :n]
        t = torch.arange(n, device="cuda")
        for at in range(row.start, row.stop, 512):        # (a slice of rows at a time: the scores are many times the cache)
            part = slice(at, min(at + 512, row.stop))
            pos = torch.arange(part.start - row.start, part.stop - row.start, device="cuda") + (n - k)
            first = torch.zeros_like(pos) if s["first"] is None else s["first"][part].long()
            end = pos + 1 if s["end"] is None else s["end"][part].long()
            if case["window"]:
                first = torch.maximum(first, pos - case["window"] + 1)
            there = (t >= first[:, None]) & (t < end[:, None])                # [rows, tokens]
            q = s["q"][part].view(torch.float8_e4m3fn).float() * s["qs"][part][..., None] * SCALE
            q = q.reshape(-1, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, -1, D)
            x = torch.matmul(q, key.transpose(1, 2).contiguous()).reshape(Hkv, G, -1, n)
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if case["bias"]:
                x = x - s["slopes"].reshape(Hkv, G, 1, 1) * (pos[:, None] - t).abs().float()
            x = torch.where(there, x, -math.inf)
            top = x.amax(-1, keepdim=True)
            e = torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top)))
            norm = e.sum(-1, keepdim=True)
            o = torch.matmul(e.reshape(Hkv, -1, n), value).reshape(Hkv, G, -1, D)
            o = torch.where(norm > 0, o / norm, torch.zeros_like(o))          # a row without tokens: zeros
            out[part] = o.permute(2, 0, 1, 3).reshape(-1, Hq, D).to(torch.bfloat16)
    return out


def _sample(s):
    # in 64 bits: sums over the vocabulary, and borders between two tokens
    x = s["logits"].double()
    V = x.shape[1]
    greedy = (s["temperature"] == 0)[:, None]
    T = torch.where(greedy, torch.ones_like(s["temperature"][:, None]), s["temperature"][:, None]).double()
    top = x.amax(-1, keepdim=True)
    e = torch.exp((x - top) / T)
    order = torch.sort(x, dim=-1, descending=True, stable=True)[1]
    sorted_x, sorted_e = x.gather(1, order), e.gather(1, order)
    rank = torch.arange(V, device="cuda")
    k = torch.where(greedy, torch.ones_like(s["top_k"][:, None]), s["top_k"][:, None])
    keep = (k <= 0) | (rank < k)
    keep = keep & (sorted_x - top >= T * torch.log(s["min_p"].double())[:, None])
    mass = torch.where(keep, sorted_e, torch.zeros_like(sorted_e))
    before = mass.cumsum(-1) - mass
    p = s["top_p"].double()[:, None]
    keep = keep & ((p >= 1) | (rank == 0) | (before < p * mass.sum(-1, keepdim=True)))
    kept = torch.zeros_like(e).scatter(1, order, torch.where(keep, sorted_e, torch.zeros_like(sorted_e)))
    run = kept.cumsum(-1)
    token = (run <= s["u"].double()[:, None] * run[:, -1:]).sum(-1)
    token = token.clamp(max=V - 1)
    logp = (x.gather(1, token[:, None]) - top) / T - torch.log(e.sum(-1, keepdim=True))
    return {"token": token.to(torch.int32), "logprob": logp[:, 0].float()}


# ---- one pass ----

def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if own:
        from paper_2505_20839_amd import binding as fq
        if kind == "block":
            call = fq.fq_rmsnorm_block if case["form"] == "bf16" else fq.fq_rmsnorm_block_quant
            r = call(s["x"], s["w"], EPS, s["res"], post=s["post"], gate=s["gate"], gate_rows=s["rows"], scale=case["scale"])
            if case["form"] == "bf16":
                return {"y": r[0], "h": r[1]}
            return {"codes": r[0].view(torch.float8_e4m3fn), "scale": r[1], "h": r[2]}
        if kind == "axes":
            codes, scale = fq.fq_kv4_append_axes(s["qkv"], s["rot"], s["pos"], s["axis_of"], s["slots"], s["cache"], interleaved=case["interleaved"])
            k, v = fq.fq_kv4_read(s["cache"], s["slots"])
            return {"k": k, "v": v, "codes": codes.view(torch.float8_e4m3fn), "scale": scale}
        if kind == "chunk":
            return fq.fq_kv4_attention_chunk(s["q"], s["qs"], s["cache"], s["table"], s["starts"], s["lens"], SCALE, max_new=s["most_new"],
                                             max_len=s["most"], first=s["first"], end=s["end"], window=case["window"], cap=case["cap"],
                                             slopes=s["slopes"])
        token, logprob = fq.fq_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return {"token": token, "logprob": logprob}
    if kind == "block":
        return _block(s)
    if kind == "axes":
        return _axes(s)
    if kind == "chunk":
        return _chunk(s)
    return _sample(s)


def work(case):
    kind = case["kind"]
    if kind == "block":
        M, K = case["M"], case["K"]
        per = 6 + (1 if case["form"] == "quant" else 2)
        extra = 2 * K * (1 + (1 if case["post"] else 0) + case["gates"]) + (4 * M if case["form"] == "quant" else 0)
        return {"bytes": per * M * K + extra, "flops": 12 * M * K}
    if kind == "axes":                                    # the append, and the same tokens read back
        T, Hq, Hkv = case["T"], case["Hq"], case["Hkv"]
        rot = 512 * min(T, 32768)
        return {"bytes": T * (256 * (Hq + 2 * Hkv) + 132 * Hq + 130 * Hkv + 8 + 4 * case["axes"]) + rot + T * (642 * Hkv + 8), "flops": T * D * (8 * Hq + 14 * Hkv)}
    if kind == "sample":
        B, V = case["B"], case["V"]
        return {"bytes": B * V * (4 if case["wide"] else 2) + 28 * B, "flops": 4 * B * V}
    Hq, Hkv, tokens, pairs, rows, pages = case["Hq"], case["Hkv"], 0, 0, 0, 0
    for b, (k, n) in enumerate(_lengths(case)):
        first, end = _ranges(case, b)
        some = [(f, e) for f, e in zip(first, end) if f < e]
        rows += k
        pairs += sum(e - f for f, e in some)
        if some:
            lo, hi = min(f for f, _ in some), max(e for _, e in some)
            tokens += hi - max(lo, 0)
            pages += -(-hi // case["page"]) - max(lo, 0) // case["page"]
    return {"bytes": 130 * Hkv * tokens + 4 * pages + 8 * case["B"] + rows * Hq * (D + 4 + 2 * D), "flops": 4 * D * Hq * pairs}


# ---- the definition in 64 bits ----

def _exact_codes(y):
    """Values of the E4M3 codes and the scales of rows of 64-bit numbers."""
    s = _over(y.abs().amax(-1), 448.0)
    s[s == 0] = 1.0
    q = y / s[..., None]
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))).clamp(max=8) - 3)
    return (torch.round(q / step) * step).clamp(-448, 448), s


def _exact_int4(x):
    """Rows of 64-bit numbers as the INT4 codes and E4M3 scales stand for them."""
    s = _over(x.abs().amax(-1, keepdim=True), 7.0)
    step = torch.exp2(torch.floor(torch.log2(s.clamp(2.0 ** -6, 448))) - 3)
    s = (torch.round(s / step) * step).clamp(max=448)
    return torch.where(s > 0, torch.round(x / s.clamp(min=2.0 ** -9)).clamp(-8, 7) * s, torch.zeros_like(x))


def _exact_cached(cache, page_of, within):
    """64-bit keys and values [tokens, heads, D] of tokens `within` (0 .. page - 1) pages `page_of`, byte by byte."""
    flat = cache.reshape(cache.shape[0], cache.shape[1], -1)[page_of]         # [tokens, heads, bytes of a page]
    d = torch.arange(D, device="cuda")
    tile, t = within // 16 * TILE, within % 16

    def nibbles(at, high):
        b = flat.gather(2, at[:, None].expand(-1, flat.shape[1], -1)).long()
        return (torch.where(high, b // 16, b % 16) - 8).double()

    high = d // 16 % 2 == 1
    k = nibbles((tile + 16 * t)[:, None] + 256 * (d // 32) + d % 16, high)
    place = torch.tensor([0, 2, 1, 3], device="cuda")[t % 4]
    v = nibbles((tile + 1024 + 256 * (t // 4) + place)[:, None] + 16 * (d % 16) + 4 * (d // 32), high)

    def scale(at):
        c = flat.gather(2, at[:, None, None].expand(-1, flat.shape[1], 1)).long()
        e, m = c % 128 // 8, (c % 8).double()
        x = torch.where(e > 0, (8 + m) * torch.exp2(e.double() - 10), m * 2.0 ** -9)
        return torch.where(c > 127, -x, x)

    at = tile + 2048 + 8 * (t // 4) + t % 4
    return k * scale(at), v * scale(at + 4)


def _exact_block(s, case):
    x = s["x"].double()
    if s["post"] is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["K"] + EPS) * s["post"].double()
    if s["gate"] is not None:
        rows = s["rows"] if s["rows"] is not None else torch.arange(case["M"], device="cuda") % s["gate"].shape[0]
        x = x * s["gate"].double()[rows.long()]
    h = s["res"].double() + case["scale"] * x
    r = h.to(torch.bfloat16).double()                     # the definition rounds the stream
    y = r / torch.sqrt(r.square().sum(-1, keepdim=True) / case["K"] + EPS) * s["w"].double()
    if case["form"] == "bf16":
        return {"y": y, "h": h}
    codes, scale = _exact_codes(y)
    return {"codes": codes, "scale": scale, "h": h}


def _exact_sample(s, case):
    tokens, logs = [], []
    for b in range(case["B"]):
        x = s["logits"][b].double()
        T, k, p, low = (s[n][b].item() for n in ("temperature", "top_k", "top_p", "min_p"))
        if T == 0:
            T, k = 1.0, 1
        logp = torch.log_softmax(x / T, dim=-1)
        live = torch.nonzero(x >= x.max() + T * math.log(low))[:, 0] if low > 0 else torch.arange(case["V"], device="cuda")
        # best first, equals by index: sorted by index already, so one stable pass over the negated values
        live = live[torch.sort(-x[live], stable=True)[1]]
        if k > 0:
            live = live[:k]
        mass = torch.exp(logp[live])
        if p < 1:
            reached = torch.nonzero(torch.cumsum(mass, 0) >= p * mass.sum())
            live = live[: int(reached[0]) + 1] if len(reached) else live
        live = live.sort()[0]
        mass = torch.cumsum(torch.exp(logp[live]), 0)
        at = torch.nonzero(mass > s["u"][b].double() * mass[-1])
        token = int(live[int(at[0])] if len(at) else live[-1])
        tokens.append(token)
        logs.append(logp[token])
    return {"token": torch.tensor(tokens, dtype=torch.int32, device="cuda"), "logprob": torch.stack(logs)}


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "block":
        return _exact_block(s, case)
    if kind == "sample":
        return _exact_sample(s, case)
    if kind == "axes":
        on, Hq, Hkv = s["slots"] >= 0, case["Hq"], case["Hkv"]
        x = s["qkv"].double().reshape(case["T"], Hq + 2 * Hkv, D)
        table = torch.view_as_complex(s["rot"].double())
        z = torch.stack([table[s["pos"][a].long(), j] if a >= 0 else torch.ones_like(table[s["pos"][0].long(), j]) for j, a in enumerate(s["axis_of"])], dim=-1)[:, None]
        qk = x[:, : Hq + Hkv]
        if case["interleaved"]:
            r = torch.view_as_real(torch.view_as_complex(qk.reshape(qk.shape[:2] + (64, 2)).contiguous()) * z).reshape(qk.shape)
        else:
            r = torch.complex(qk[..., :64].contiguous(), qk[..., 64:].contiguous()) * z
            r = torch.cat((r.real, r.imag), dim=-1)
        r = r.float().double()                            # the definition rounds the rotated heads to 32 bits
        codes, scale = _exact_codes(r[:, :Hq])
        return {"k": _exact_int4(r[:, Hq:]) * on[:, None, None], "v": _exact_int4(x[:, Hq + Hkv:]) * on[:, None, None], "codes": codes, "scale": scale}
    Hq, Hkv, page = case["Hq"], case["Hkv"], case["page"]
    q = s["q"].view(torch.float8_e4m3fn).double() * s["qs"].double()[..., None]
    out = torch.zeros((q.shape[0], Hq, D), dtype=torch.float64, device="cuda")
    lo = 0
    for b, (k, n) in enumerate(_lengths(case)):
        if k == 0 or n <= 0:
            lo += k
            continue
        t = torch.arange(n, device="cuda")
        got = [_exact_cached(s["cache"], s["table"][b].long()[t[i:i + 2048] // page], t[i:i + 2048] % page) for i in range(0, n, 2048)]
        key, value = (torch.cat([x[i] for x in got]) for i in (0, 1))
        first, end = (torch.tensor(r, device="cuda")[:, None] for r in _ranges(case, b))
        for h in range(Hq):                               # head by head, some rows at a time
            kh, vh = key[:, h * Hkv // Hq].t().contiguous(), value[:, h * Hkv // Hq].contiguous()
            for i in range(0, k, 2048):
                x = torch.matmul(q[lo + i:lo + min(i + 2048, k), h], kh) * SCALE
                if case["cap"]:
                    x = torch.tanh(x / case["cap"]) * case["cap"]
                if case["bias"]:
                    x -= 2.0 ** (-8.0 * (h + 1) / Hq) * (t - torch.arange(n - k + i, n - k + i + x.shape[0], device="cuda")[:, None]).abs()
                x = x.masked_fill((t < first[i:i + 2048]) | (t >= end[i:i + 2048]), -math.inf)
                out[lo + i:lo + i + x.shape[0], h] = torch.matmul(torch.nan_to_num(torch.softmax(x, dim=-1), nan=0.0), vh)
        lo += k
    return out
