"""Sampling (fireq_sample.h) where a border, a sum or an exponential ends: tokens that the definition fixes without a tolerance."""
import math
import random
from fractions import Fraction

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU: torch.cuda.is_available() is False")
    from paper_2505_20839_amd import binding
    return binding


def draw(fq, x, u, **filters):
    """Tokens and log-probabilities by the C call, into outputs that hold a token that no row has; filters: a number for all rows."""
    B, V = x.shape
    t = {n: torch.full((B,), v, dtype=torch.int32 if n == "k" else torch.float32, device="cuda") for n, v in filters.items()}
    uu = torch.tensor(u, dtype=torch.float32, device="cuda")
    token, logprob = torch.full((B,), -7, dtype=torch.int32, device="cuda"), torch.full((B,), 7.0, device="cuda")
    need = fq.fq_sample_workspace_bytes(B, V)
    ws = torch.full((max(need, 16),), 0xA5, dtype=torch.uint8, device="cuda")
    call = fq.lib().fq_sample_bf16_ws if x.dtype == torch.bfloat16 else fq.lib().fq_sample_fp32_ws
    p = lambda n: t[n].data_ptr() if n in t else 0        # noqa: E731
    rc = call(x.data_ptr(), x.stride(0), uu.data_ptr(), p("T"), p("k"), p("p"), p("m"), token.data_ptr(), logprob.data_ptr(), B, V, ws.data_ptr() if need else 0, need,
              torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    torch.cuda.synchronize()
    return token.tolist(), logprob.tolist()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [30000, 40000, 131072])
@pytest.mark.parametrize("T", [1.0, 0.25])
def test_min_p_beyond_the_masses(fq, dtype, V, T):
    """min-p's border lies where a token has no mass of its own, but thousands of them have one together: those below it are not drawn all the same, and the
    first token by index that is kept is, also with u = 0."""
    x = torch.full((4, V), -28.0 * T, dtype=dtype, device="cuda")     # e^-28; the border is at log 1e-12 = -27.6
    x[:, -1] = 0.0
    x[2, V // 2:] = -29.0 * T
    x[3, V // 3] = -1.0 * T
    token, logprob = draw(fq, x, [0.0, 1e-9, 0.0, 0.0], T=T, m=1e-12)
    assert token == [V - 1, V - 1, 0, V // 3]             # (the best of the third row is at -28 T: all its tokens are kept)
    for b in range(4):
        want = torch.log_softmax(x[b].double() / T, -1)[token[b]].item()
        assert abs(logprob[b] - want) <= 2.0 ** -23 * abs(want) + 2.0 ** -16 + V * 2.0 ** -33      # (FP32 exponentials; 2^-33 a token)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [3, 1000, 40000])
def test_shares_that_add_up_to_one(fq, dtype, V):
    """The best token and two of half its mass, or four of a quarter: the best alone has half of all."""
    x = torch.full((2, V), -math.inf, dtype=dtype, device="cuda")
    x[:, 0] = 0.0
    x[0, -2:] = -1.0
    x[1, -min(V - 1, 4):] = -2.0
    T = 1.4426950216293335                                # log2 e in FP32, a little less: e^(-1/T) is 2^-1 (1 - 10^-8)
    for k in (0, min(V, 30)):
        token, _ = draw(fq, x, [0.9999, 0.9999], T=T, p=0.5, k=k)
        assert token == [0, 0]
        token, _ = draw(fq, x, [0.9999, 0.9999], T=T, p=0.6, k=k)
        assert token[0] == V - 2                           # (three fifths need one more, the first by index)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [4, 8, 1000, 8192, 32760, 40000, 131072])
@pytest.mark.parametrize("k", [0, -1])
def test_top_p_of_equal_logits(fq, dtype, V, k):
    """All alike: the first half of the tokens has half of the mass, and a quarter a quarter, in whole numbers."""
    x = torch.full((3, V), 1.5, dtype=dtype, device="cuda")
    for p, kept in ((0.5, V // 2), (0.25, V // 4), (0.75, 3 * V // 4)):
        token, _ = draw(fq, x, [0.0, 0.5, 1 - 2.0 ** -24], p=p, k=k)
        assert token == [0, kept // 2, kept - 1]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [20000, 32000, 32761, 40000])
@pytest.mark.parametrize("p", [0.9995, 0.9999, 0.99999])
def test_top_p_of_many_small_masses(fq, dtype, V, p):
    """One token and thousands of 2^-25 of its mass: what top-p leaves out is counted in these, and none is lost beside the large one."""
    x = torch.full((1, V), -25.0, dtype=dtype, device="cuda")
    x[:, 0] = 0.0
    p = torch.tensor(p, dtype=torch.float32).item()
    kept = math.ceil((p * (1 + (V - 1) * 2.0 ** -25) - 1) * 2 ** 25)     # of the small ones, the first by index
    token, _ = draw(fq, x, [1 - 2.0 ** -24], T=1.4426950216293335, p=p)
    assert kept - 3 <= token[0] <= kept                    # (u leaves out two of them, and a small mass is 128 - 2^-17 of the units)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1000, 30000])
@pytest.mark.parametrize("T", [1.0, 1e8, 1e30])
def test_top_k_of_logits_next_to_zero(fq, dtype, V, T):
    """Logits whose steps of x / T underflow: 0, then the others, of which the first by index is kept beside it."""
    x = torch.full((3, V), -2.0 ** -133, dtype=dtype, device="cuda")
    x[:, V // 2] = 0.0
    x[2] *= 2.0
    x[2, 7] = -2.0 ** -133
    token, logprob = draw(fq, x, [0.2, 0.8, 0.2], T=T, k=2)
    assert token == [0, V // 2, 7]
    assert all(abs(v + math.log(V)) < 1e-4 for v in logprob)


@pytest.mark.parametrize("V", [3000, 40000])
def test_temperatures_past_their_range(fq, V):
    """A temperature outside 2^-100 .. 2^100 counts as the nearest of these."""
    x = torch.zeros((2, V), device="cuda")
    x[0, 1::2], x[1, 1::2] = -1.5 * 2.0 ** 100, -1.5 * 2.0 ** -100
    for T, same in ((3e38, 2.0 ** 100), (2.0 ** 101, 2.0 ** 100), (1e-38, 2.0 ** -100), (2.0 ** -149, 2.0 ** -100)):
        for u in (0.1, 0.93):
            assert draw(fq, x, [u, u], T=T) == draw(fq, x, [u, u], T=same)


def expected(x, u, k, p, m):
    """The definition in whole numbers, for whole logits at T = log2 e that lie up to 8 below the best: masses are 2^32 - 2^8 shifted right."""
    top = max(x)
    keep = sorted(range(len(x)), key=lambda i: (-x[i], i))
    if m > 0:
        keep = [i for i in keep if x[i] >= top + 1.4426950216293335 * math.log(m)]
    keep = keep[:k] if 0 < k < len(x) else keep
    mass = lambda i: (2 ** 32 - 2 ** 8) >> (top - x[i])   # noqa: E731
    if p < 1:
        want, n = Fraction(p) * sum(map(mass, keep)), 0
        while n == 0 or sum(map(mass, keep[:n])) < want:
            n += 1
        keep = keep[:n]
    want, c = Fraction(u) * sum(map(mass, keep)), 0
    for i in sorted(keep):
        c += mass(i)
        if c > want:
            return i


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1, 5, 64, 300, 2500, 40000])
def test_tokens_of_exact_masses(fq, dtype, V):
    """Ties everywhere, borders of every filter on them: the very token of the definition."""
    rng = random.Random(V)
    f32 = lambda v: torch.tensor(v, dtype=torch.float32).item()     # noqa: E731
    for depth in (0, 1, 2, 8):
        # (long rows: a few tokens at the depths, the others have no mass)
        some = rng.sample(range(V), min(V, 300))
        x = torch.full((1, V), -math.inf)
        x[0, some] = torch.tensor([float(-rng.randint(0, depth)) for _ in some])
        x = x.to(dtype).cuda()
        places = sorted(some)
        y = [int(v) for v in x[0, places].tolist()]
        for _ in range(12):
            k, p, m = rng.choice([0, 1, 2, 7, 50, len(y) - 1]), f32(rng.choice([1.0, 0.5, 0.25, 0.0, 0.9, rng.random()])), f32(rng.choice([0.0, 0.0, 0.3, 0.1, 0.01]))
            u = f32(rng.choice([0.0, 0.5, 1 - 2.0 ** -24, rng.random()]))
            token, _ = draw(fq, x, [u], T=1.4426950216293335, k=k, p=p, m=m)
            assert token[0] == places[expected(y, u, k if k < len(y) else 0, p, m)], (depth, k, p, m, u)
