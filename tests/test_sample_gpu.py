"""kl_sample against the definition in 64 bits, row after row in numpy: tokens are compared exactly.

Weights differ from the library's by roundings of 64 bits alone: the exponent, at most 80 in magnitude, by 2^-53 of itself, hence a
weight by 2^-46.  The library adds at most 80 positive numbers in a row and joins such sums in trees, under 128 additions from any
weight to the end: 2^-46 more; the oracle adds in 80 bits.  Two such sums compare alike on both sides where they are further apart than
2 * (2^-46 + 2^-46) < 2^-43, which the oracle checks of every comparison, except where the sums are whole numbers and ties are exact."""
import math

import numpy as np
import pytest
import torch

from paper_2410_23668_b200 import binding as kl

pytestmark = pytest.mark.gpu


def one_row(x, u, t=1.0, k=0, p=1.0, q=0.0):
    """(token, logprob, distance of the nearest comparison from a tie, relative)."""
    x = np.where(np.isnan(x), -np.inf, x).astype(np.float64)
    f = np.float32
    t, p, q, u = (float(f(v)) for v in (t, p, q, u))
    m = x.max()
    if m == -np.inf:
        return -1, -math.inf, 1.0
    order = np.lexsort((np.arange(len(x)), -x))
    if not t > 0 or k == 1 or p <= 0 or q > 1:
        return int(order[0]), 0.0, 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.where(x == m, 0.0, np.where(x == -np.inf, -np.inf, (x - m) / t))
    w = np.exp(y).astype(np.longdouble)
    order = order[x[order] > -np.inf]
    if k > 0:
        order = order[:k]
    near = 1.0
    if p < 1:
        mass = np.cumsum(w[order])
        before = mass - w[order]
        near = min(near, np.min(np.abs(before / (p * mass[-1]) - 1)))
        order = order[(before < p * mass[-1]) | (np.arange(len(order)) == 0)]
    if q > 0:
        near = min(near, np.min(np.abs(w[order] / q - 1)))
        order = order[(w[order] >= q) | (np.arange(len(order)) == 0)]
    stay = np.sort(order)
    mass = np.cumsum(w[stay])
    goal = min(max(u, 0.0), 1.0) * mass[-1]
    near = min(near, np.min(np.abs(mass[:-1] / goal - 1)) if len(stay) > 1 and goal > 0 else 1.0)
    over = np.nonzero(mass > goal)[0]
    at = over[0] if len(over) else np.nonzero(w[stay] > 0)[0][-1]
    while w[stay[at]] == 0:
        at += 1
    return int(stay[at]), float(np.log(w[stay[at]] / mass[-1])), near


def run(x, u, t=None, k=None, p=None, q=None, ties=False, stride=0):
    n, vocab = x.shape
    dev = torch.full((n, vocab + stride), math.nan)
    dev[:, :vocab] = torch.from_numpy(x)
    dev = dev.cuda()[:, :vocab]
    f = lambda v, d=torch.float32: None if v is None else torch.tensor(np.broadcast_to(np.asarray(v), (n,)).copy(), dtype=d).cuda()  # noqa: E731
    tokens = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    logprobs = torch.full((n,), 7.0, device="cuda")
    kl.kl_sample(dev, f(u), tokens, temperature=f(t), top_k=f(k, torch.int32), top_p=f(p), min_p=f(q), logprobs=logprobs)
    tokens, logprobs = tokens.cpu().numpy(), logprobs.cpu().numpy()
    at = lambda v, i, off: off if v is None else np.broadcast_to(np.asarray(v), (n,))[i]  # noqa: E731
    for i in range(n):
        want, lp, near = one_row(x[i], at(u, i, 0), at(t, i, 1.0), int(at(k, i, 0)), at(p, i, 1.0), at(q, i, 0.0))
        assert ties or near > 2.0 ** -43, f"row {i}: the case is a tie ({near})"
        assert tokens[i] == want, (i, tokens[i], want)
        # the logarithm of a ratio of 64-bit sums, rounded to 32 bits: half a step of 2^-24, and 2^-35 from the sums
        assert logprobs[i] == lp or abs(logprobs[i] - lp) <= 2.0 ** -23 * abs(lp) + 2.0 ** -34, (i, logprobs[i], lp)
    return tokens


def logits(n, vocab, seed, loud=2.5):
    r = np.random.default_rng(seed)
    return (r.standard_normal((n, vocab)) * loud).astype(np.float32), r


@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 1000, 1024, 16384, 16385, 32000, 50257, 128256, 151936, 262144, 327680])
def test_temperature_alone(vocab):
    x, r = logits(5, vocab, vocab)
    run(x, r.random(5), t=[0.7, 1.0, 1.3, 0.1, 3.0])


@pytest.mark.parametrize("vocab", [7, 1000, 32000, 128256])
@pytest.mark.parametrize("k", [1, 2, 5, 50, 999, 2047, 2048, 2049, 20000])
def test_top_k(vocab, k):
    x, r = logits(3, vocab, vocab + k)
    run(x, r.random(3), t=[0.8, 1.0, 2.0], k=k)
    run(x, r.random(3), k=[k, 0, vocab], p=0.9)


@pytest.mark.parametrize("vocab", [3, 1000, 32000, 128256])
@pytest.mark.parametrize("p", [1e-6, 0.1, 0.5, 0.9, 0.99, 0.9999, 0.9999999])
def test_top_p(vocab, p):
    x, r = logits(4, vocab, vocab, loud=1.0)
    x[1] *= 3
    x[2] *= 0.01
    run(x, r.random(4), p=p)
    run(x, r.random(4), p=p, k=vocab // 2, q=1e-3)


@pytest.mark.parametrize("q", [1e-8, 0.02, 0.3, 0.999, 1.5])
def test_min_p(q):
    x, r = logits(4, 32000, 3)
    run(x, r.random(4), q=q, t=[0.5, 1.0, 1.5, 2.0])
    run(x, r.random(4), q=q, k=40, p=0.8)


def test_settings_of_every_row_its_own():
    n = 200
    x, r = logits(n, 5000, 17)
    run(x, r.random(n), t=r.uniform(0.2, 2, n), k=r.integers(0, 300, n), p=r.uniform(0.2, 1.2, n), q=r.uniform(-0.1, 0.2, n), stride=3)


@pytest.mark.parametrize("vocab", [4096, 131072])
def test_equal_logits_are_taken_lower_token_first(vocab):
    x = np.zeros((6, vocab), np.float32)
    x[1, ::2] = -0.0
    x[2, 1000:] = -1
    u = np.array([0.0, 0.25, 0.5, 0.75, 0.999, 0.125])
    # sums of equal weights are whole numbers (times one weight): exact in any order
    run(x[:2], u[:2], k=[3, vocab // 2], ties=True)
    run(x[:2], u[2:4], p=0.5, ties=True)
    run(x[:2], u[2:4], p=0.25, k=vocab // 2, ties=True)
    run(x[2:3], u[4:5], p=0.75)
    run(x[2:3], u[4:5], k=vocab - 500)


def test_far_apart_and_forbidden():
    r = np.random.default_rng(5)
    x = np.full((9, 20000), -np.inf, np.float32)
    x[0, 123] = -3.0                                       # one token alone
    x[1] = np.finfo(np.float32).min                        # the type's lowest value everywhere
    x[2] = np.finfo(np.float32).min
    x[2, 77] = 1.0                                         # and one above it
    x[3, 5], x[3, 6], x[3, 19999] = np.inf, 3.0, np.inf    # infinite ones share the chances
    x[4] = np.nan
    x[4, 9], x[4, 11] = 1.0, 1.5                           # NaN is not allowed
    x[5] = np.nan                                          # nothing is
    # row 6: nothing is
    x[7] = r.standard_normal(20000) * 1e30                 # differences that overflow the temperature
    x[8, :100] = 60 * r.random(100)
    u = r.random(9)
    for kw in (dict(), dict(k=40), dict(p=0.9), dict(k=40, p=0.9, q=0.01), dict(k=3000), dict(t=1e-30), dict(t=1e30, p=0.7), dict(t=0.0), dict(t=-1.0), dict(t=math.nan),
               dict(p=0.0), dict(p=-1.0), dict(p=math.nan), dict(q=math.nan), dict(k=-3)):
        run(x, u, ties=True, **kw)


def test_random_numbers_at_the_ends():
    x, _ = logits(6, 1000, 9)
    run(x, [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, 0.5], ties=True)
    run(x, [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, 0.5], k=20, ties=True)
    x[:, 0] = x[:, -1] = -np.inf   # the first and the last token that are allowed
    run(x, [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, 0.5], ties=True)


def test_positions_empty_slots_and_a_captured_call():
    x, r = logits(4, 3000, 21)
    dev, u = torch.from_numpy(x).cuda(), torch.from_numpy(r.random(4).astype(np.float32)).cuda()
    dev[3] = -math.inf
    tokens = torch.full((4,), -7, dtype=torch.int32, device="cuda")
    logprobs = torch.full((4,), 9.0, device="cuda")
    positions = torch.tensor([5, -1, 0, 8], dtype=torch.int32, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        kl.kl_sample(dev, u, tokens, logprobs=logprobs, positions=positions, stream=st)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            kl.kl_sample(dev, u, tokens, logprobs=logprobs, positions=positions, stream=torch.cuda.current_stream())
        first = tokens.clone()
        u.copy_(1 - u)
        graph.replay()
    torch.cuda.synchronize()
    assert positions.tolist() == [7, -1, 2, 8]
    assert first[1] == -7 and tokens[1] == -7 and logprobs[1] == 9.0 and tokens[3] == -1 and logprobs[3] == -math.inf
    for i in (0, 2):
        assert first[i] == one_row(x[i], float(1 - u[i]))[0] and tokens[i] == one_row(x[i], float(u[i]))[0]


def test_chances_follow_the_distribution():
    """Uniforms on a grid: every token is drawn as often as its probability says, give or take one at each end of its run."""
    n = 4096
    x = np.tile(np.random.default_rng(2).standard_normal(50).astype(np.float32), (n, 1))
    tokens = run(x, (np.arange(n) + 0.5) / n, ties=True)
    w = np.exp(x[0].astype(np.float64))
    assert np.all(np.abs(np.bincount(tokens, minlength=50) - n * w / w.sum()) <= 1.0)
