"""The operators for drafted tokens on a paged cache against plain 64-bit restatements, through the C ABI.

Rotated keys are rounded once from 64 bits on both sides and compared exactly: sines, cosines and products differ by a few 2^-53
of |a| + |b|, and a seeded key lies that near a border between two codes with a chance of some 10^-12.  Queries turn in 32 bits:
cosine and sine rounded (2^-24 each), a product rounded and the sum rounded, 4 * 2^-24 of |a| + |b| in all, and half a step of bf16 (2^-8)
where the output is that."""
import math

import numpy as np
import pytest
import torch

from paper_2410_23668_b200 import binding as kl, build
from tests import paged_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build_library()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def freqs(hd, theta=10000.0):
    return torch.tensor(theta ** (-2.0 * np.arange(hd // 2) / hd), dtype=torch.float64)


def turned(x, position, f):
    """x [heads, hd] in 64 bits, turned."""
    a, b = x.double().chunk(2, -1)
    angle = torch.from_numpy(position * f.numpy())
    c, s = torch.from_numpy(np.cos(angle.numpy())), torch.from_numpy(np.sin(angle.numpy()))
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def starts_of(seqs):
    return [sum(r for _, r in seqs[:i]) for i in range(len(seqs) + 1)]


# ---- append with rotation

ROTATIONS = [
    # e4m3, rows, hd, nkv, nq, page, [(first position, rows)], pages in [page][row][head] order
    (False, torch.bfloat16, 128, 8, 32, 16, [(0, 1)], False),
    (True, torch.bfloat16, 128, 8, 32, 16, [(4095, 1)], False),
    (True, torch.float32, 128, 2, 6, 4, [(3, 1), (-1, 0), (7, 9), (0, 4)], False),
    (False, torch.float32, 64, 3, 3, 24, [(23, 50), (0, 0), (5, 1), (48, 25)], True),
    (True, torch.bfloat16, 64, 1, 12, 64, [(63, 130), (10, 3)], False),
    (True, torch.bfloat16, 256, 4, 4, 8, [(0, 8), (8, 8), (17, 1)], True),
    (False, torch.bfloat16, 256, 2, 16, 1024, [(1000, 40), (0, 3)], False),
    (True, torch.float32, 128, 8, 64, 16, [(15, 33), (0, 100), (-1, 5), (31, 2)], False),
    (True, torch.bfloat16, 128, 11, 11, 32, [(131000, 40), (7, 17)], False),
]


@pytest.mark.parametrize("e4m3,dtype,hd,nkv,nq,page,seqs,rows_first", ROTATIONS)
@pytest.mark.parametrize("form", ["plain", "bounds", "positions", "in place"])
def test_append_rotated(e4m3, dtype, hd, nkv, nq, page, seqs, rows_first, form):
    lengths = [max(p, 0) % 1024 + r for p, r in seqs]   # far positions lie in the pages that a shorter sequence would fill
    far = [p - p % 1024 if p >= 1024 and form == "positions" else 0 for p, _ in seqs]
    seqs = [(p % 1024 if p >= 1024 else p, r) for p, r in seqs]
    n_pages = sum(-(-x // page) for x in lengths) + 3
    bounds = form != "plain"
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, bounds, rows_first, seed=1)
    table = ref.scattered_table(lengths, page, n_pages, seed=2)
    starts = starts_of(seqs)
    n = starts[-1] + 5   # rows behind the last sequence
    g = torch.Generator().manual_seed(3)
    fused = (torch.randn(n, nq + 2 * nkv, hd, generator=g) * torch.exp(torch.randn(n, nq + 2 * nkv, 1, generator=g))).to(dtype).cuda()
    k, q, v = fused[:, :nkv], fused[:, nkv:nkv + nq], fused[:, nkv + nq:]
    q0 = q.cpu().clone()
    f = freqs(hd)
    at = torch.zeros(n, dtype=torch.int64)
    for s, (p0, r) in enumerate(seqs):
        for i in range(r):
            at[starts[s] + i] = far[s] + p0 + (i if form != "positions" else (i * 7) % 5 - 2)
    q_out = torch.full((n, nq, hd), 5.0, dtype=dtype, device="cuda") if form in ("bounds", "positions") else None if form == "plain" else q
    before = {x: getattr(c, x).cpu().clone() for x in ("k", "v", "ke", "ve", "bounds") if getattr(c, x) is not None}
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kl.kl_paged_append_rotated(c.handle, k, v, i32([p for p, _ in seqs]), table.cuda(), f.cuda(), row_starts=i32(starts),
                               row_positions=at.to(torch.int32).cuda() if form == "positions" else None, q=q if q_out is not None else None, q_out=q_out, status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    want = {x: t.clone() for x, t in before.items()}
    live = set()
    for s, (p0, cnt) in enumerate(seqs):
        for i in range(cnt if p0 >= 0 else 0):
            live.add(starts[s] + i)
            phys, off = int(table[s, (p0 + i) // page]), (p0 + i) % page
            for which, rows in (("k", k), ("v", v)):
                x = rows[starts[s] + i].cpu().double()
                if which == "k":
                    x = turned(x, int(at[starts[s] + i]), f)
                for h in range(nkv):
                    if e4m3:
                        e = ref.row_exponent(float(x[h].abs().max()))
                        val = ref.e4m3_round(x[h] * 2.0 ** -e)
                        want[which + "e"][phys, h, off] = e + 127
                        assert torch.equal(ref.e4m3_values(getattr(c, which)[phys, h, off]), val)
                        want[which][phys, h, off] = getattr(c, which)[phys, h, off].cpu()
                        y = val * 2.0 ** e
                    else:
                        want[which][phys, h, off] = x[h].float().to(torch.bfloat16) if dtype is torch.bfloat16 and which == "v" else round_bf16(x[h])
                        y = want[which][phys, h, off].double()
                    if which == "k" and bounds:
                        b = want["bounds"][phys, h].double()
                        if off == 0:
                            b = torch.stack([y, y])
                        want["bounds"][phys, h] = torch.stack([torch.minimum(b[0], y), torch.maximum(b[1], y)]).to(torch.bfloat16)
    for x, t in want.items():
        assert torch.equal(getattr(c, x).cpu().contiguous().view(torch.uint8), t.contiguous().view(torch.uint8)) or \
            (x in ("bounds", "k", "v") and torch.equal(getattr(c, x).cpu().float(), t.float())), x
    if q_out is None:
        return
    got = q_out.cpu()
    for r in range(n):
        if r not in live:
            assert torch.equal(got[r], q0[r] if form == "in place" else torch.full_like(got[r], 5.0))
            continue
        x = turned(q0[r], int(at[r]), f)
        a, b = q0[r].double().abs().chunk(2, -1)
        err = torch.cat([a + b, a + b], -1) * 2.0 ** -22 + (2.0 ** -8 * x.abs() if dtype is torch.bfloat16 else 0)
        assert bool(((got[r].double() - x).abs() <= err).all()), r


def round_bf16(x):
    """Nearest bf16 of 64-bit numbers (through 32 bits with the last bit set where something was cut off)."""
    f = x.float()
    f = torch.where(f.double().abs() > x.abs(), torch.nextafter(f, torch.zeros_like(f)), f)
    bits = f.view(torch.int32) | (f.double() != x).to(torch.int32)
    return bits.view(torch.float32).to(torch.bfloat16)


def test_append_rotated_by_nothing_is_append():
    """Angles of zero: the same bits as kl_paged_append, one row per sequence or through row_starts."""
    for e4m3 in (False, True):
        a, b = (ref.Cache(6, 4, 16, 128, e4m3, True, seed=4) for _ in range(2))
        g = torch.Generator().manual_seed(5)
        k, v = (torch.randn(3, 4, 128, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        table = ref.scattered_table([20, 3, 33], 16, 6, seed=6)
        pos = i32([19, -1, 32])
        kl.kl_paged_append(a.handle, k, v, pos, table.cuda())
        kl.kl_paged_append_rotated(b.handle, k, v, pos, table.cuda(), freqs(128).cuda(), row_positions=i32([0, 0, 0]))
        for x in ("k", "v", "ke", "ve", "bounds"):
            if getattr(a, x) is not None:
                assert torch.equal(getattr(a, x).view(torch.uint8), getattr(b, x).view(torch.uint8)), x


def test_append_rotated_values_without_a_number():
    """Infinities and NaN stay with the pairs they turn with; e4m3 rows scale by what is finite."""
    c = ref.Cache(2, 1, 16, 64, True, True, seed=7)
    x = torch.ones(1, 1, 64)
    x[0, 0, 3], x[0, 0, 5] = math.inf, math.nan
    x[0, 0, 7] = 1000.0
    pos, table = i32([0]), i32([[1]])
    kl.kl_paged_append_rotated(c.handle, x.cuda(), torch.zeros_like(x).cuda(), pos, table, freqs(64).cuda(), row_positions=i32([3]))
    want = turned(x[0], 3, freqs(64))[0]
    got = c.values("k")[1, 0, 0]
    assert int(c.ke[1, 0, 0]) == ref.row_exponent(float(want[want.isfinite()].abs().max())) + 127
    assert torch.equal(got.isnan(), want.isnan())
    e = int(c.ke[1, 0, 0]) - 127
    assert torch.equal(got[want.isinf()], torch.copysign(torch.tensor(448.0 * 2.0 ** e, dtype=torch.float64), want[want.isinf()]))
    fine = want.isfinite()
    assert torch.equal(got[fine], ref.e4m3_round(want[fine] * 2.0 ** -e) * 2.0 ** e)
    assert c.ve[1, 0, 0] == 0 and not c.values("v")[1, 0, 0].any()


def test_append_rotated_reports_bad_pages():
    c = ref.Cache(4, 2, 16, 64, False, seed=8)
    k0 = c.k.clone()
    k = torch.ones(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    for pos, table, starts in ((i32([0]), i32([[9]]), None), (i32([16]), i32([[1]]), None), (i32([0]), i32([[-1]]), None), (i32([0, 0]), i32([[1], [2]]), [0, 2, 1]),
                               (i32([0, 0]), i32([[-3], [7]]), [0, 1, 9])):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        n = pos.numel() if starts is None else 3
        kl.kl_paged_append_rotated(c.handle, k[:n], k[:n], pos, table, freqs(64).cuda(), row_starts=None if starts is None else i32(starts), q=k[:n].clone(),
                                   q_out=k[:n].clone(), status=status)
        assert status.item() == kl.KL_ERR_OUT_OF_RANGE
        keep = c.k.clone()
        kl.kl_paged_append_rotated(c.handle, k[:1] * 3, k[:1], i32([1]), i32([[0]]), freqs(64).cuda(), status=status)   # the word is sticky
        assert torch.equal(c.k, keep)
    assert torch.equal(c.k[3], k0[3])


# ---- attention of a tree of new tokens
#
# Tolerances, derived: the tensor cores add 16 products at a time to a 32-bit sum and cut off what does not fit, which costs at most
# 2^-22 of the sum of magnitudes per step: (hd / 16 + 2) steps of a score, N / 16 + 2 of a result over N positions.  A score's error
# (relative to `reach`, the largest scale * sum |q k|) is a relative error of a probability; the exponential adds 2^-21 and the rounding of
# its argument reach * 2^-23.  A probability enters the second product with 2^-15 (bf16 caches: its upper 8 bits cut off, which leaves
# less than 2^-7 of it, and that rounded to 8 bits, half a step of which is 2^-8) or 2^-11 (e4m3: half a step of f16, twice where its largest
# scale moved) left out.  Errors of probabilities count twice, in the numerator and in the denominator.
# The sum of probabilities: N * 2^-24 at most.  The result is rounded to bf16, half a step of which is 2^-8 of it.

def tree_ref(c, q, seqs, starts, table, at, mask, window, sinks, scale):
    """out, lse, sum p |v|, reach in 64 bits."""
    k, v = c.values("k"), c.values("v")
    n, nq, hd = q.shape
    G = nq // c.nkv
    out, mass = (torch.zeros(n, nq, hd, dtype=torch.float64) for _ in range(2))
    lse, reach = torch.full((n, nq), -math.inf, dtype=torch.float64), torch.zeros(n, nq, dtype=torch.float64)
    for s, (base, T) in enumerate(seqs):
        for i in range(T if base >= 0 else 0):
            r = starts[s] + i
            me = base + i if at is None else max(int(at[r]), base)
            see = [p for p in range(base) if not window or p < sinks or p > me - window]
            for j in range(T):
                yes = (j <= i and (not window or i - j < window)) if mask is None else j // 32 < mask.shape[1] and (int(mask[r, j // 32]) >> (j % 32)) & 1
                if yes:
                    see.append(base + j)
            if not see:
                continue
            p = torch.tensor(see)
            phys, off = table[s].long()[p // c.page], p % c.page
            for h in range(c.nkv):
                kk, vv, qq = k[phys, h, off], v[phys, h, off], q[r, h * G:(h + 1) * G].double()
                sc = scale * qq @ kk.T
                w = torch.softmax(sc, 1)
                out[r, h * G:(h + 1) * G] = w @ vv
                mass[r, h * G:(h + 1) * G] = w @ vv.abs()
                lse[r, h * G:(h + 1) * G] = torch.logsumexp(sc, 1)
                reach[r, h * G:(h + 1) * G] = scale * (qq.abs() @ kk.abs().T).amax(1)
    return out, lse, mass, reach


def random_tree(T, seed):
    """Mask words and depths of a random tree of T tokens, every parent one of the few before."""
    g = np.random.default_rng(seed)
    words = -(-T // 32)
    seen, depth = [], []
    for i in range(T):
        p = max(0, i - int(g.integers(1, 4))) if i else -1
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return seen, depth, words


def check_tree(c, q, seqs, table, form="causal", window=0, sinks=0, scale=0.0, seed=0, mask=None, at=None, stream=None, single=False):
    starts = starts_of(seqs)
    n, nq, hd = q.shape
    if form == "tree":
        words = max(1, -(-max(t for _, t in seqs) // 32))
        mask = torch.zeros(n, words, dtype=torch.int64)
        at = torch.zeros(n, dtype=torch.int64)
        for s, (base, T) in enumerate(seqs):
            seen, depth, _ = random_tree(T, seed + s)
            for i in range(T):
                at[starts[s] + i] = max(base, 0) + depth[i]
                for w in range(words):
                    mask[starts[s] + i, w] = seen[i] >> 32 * w & 0xffffffff
    need = kl.kl_paged_tree_workspace_bytes(c.handle, nq)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    ws.fill_(0xff)
    out = torch.full((n, nq, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, nq), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dmask = None if mask is None else torch.where(mask >= 1 << 31, mask - (1 << 32), mask).to(torch.int32).cuda()
    kl.kl_paged_tree_attention(c.handle, q, out, i32([p for p, _ in seqs]), table.cuda(), ws, row_starts=None if single else i32(starts),
                               row_positions=None if at is None else at.to(torch.int32).cuda(), mask=dmask, scale=scale, window=window, n_sinks=sinks, lse=lse,
                               status=status, stream=stream)
    torch.cuda.synchronize()
    assert status.item() == 0
    sc = scale if scale > 0 else 1.0 / math.sqrt(hd)
    want, want_lse, mass, reach = tree_ref(c, q.cpu(), seqs, starts, table, at, mask, window, sinks, sc)
    N = max(b + t for b, t in seqs)
    score = reach * ((hd / 16 + 2) * 2.0 ** -22 + 2.0 ** -23) + 2.0 ** -21
    err = (2 * (score + 2.0 ** (-11 if c.e4m3 else -15))[..., None] + (N / 16 + 2) * 2.0 ** -22 + N * 2.0 ** -24) * mass + 2.0 ** -8 * want.abs() + 1e-30
    live = torch.zeros(n, dtype=torch.bool)
    for s, (base, T) in enumerate(seqs):
        live[starts[s]:starts[s] + T] = base >= 0
    got, got_lse = out.cpu().double(), lse.cpu().double()
    assert bool((got[~live] == 7.0).all()) and bool((got_lse[~live] == 7.0).all())
    off = (got - want).abs()[live]
    assert bool((off <= err[live]).all()), float((off / err[live]).max())
    empty = want_lse[live].isinf()
    assert torch.equal(got_lse[live][empty], want_lse[live][empty])
    tol = score + N * 2.0 ** -24 + 2.0 ** -20 * (1 + want_lse.abs())
    assert bool(((got_lse - want_lse).abs() <= tol)[live][~empty].all())
    return out, lse


TREES = [
    # e4m3, hd, nkv, nq, page, [(cached, new)], pages in [page][row][head] order
    (False, 128, 1, 4, 16, [(0, 1)], False),
    (False, 128, 2, 8, 16, [(700, 5)], False),
    (False, 128, 8, 32, 16, [(127, 1), (128, 2), (129, 3), (0, 7), (-1, 4), (1000, 8)], False),
    (False, 128, 1, 1, 4, [(60, 33), (0, 70), (255, 1)], True),
    (False, 128, 2, 24, 24, [(300, 11), (5, 20)], False),
    (False, 128, 1, 8, 64, [(2000, 64)], False),
    (False, 64, 3, 9, 8, [(513, 4), (90, 60)], True),
    (False, 64, 2, 2, 1024, [(1500, 100)], False),
    (False, 256, 2, 8, 16, [(333, 6), (0, 3), (64, 40)], False),
    (False, 256, 1, 12, 32, [(900, 1)], True),
    (True, 128, 1, 4, 16, [(0, 1)], False),
    (True, 128, 2, 8, 16, [(700, 5), (-1, 2), (20, 9)], False),
    (True, 128, 8, 32, 64, [(127, 1), (128, 2), (129, 3), (0, 7), (1000, 8)], True),
    (True, 128, 1, 8, 4, [(1500, 64)], False),
    (True, 64, 2, 6, 24, [(513, 4), (90, 60)], False),
    (True, 256, 2, 8, 16, [(333, 6), (0, 3), (64, 40)], True),
]


@pytest.mark.parametrize("e4m3,hd,nkv,nq,page,seqs,rows_first", TREES)
@pytest.mark.parametrize("form", ["causal", "tree"])
def test_tree_attention(e4m3, hd, nkv, nq, page, seqs, rows_first, form):
    lengths = [max(b, 0) + t for b, t in seqs]
    n_pages = sum(-(-x // page) for x in lengths) + 2
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, rows_first=rows_first, seed=11)
    table = ref.scattered_table(lengths, page, n_pages, seed=12)
    n = sum(t for _, t in seqs) + 3
    q = (torch.randn(n, nq + 1, hd, generator=torch.Generator().manual_seed(13)) * 1.5).to(torch.bfloat16).cuda()[:, :nq]
    check_tree(c, q, seqs, table, form, seed=14)


@pytest.mark.parametrize("e4m3,hd,nq,tokens", [(False, 128, 32, 2), (True, 128, 32, 2), (False, 128, 32, 9), (True, 64, 16, 5), (False, 256, 8, 3), (True, 256, 8, 40), (False, 64, 8, 64)])
def test_many_tiles_per_block_and_the_same_bits_every_time(e4m3, hd, nq, tokens):
    """Shares of many tiles, units cut by borders everywhere, lengths of every kind; no result may hang on the order of things."""
    g = np.random.default_rng(hd + tokens)
    seqs = [(int(g.integers(0, 2600)), tokens if i % 3 else 1 + i % tokens) for i in range(20)]
    seqs[5] = (-1, 3)
    page, nkv = 16, 8
    lengths = [max(b, 0) + t for b, t in seqs]
    n_pages = sum(-(-x // page) for x in lengths) + 2
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, seed=21)
    table = ref.scattered_table(lengths, page, n_pages, seed=22)
    n = sum(t for _, t in seqs)
    q = (torch.randn(n, nq, hd, generator=torch.Generator().manual_seed(23)) * 2).to(torch.bfloat16).cuda()
    first = check_tree(c, q, seqs, table, "tree" if tokens > 1 else "causal", seed=24)
    for _ in range(6):
        again = check_repeat(c, q, seqs, table, seed=24, tree=tokens > 1)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def check_repeat(c, q, seqs, table, seed, tree):
    """The same call without the reference."""
    starts, n = starts_of(seqs), q.shape[0]
    words = max(1, -(-max(t for _, t in seqs) // 32))
    mask, at = torch.zeros(n, words, dtype=torch.int64), torch.zeros(n, dtype=torch.int32)
    for s, (base, T) in enumerate(seqs):
        seen, depth, _ = random_tree(T, seed + s)
        for i in range(T):
            at[starts[s] + i] = max(base, 0) + depth[i]
            mask[starts[s] + i] = torch.tensor([seen[i] >> 32 * w & 0xffffffff for w in range(words)])
    ws = torch.empty(kl.kl_paged_tree_workspace_bytes(c.handle, q.shape[1]), dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    kl.kl_paged_tree_attention(c.handle, q, out, i32([p for p, _ in seqs]), table.cuda(), ws, row_starts=i32(starts), row_positions=at.cuda() if tree else None,
                               mask=torch.where(mask >= 1 << 31, mask - (1 << 32), mask).to(torch.int32).cuda() if tree else None, lse=lse)
    return out, lse


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (5, 1), (100, 4), (128, 128), (300, 130), (1000, 17), (5000, 4), (64, 5000)])
@pytest.mark.parametrize("form", ["single", "causal", "tree"])
def test_window_and_first_positions(e4m3, window, sinks, form):
    tokens = 1 if form == "single" else 13
    seqs = [(b, tokens) for b in (0, 3, 127, 128, 400, 777, 1100)] + [(-1, tokens)]
    page = 16
    lengths = [max(b, 0) + t for b, t in seqs]
    n_pages = sum(-(-x // page) for x in lengths) + 2
    c = ref.Cache(n_pages, 2, page, 128, e4m3, seed=31)
    table = ref.scattered_table(lengths, page, n_pages, seed=32)
    for s, (b, t) in enumerate(seqs):   # pages that nobody may look up name nothing
        for p in range(max(0, b) // page):
            if p * page >= sinks and (p + 1) * page <= b - window + 1:
                table[s, p] = -5
    q = torch.randn(sum(t for _, t in seqs), 6, 128, generator=torch.Generator().manual_seed(33)).to(torch.bfloat16).cuda()
    check_tree(c, q, seqs, table, "tree" if form == "tree" else "causal", window, sinks, seed=34, single=form == "single")


def test_masks_that_leave_rows_empty_and_bits_of_all_kinds():
    """Masks of any bits: rows that see nothing (no cached positions either), only later tokens, words that are missing or too many."""
    for e4m3 in (False, True):
        seqs = [(0, 40), (5, 70), (200, 3), (0, 1)]
        lengths = [b + t for b, t in seqs]
        c = ref.Cache(20, 2, 32, 128, e4m3, seed=41)
        table = ref.scattered_table(lengths, 32, 20, seed=42)
        n = sum(t for _, t in seqs)
        g = torch.Generator().manual_seed(43)
        q = torch.randn(n, 8, 128, generator=g).to(torch.bfloat16).cuda()
        for words in (1, 2, 3, 5):
            mask = torch.randint(0, 1 << 32, (n, words), generator=g)
            mask[::3] = 0
            mask[1] = 0xffffffff
            mask[2, 0] = 1 << 31
            check_tree(c, q, seqs, table, "mask", mask=mask)
        out, lse = check_tree(c, q, seqs, table, "mask", mask=torch.zeros(n, 2, dtype=torch.int64))
        assert not out[:40].any() and bool((lse[:40] == -math.inf).all())


@pytest.mark.parametrize("e4m3", [False, True])
def test_what_a_token_does_not_see_does_not_matter(e4m3):
    """NaN in unused pages and rows, and in new tokens that others do not see: they reach only the tokens that see them."""
    seqs = [(100, 6), (30, 40)]
    page, nkv, hd = 16, 2, 128
    lengths = [b + t for b, t in seqs]
    clean = ref.Cache(20, nkv, page, hd, e4m3, seed=51)
    table = ref.scattered_table(lengths, page, 20, seed=52)
    n = sum(t for _, t in seqs)
    q = torch.randn(n, 6, hd, generator=torch.Generator().manual_seed(53)).to(torch.bfloat16).cuda()
    want, want_lse = check_tree(clean, q, seqs, table, "tree", seed=54)
    bad = ref.Cache(20, nkv, page, hd, e4m3, seed=51, poison=True)
    used = torch.zeros(20, page, dtype=torch.bool)
    for s, x in enumerate(lengths):
        for p in range(x):
            used[int(table[s, p // page]), p % page] = True
    for which in ("k", "v"):
        keep = used[:, None, :, None].expand(20, nkv, page, hd).cuda()
        t, src = getattr(bad, which), getattr(clean, which)
        t.view(torch.uint8 if e4m3 else torch.bfloat16).copy_(torch.where(keep, src.view(torch.uint8 if e4m3 else torch.bfloat16), t.view(torch.uint8 if e4m3 else torch.bfloat16)))
    if e4m3:
        bad.ke.copy_(clean.ke)
        bad.ve.copy_(clean.ve)
        bad.ke[~used[:, None, :].expand(20, nkv, page).cuda()] = 254
        bad.ve[~used[:, None, :].expand(20, nkv, page).cuda()] = 254
    got, got_lse = check_repeat(bad, q, seqs, table, 54, True)
    assert torch.equal(got, want) and torch.equal(got_lse, want_lse)
    # a key and a value of new tokens that hold NaN (bf16: infinity in the value): token 2 of the first sequence, 5 of the second
    nan = 0x7f if e4m3 else math.nan
    starts = starts_of(seqs)
    hit_v, hit_k = torch.zeros(n, dtype=torch.bool), torch.zeros(n, dtype=torch.bool)
    for s, j in ((0, 2), (1, 5)):
        at = seqs[s][0] + j
        phys, off = int(table[s, at // page]), at % page
        (bad.v.view(torch.uint8) if e4m3 else bad.v)[phys, 1, off, 7] = nan if e4m3 else math.inf
        seen, _, _ = random_tree(seqs[s][1], 54 + s)
        for i in range(seqs[s][1]):
            hit_v[starts[s] + i] = bool(seen[i] >> j & 1)
    got, got_lse = check_repeat(bad, q, seqs, table, 54, True)
    assert torch.equal(got_lse, want_lse)
    for h in range(6):
        for r in range(n):
            other = torch.ones(hd, dtype=torch.bool)
            if h >= 3 and hit_v[r]:
                assert not bool(got[r, h, 7].isfinite())
                other[7] = False
            assert torch.equal(got[r, h][other], want[r, h][other]), (r, h)
    (bad.v.view(torch.uint8) if e4m3 else bad.v).copy_(clean.v.view(torch.uint8) if e4m3 else clean.v)
    at = seqs[1][0] + 5
    (bad.k.view(torch.uint8) if e4m3 else bad.k)[int(table[1, at // page]), 0, at % page, 3] = nan
    seen, _, _ = random_tree(seqs[1][1], 55)
    for i in range(seqs[1][1]):
        hit_k[starts[1] + i] = bool(seen[i] >> 5 & 1)
    got, got_lse = check_repeat(bad, q, seqs, table, 54, True)
    for r in range(n):
        if hit_k[r]:
            assert bool(got[r, :3].isnan().all()) and bool(got_lse[r, :3].isnan().all())
            assert torch.equal(got[r, 3:], want[r, 3:])
        else:
            assert torch.equal(got[r], want[r])


def test_values_of_very_different_scales():
    """e4m3: zero rows (scale byte 0) count in the denominator; scales that grow along the sequence; keys of large scales."""
    c = ref.Cache(40, 1, 16, 128, True, seed=61)
    c.ve[:] = 118
    c.ve[::3] = 0
    c.v.view(torch.uint8)[::3] = 0
    c.ve[::7] = 126
    c.ke[::5] = 123
    table = ref.scattered_table([600], 16, 40, seed=62)
    q = torch.randn(5, 4, 128, generator=torch.Generator().manual_seed(63)).to(torch.bfloat16).cuda()
    check_tree(c, q, [(595, 5)], table)


def test_single_tokens_agree_with_paged_attention():
    """One row per sequence, no window or a window: the single-token operator's answers, to both operators' roundings."""
    for e4m3 in (False, True):
        pos = [0, 15, 300, -1, 1000]
        c = ref.Cache(100, 4, 16, 128, e4m3, seed=71)
        table = ref.scattered_table([p + 1 for p in pos], 16, 100, seed=72)
        q = torch.randn(5, 16, 128, generator=torch.Generator().manual_seed(73)).to(torch.bfloat16).cuda()
        for window in (0, 100):
            a, b = torch.zeros_like(q), torch.zeros_like(q)
            ws = torch.empty(max(kl.kl_paged_workspace_bytes(c.handle, 16, 5, table.shape[1]), kl.kl_paged_tree_workspace_bytes(c.handle, 16)), dtype=torch.uint8, device="cuda")
            kl.kl_paged_attention(c.handle, q, a, i32(pos), table.cuda(), ws, window=window)
            kl.kl_paged_tree_attention(c.handle, q, b, i32(pos), table.cuda(), ws, window=window)
            # two roundings to bf16, and the e4m3 form's 2^-11 (twice; bf16 2^-15) of sum p |v|, at most the largest |v|
            tol = 2.0 ** -7 * a.abs() + (2.0 ** -10 * 448 * 2.0 ** -5 if e4m3 else 2.0 ** -14 * 5)
            assert bool(((a.float() - b.float()).abs() <= tol.float()).all())
            assert not b[3].any()


def test_captured_on_a_stream_and_replayed_while_the_sequences_grow():
    """Append, attention and sampling of a drafted chain captured once and replayed with other positions and rows."""
    page, nkv, nq, hd, vocab = 16, 2, 8, 128, 500
    c = ref.Cache(30, nkv, page, hd, False, seed=81)
    table = ref.scattered_table([200, 150], page, 30, seed=82).cuda()
    g = torch.Generator().manual_seed(83)
    n = 6
    k, v, q, qo, out = (torch.zeros(n, h, hd, dtype=torch.bfloat16, device="cuda") for h in (nkv, nkv, nq, nq, nq))
    pos, starts, u, tokens = i32([0, 0]), i32([0, 4, 6]), torch.zeros(n, device="cuda"), i32([0] * n)
    head = (torch.randn(nq * hd, vocab, generator=g) / 20).cuda()
    logits = torch.zeros(n, vocab, device="cuda")
    ws = torch.empty(kl.kl_paged_tree_workspace_bytes(c.handle, nq), dtype=torch.uint8, device="cuda")
    f = freqs(hd).cuda()

    def step(stream):
        kl.kl_paged_append_rotated(c.handle, k, v, pos, table, f, row_starts=starts, q=q, q_out=qo, stream=stream)
        kl.kl_paged_tree_attention(c.handle, qo, out, pos, table, ws, row_starts=starts, stream=stream)
        torch.mm(out.view(n, -1).float(), head, out=logits)
        kl.kl_sample(logits, u, tokens, stream=stream)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        step(st)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step(torch.cuda.current_stream())
        for at in ([0, 0], [150, 33], [-1, 60], [196, 148]):
            for t in (k, v, q):
                t.copy_(torch.randn(t.shape, generator=g).to(torch.bfloat16))
            u.copy_(torch.rand(n, generator=g))
            pos.copy_(torch.tensor(at, dtype=torch.int32))
            tokens.fill_(-9)
            graph.replay()
            st.synchronize()
            seqs = [(at[0], 4), (at[1], 2)]
            want_q = torch.stack([turned(q[r].cpu(), max(at[s], 0) + i, f.cpu()) for s, (_, t) in enumerate(seqs) for i, r in enumerate(range(starts_of(seqs)[s], starts_of(seqs)[s] + t))])
            live = [r for s, (b, t) in enumerate(seqs) for r in range(starts_of(seqs)[s], starts_of(seqs)[s] + t) if b >= 0]
            assert bool(((qo.cpu().double() - want_q).abs() <= 2.0 ** -8 * want_q.abs() + 2.0 ** -20)[live].all())
            want, _, mass, reach = tree_ref(c, qo.cpu(), seqs, starts_of(seqs), table.cpu(), None, None, 0, 0, 1 / math.sqrt(hd))
            score = reach * ((hd / 16 + 2) * 2.0 ** -22 + 2.0 ** -23) + 2.0 ** -21
            err = (2 * (score + 2.0 ** -15)[..., None] + 15 * 2.0 ** -22 + 200 * 2.0 ** -24) * mass + 2.0 ** -8 * want.abs() + 1e-30
            assert bool(((out.cpu().double() - want).abs() <= err)[live].all())
            for r in range(n):
                w = torch.softmax(logits[r].cpu().double(), 0)
                cum = torch.cumsum(w, 0)
                assert int(tokens[r]) == int((cum <= float(u[r]) * cum[-1]).sum())


def test_tree_attention_reports_bad_pages_and_positions():
    c = ref.Cache(4, 2, 16, 128, False, seed=91)
    q = torch.ones(3, 4, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(kl.kl_paged_tree_workspace_bytes(c.handle, 4), dtype=torch.uint8, device="cuda")
    for pos, table, starts in ((i32([0]), i32([[9]]), [0, 3]), (i32([15]), i32([[1]]), [0, 3]), (i32([1 << 30]), i32([[1]]), [0, 3]), (i32([20]), i32([[1, -1]]), [0, 3]),
                               (i32([0, 0]), i32([[1], [2]]), [0, 2, 1]), (i32([0, 0]), i32([[1], [2]]), [0, 1, 9]), (i32([0, 0]), i32([[1], [2]]), [-1, 1, 2])):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 7.0)
        kl.kl_paged_tree_attention(c.handle, q, out, pos, table, ws, row_starts=i32(starts), status=status)
        assert status.item() == kl.KL_ERR_OUT_OF_RANGE
        out.fill_(7.0)
        kl.kl_paged_tree_attention(c.handle, q, out, i32([0]), i32([[0]]), ws, row_starts=i32([0, 3]), status=status)   # the word is sticky
        assert bool((out == 7.0).all())
