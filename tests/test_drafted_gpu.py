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
