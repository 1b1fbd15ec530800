"""The paged key-value cache operators against plain 64-bit restatements, through the C ABI.

Tolerances of the attention tests, derived: with u = 2^-8 (half a bf16 step, relative) a query enters the score product
as two bf16 numbers, which leaves u^2 = 2^-16 of it out (nothing when the query is bf16); the products are summed in 32
bits (head_dim + a few roundings of 2^-24 of sum |q k|); the exponential is good to 2^-21; a probability enters the value
product as two numbers of at least 8 bits, which leaves 2^-16 of it out; up to N terms are added in 32 bits (N * 2^-24 of
sum p |v|).  Relative errors of the probabilities count twice, in the numerator and in the denominator.  The result is
rounded once more where the output is bf16."""
import math

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


def rows_like(n, nkv, hd, dtype, seed, fused=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, 3, nkv, hd, generator=g) * torch.exp(torch.randn(n, 3, nkv, 1, generator=g))
    x = x.to(dtype).cuda()
    return x[:, 0], x[:, 2]   # rows of a wider tensor


def check_attention(cache, q, positions, table, scale=0.0, window=0, selected=None, with_lse=True, out=None, stream=None):
    n, nq, hd = q.shape
    ws = torch.empty(kl.kl_paged_workspace_bytes(cache.handle, nq, n, table.shape[1]), dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 7.0) if out is None else out
    lse = torch.full((n, nq), 7.0, device="cuda") if with_lse else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sel = None if selected is None else selected.cuda()
    ws.fill_(0xff)
    kl.kl_paged_attention(cache.handle, q, out, positions.cuda(), table.cuda(), ws, scale=scale, window=window, selected=sel, lse=lse, status=status,
                          stream=stream)
    torch.cuda.synchronize()
    assert status.item() == 0
    sc = scale if scale > 0 else 1.0 / math.sqrt(hd)
    want, want_lse, mass, reach = ref.attention_ref(cache.values("k"), cache.values("v"), q.cpu(), positions.tolist(), table, cache.page, sc, window,
                                                    selected)
    terms = int(positions.max()) + 1
    score = reach * ((2.0 ** -16 if q.dtype == torch.float32 else 0.0) + (hd + 8) * 2.0 ** -24)
    err = 2 * (score + 2.0 ** -21 + 2.0 ** -16)[..., None] * mass + terms * 2.0 ** -24 * mass + 1e-30
    if q.dtype == torch.bfloat16:
        err = err + 2.0 ** -8 * want.abs()
    off = (out.cpu().double() - want).abs()
    assert bool((off <= err).all()), float((off / err).max())
    if with_lse:
        empty = want_lse.isinf()
        got = lse.cpu().double()
        assert torch.equal(got[empty], want_lse[empty])
        tol = score + terms * 2.0 ** -24 + 2.0 ** -20 * (1 + want_lse.abs())
        assert bool(((got - want_lse).abs() <= tol)[~empty].all())
    return out


# ---- append and read

APPENDS = [
    # e4m3, rows, hd, nkv, page, [(first position, rows)], pages in [page][row][head] order
    (False, torch.bfloat16, 128, 8, 16, [(0, 1)], False),
    (True, torch.bfloat16, 128, 8, 16, [(0, 1)], False),
    (True, torch.float32, 128, 2, 4, [(3, 1), (-1, 0), (7, 9), (0, 4)], False),
    (False, torch.float32, 64, 3, 24, [(23, 50), (0, 0), (5, 1), (48, 25)], True),
    (True, torch.bfloat16, 64, 1, 64, [(63, 130), (10, 3)], False),
    (True, torch.bfloat16, 256, 4, 8, [(0, 8), (8, 8), (17, 1)], True),
    (False, torch.bfloat16, 256, 2, 1024, [(1000, 40), (0, 3)], False),
    (True, torch.float32, 128, 8, 16, [(15, 33), (0, 100), (-1, 5), (31, 2)], False),
]


@pytest.mark.parametrize("e4m3,dtype,hd,nkv,page,seqs,rows_first", APPENDS)
@pytest.mark.parametrize("bounds", [True, False])
def test_append_and_read(e4m3, dtype, hd, nkv, page, seqs, rows_first, bounds):
    lengths = [max(p, 0) + r for p, r in seqs]
    n_pages = sum(-(-x // page) for x in lengths) + 3
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, bounds, rows_first, seed=1)
    table = ref.scattered_table(lengths, page, n_pages, seed=2)
    positions = [p for p, _ in seqs]
    starts = [sum(r for _, r in seqs[:i]) for i in range(len(seqs) + 1)]
    n = starts[-1] + 5   # rows behind the last sequence
    k, v = rows_like(n, nkv, hd, dtype, 3)
    before = {x: getattr(c, x).cpu().clone() for x in ("k", "v", "ke", "ve", "bounds") if getattr(c, x) is not None}
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kl.kl_paged_append(c.handle, k, v, i32(positions), table.cuda(), row_starts=i32(starts), status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    want = {x: t.clone() for x, t in before.items()}
    held = {"k": {}, "v": {}}
    for s, (p0, cnt) in enumerate(seqs):
        for i in range(cnt if p0 >= 0 else 0):
            phys, off = int(table[s, (p0 + i) // page]), (p0 + i) % page
            for which, rows in (("k", k), ("v", v)):
                x = rows[starts[s] + i].cpu()
                for h in range(nkv):
                    if e4m3:
                        e = ref.row_exponent(float(x[h].double().abs().max()))
                        val = ref.e4m3_round(x[h].double() * 2.0 ** -e)
                        want[which + "e"][phys, h, off] = e + 127
                        got = ref.e4m3_values(getattr(c, which)[phys, h, off])
                        assert torch.equal(got, val)
                        want[which][phys, h, off] = getattr(c, which)[phys, h, off].cpu()
                        held[which][(s, i, h)] = val * 2.0 ** e
                    else:
                        want[which][phys, h, off] = x[h].to(torch.bfloat16)
                        held[which][(s, i, h)] = x[h].to(torch.bfloat16).double()
                    if which == "k" and bounds:
                        b = want["bounds"][phys, h].double()
                        y = held["k"][(s, i, h)]
                        if off == 0:
                            b = torch.stack([y, y])
                        want["bounds"][phys, h] = torch.stack([torch.minimum(b[0], y), torch.maximum(b[1], y)]).to(torch.bfloat16)
    for x, t in want.items():
        assert torch.equal(getattr(c, x).cpu().contiguous().view(torch.uint8), t.contiguous().view(torch.uint8)) or \
            (x == "bounds" and torch.equal(getattr(c, x).cpu(), t)), x

    for out_type in (torch.bfloat16, torch.float32):
        ko, vo = (torch.full((n, nkv, hd), 5.0, dtype=out_type, device="cuda") for _ in range(2))
        kl.kl_paged_read(c.handle, ko, vo, i32(positions), table.cuda(), row_starts=i32(starts), status=status)
        torch.cuda.synchronize()
        assert status.item() == 0
        for which, o in (("k", ko), ("v", vo)):
            exp = torch.full((n, nkv, hd), 5.0, dtype=torch.float64)
            for (s, i, h), y in held[which].items():
                exp[starts[s] + i, h] = y
            assert torch.equal(o.cpu().double(), exp)


def test_append_one_row_per_sequence_equals_row_starts():
    for e4m3 in (False, True):
        a, b = (ref.Cache(40, 4, 16, 128, e4m3, bounds=True, seed=5) for _ in range(2))
        lengths = [17, 1, 33, 16, 5]
        table = ref.scattered_table(lengths, 16, 40, seed=6)
        pos = i32([16, 0, -1, 15, 4])
        k, v = rows_like(5, 4, 128, torch.bfloat16, 7)
        kl.kl_paged_append(a.handle, k, v, pos, table.cuda())
        kl.kl_paged_append(b.handle, k, v, pos, table.cuda(), row_starts=i32([0, 1, 2, 3, 4, 5]))
        torch.cuda.synchronize()
        for x in ("k", "v", "ke", "ve", "bounds"):
            if getattr(a, x) is not None:
                assert torch.equal(getattr(a, x).view(torch.uint8), getattr(b, x).view(torch.uint8)), x


def test_append_extreme_rows():
    """Zeros, the smallest and largest numbers, an exact border of the scale, infinities and NaN."""
    hd = 64
    x = torch.zeros(8, 1, hd)
    x[1, 0, 3] = 1e-45
    x[2, 0, 5] = 3.3e38
    x[2, 0, 6] = -1e38
    x[3, 0, 0] = 448.0
    x[3, 0, 1] = 447.0
    x[4, 0, 0] = torch.nextafter(torch.tensor(448.0), torch.tensor(1e9))
    x[5, 0, 0], x[5, 0, 1], x[5, 0, 2] = math.inf, -math.inf, 3.0
    x[6, 0, 0], x[6, 0, 1] = math.nan, 1.0
    x[7] = math.inf
    c = ref.Cache(3, 1, 4, hd, True, bounds=True, seed=1)
    kl.kl_paged_append(c.handle, x.cuda(), x.cuda(), i32([0]), i32([[2, 0]]), row_starts=i32([0, 8]))
    torch.cuda.synchronize()
    want_e = [0, 0, 247, 127, 128, None, None, 0]
    for i in range(8):
        phys, off = (2, 0)[i // 4], i % 4
        e = int(c.ke[phys, 0, off]) - 127
        if want_e[i] is not None:
            assert e + 127 == want_e[i], i
        fin = x[i, 0].double()
        big = float(fin[fin.isfinite()].abs().max()) if fin.isfinite().any() else 0.0
        assert e == ref.row_exponent(big)
        val, exp = ref.e4m3_values(c.k[phys, 0, off]), ref.e4m3_round(fin * 2.0 ** -e)
        assert torch.equal(val.isnan(), exp.isnan()) and torch.equal(val.nan_to_num(0.0), exp.nan_to_num(0.0)), i
    lo, hi = c.bounds[0, 0].cpu().double()   # rows 4..7: a column that holds NaN is bounded by its other rows
    held = c.values("k")[0, 0]
    big = torch.where(held.isnan(), -math.inf, held).amax(0).to(torch.bfloat16).double()
    low = torch.where(held.isnan(), math.inf, held).amin(0).to(torch.bfloat16).double()
    assert torch.equal(hi, big) and torch.equal(lo, low)


# ---- attention

ATTENTION = [
    # e4m3, dtype, hd, nq, nkv, page, positions, rows_first
    (False, torch.bfloat16, 128, 8, 2, 16, [0], False),
    (False, torch.bfloat16, 128, 32, 8, 16, [332], False),
    (True, torch.bfloat16, 128, 32, 8, 64, [700, 0, -1, 63, 64, 65], False),
    (False, torch.float32, 128, 4, 4, 4, [5, 130, 15, 16, 17], False),
    (True, torch.float32, 128, 16, 2, 8, [90, -1, 31, 7, 200], True),
    (False, torch.bfloat16, 64, 6, 2, 24, [500, 23, 24, 47], True),
    (True, torch.bfloat16, 64, 12, 4, 4, [61, 3, 255], False),
    (False, torch.bfloat16, 256, 8, 1, 16, [111, 16], False),
    (True, torch.bfloat16, 256, 24, 2, 128, [400, 127, 128], True),
    (False, torch.float32, 64, 33, 3, 12, [100, 11], False),
    (True, torch.float32, 256, 10, 10, 20, [77], False),
    (True, torch.bfloat16, 128, 40, 2, 1024, [2500, 1023], False),
    (False, torch.bfloat16, 128, 4, 2, 32, [20000], False),
    (True, torch.float32, 64, 8, 8, 16, list(range(-1, 90)), False),
]


@pytest.mark.parametrize("e4m3,dtype,hd,nq,nkv,page,positions,rows_first", ATTENTION)
@pytest.mark.parametrize("window", [0, 1, 37])
def test_attention(e4m3, dtype, hd, nq, nkv, page, positions, rows_first, window):
    lengths = [p + 1 for p in positions]
    n_pages = sum(-(-x // page) for x in lengths) + 2
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, rows_first=rows_first, seed=11)
    table = ref.scattered_table(lengths, page, n_pages, seed=12)
    g = torch.Generator().manual_seed(13)
    q = (torch.randn(len(positions), 2, nq, hd, generator=g) * (0.02 if e4m3 else 1.0)).to(dtype).cuda()[:, 1]   # strided
    check_attention(c, q, torch.tensor(positions, dtype=torch.int32), table, window=window)


@pytest.mark.parametrize("e4m3", [False, True])
def test_attention_ignores_what_lies_outside(e4m3):
    """Everything but the attended rows of the pool is NaN, infinite or 1e38: no trace of it may reach the result."""
    page, hd, nkv = 8, 128, 2
    positions = torch.tensor([19, 0, 40], dtype=torch.int32)
    table = ref.scattered_table([20, 1, 41], page, 16, seed=3)
    good = ref.Cache(16, nkv, page, hd, e4m3, seed=4)
    bad = ref.Cache(16, nkv, page, hd, e4m3, seed=4, poison=True)
    if e4m3:
        bad.ke.fill_(255), bad.ve.fill_(255)
    for s in range(3):
        for p in range(max(0, int(positions[s]) - 12), int(positions[s]) + 1):
            phys, r = int(table[s, p // page]), p % page
            for x in ("k", "v", "ke", "ve"):
                if getattr(good, x) is not None:
                    getattr(bad, x)[phys, :, r] = getattr(good, x)[phys, :, r]
    q = torch.randn(3, 4, hd, generator=torch.Generator().manual_seed(1)).mul_(0.05).cuda()
    a = check_attention(good, q, positions, table, window=13)
    b = torch.full_like(q, 7.0)
    ws = torch.empty(kl.kl_paged_workspace_bytes(bad.handle, 4, 3, table.shape[1]), dtype=torch.uint8, device="cuda")
    kl.kl_paged_attention(bad.handle, q, b, positions.cuda(), table.cuda(), ws, window=13)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


@pytest.mark.parametrize("e4m3,hd,nq,nkv,page", [(False, 128, 8, 2, 16), (True, 128, 32, 4, 4), (True, 64, 3, 1, 24), (False, 256, 4, 2, 8)])
@pytest.mark.parametrize("n_select", [1, 3, 40])
@pytest.mark.parametrize("window", [0, 50])
def test_attention_over_selected_pages(e4m3, hd, nq, nkv, page, n_select, window):
    positions = [page * 37 + 3, -1, page - 1, page, 5 * page + 2]
    lengths = [p + 1 for p in positions]
    n_pages = sum(-(-x // page) for x in lengths) + 2
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, seed=21)
    table = ref.scattered_table(lengths, page, n_pages, seed=22)
    g = torch.Generator().manual_seed(23)
    sel = torch.full((len(positions), nkv, n_select), -1, dtype=torch.int32)
    for s, p in enumerate(positions):
        pages = p // page + 1 if p >= 0 else 0
        for h in range(nkv):
            keep = torch.randperm(pages, generator=g)[:max(0, min(n_select, pages) - (s == 4))]   # one entry left at -1
            keep = keep if h % 2 else keep.sort().values                                        # any order will do
            sel[s, h, :len(keep)] = keep.to(torch.int32)
    q = (torch.randn(len(positions), nq, hd, generator=g) * (0.02 if e4m3 else 1.0)).to(torch.bfloat16).cuda()
    check_attention(c, q, torch.tensor(positions, dtype=torch.int32), table, window=window, selected=sel)


def test_attention_extreme_scores():
    """Scores hundreds apart, one position far above all others, zero queries, an explicit scale."""
    for e4m3 in (False, True):
        c = ref.Cache(20, 2, 16, 128, e4m3, seed=31)
        table = ref.scattered_table([300], 16, 20, seed=32)
        pos = torch.tensor([299], dtype=torch.int32)
        g = torch.Generator().manual_seed(33)
        q = torch.randn(1, 8, 128, generator=g) * (0.3 if e4m3 else 8.0)
        q[0, 3] = 0.0
        check_attention(c, q.cuda(), pos, table, scale=0.7)
        check_attention(c, (q * 1e-30).cuda(), pos, table, scale=1.0)
        check_attention(c, (q * 1e-3).to(torch.bfloat16).cuda(), pos, table, scale=3.0)


def test_attention_scales_far_apart():
    """e4m3 rows whose scales span the whole range: the loudest values and the most likely positions are different ones."""
    c = ref.Cache(10, 1, 16, 128, True, seed=41)
    c.ve[:] = torch.randint(60, 180, c.ve.shape, generator=torch.Generator().manual_seed(42)).to(torch.uint8).cuda()
    c.ke[:] = torch.randint(100, 120, c.ke.shape, generator=torch.Generator().manual_seed(43)).to(torch.uint8).cuda()
    table = ref.scattered_table([160], 16, 10, seed=44)
    q = torch.randn(1, 5, 128, generator=torch.Generator().manual_seed(45)) * 0.2
    check_attention(c, q.cuda(), torch.tensor([159], dtype=torch.int32), table)


def test_attention_many_sequences_and_batch_order():
    """More sequences than blocks of the grid, and the same sequences in another order give the same rows, to the bit
    when each is computed by itself."""
    page, hd, nkv, nq = 16, 64, 2, 8
    g = torch.Generator().manual_seed(51)
    lengths = [int(x) for x in torch.randint(0, 120, (700,), generator=g)]
    n_pages = sum(-(-x // page) for x in lengths)
    c = ref.Cache(n_pages, nkv, page, hd, False, seed=52)
    table = ref.scattered_table(lengths, page, n_pages, seed=53)
    q = torch.randn(len(lengths), nq, hd, generator=g).cuda()
    check_attention(c, q, torch.tensor(lengths, dtype=torch.int32) - 1, table)


@pytest.mark.parametrize("e4m3,dtype,hd,nq,nkv,page,lengths", [
    (False, torch.bfloat16, 128, 32, 8, 16, [333]),
    (True, torch.float32, 128, 10, 1, 4, [1, 100, 0, 700]),
    (True, torch.bfloat16, 64, 8, 8, 64, [(37 * i) % 1000 for i in range(40)]),     # more pairs than blocks of the grid
    (False, torch.float32, 256, 3, 3, 8, [(53 * i) % 400 for i in range(70)]),
    (False, torch.bfloat16, 128, 16, 2, 16, [0, 0, 1200, 3, 0]),
])
@pytest.mark.parametrize("selected", [False, True])
def test_attention_wider_tables(e4m3, dtype, hd, nq, nkv, page, lengths, selected):
    """The width of the table, or of the page list, decides whether blocks share a (sequence, head) pair: both ways are right."""
    n_pages = sum(-(-x // page) for x in lengths)
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, seed=61)
    g = torch.Generator().manual_seed(62)
    q = (torch.randn(len(lengths), nq, hd, generator=g) * (0.02 if e4m3 else 1.0)).to(dtype).cuda()
    for extra in (0, 16384 // page):
        table = ref.scattered_table(lengths, page, n_pages, seed=63, extra=extra)
        sel = None
        if selected:   # every third page, then fillers up to the table's width
            sel = torch.full((len(lengths), nkv, table.shape[1]), -1, dtype=torch.int32)
            for i, x in enumerate(lengths):
                pages = list(range(0, -(-x // page), 3))
                sel[i, :, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
        check_attention(c, q, torch.tensor(lengths, dtype=torch.int32) - 1, table, selected=sel)


def test_attention_many_more_sequences_than_threads():
    """Lengths beyond those kept in shared memory, several sequences per thread of the prefix sum, three of four empty."""
    page, hd, n = 16, 64, 2100
    lengths = [(i * 7) % 40 if i % 4 == 0 else 0 for i in range(n)]
    n_pages = sum(-(-x // page) for x in lengths)
    c = ref.Cache(n_pages, 1, page, hd, True, seed=54)
    table = ref.scattered_table(lengths, page, n_pages, seed=55)
    q = (torch.randn(n, 2, hd, generator=torch.Generator().manual_seed(56)) * 0.05).to(torch.bfloat16).cuda()
    check_attention(c, q, torch.tensor(lengths, dtype=torch.int32) - 1, table)


def test_single_rows_pages_and_heads_of_any_stride():
    """Strides of dimensions of size one mean nothing, to torch or to the library."""
    k = torch.zeros(3, 1, 16, 64, dtype=torch.bfloat16, device="cuda").as_strided((3, 1, 16, 64), (1024, 7, 64, 1))
    v = torch.zeros_like(k)
    cache = kl.PagedCache(k, v)
    rows = torch.randn(1, 1, 64, device="cuda").as_strided((1, 1, 64), (3, 5, 1))
    table = i32([[2]]).as_strided((1, 1), (9, 1))
    kl.kl_paged_append(cache, rows, rows * 2, i32([3]), table)
    q = torch.randn(1, 4, 64, device="cuda").as_strided((1, 4, 64), (1, 64, 1))
    out = torch.zeros(1, 4, 64, device="cuda")
    ws = torch.empty(kl.kl_paged_workspace_bytes(cache, 4, 1, 1), dtype=torch.uint8, device="cuda")
    kl.kl_paged_attention(cache, q, out, i32([3]), table, ws, window=1)
    torch.cuda.synchronize()
    assert torch.equal(k[2, 0, 3], rows[0, 0].to(torch.bfloat16))
    want = (rows[0] * 2).to(torch.bfloat16).float().expand(4, 64)   # one position: its value, up to the split of p = 1 (exact)
    assert torch.equal(out[0], want)


FRESH = """
import torch
from paper_2410_23668_b200 import binding as kl
c = kl.PagedCache.allocate(8, 2, 16, 128, kl.KL_KV_E4M3, bounds=True)
pos, table = torch.tensor([40], dtype=torch.int32, device="cuda"), torch.tensor([[3, 1, 0]], dtype=torch.int32, device="cuda")
k, q = torch.randn(1, 2, 128, device="cuda"), torch.randn(1, 8, 128, device="cuda")
ws = torch.empty(kl.kl_paged_workspace_bytes(c, 8, 1, 3), dtype=torch.uint8, device="cuda")
sel, out = torch.zeros(1, 2, 2, dtype=torch.int32, device="cuda"), torch.zeros(1, 8, 128, device="cuda")
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    st = torch.cuda.current_stream()
    kl.kl_paged_append(c, k, k, pos, table, stream=st)
    kl.kl_paged_select(c, q, pos, table, sel, ws, stream=st)
    kl.kl_paged_attention(c, q, out, pos, table, ws, selected=sel, stream=st)
g.replay()
torch.cuda.synchronize()
a, b = out.clone(), torch.zeros_like(out)
kl.kl_paged_attention(c, q, b, pos, table, ws, selected=sel)
torch.cuda.synchronize()
assert torch.equal(a, b) and bool(a.abs().max() > 0) and sel.tolist() == [[[0, 2], [0, 2]]]
print("fresh ok")
"""


def test_first_calls_of_a_process_inside_a_capture():
    import subprocess
    import sys
    from pathlib import Path
    r = subprocess.run([sys.executable, "-c", FRESH], capture_output=True, text=True, timeout=300, cwd=Path(__file__).resolve().parent.parent)
    assert r.returncode == 0 and "fresh ok" in r.stdout, r.stderr[-2000:]


def test_attention_same_result_every_time():
    c = ref.Cache(700, 4, 16, 128, True, seed=61)
    table = ref.scattered_table([9000, 1200], 16, 700, seed=62)
    pos = torch.tensor([8999, 1199], dtype=torch.int32)
    q = (torch.randn(2, 16, 128, generator=torch.Generator().manual_seed(63)) * 0.02).to(torch.bfloat16).cuda()
    outs = [check_attention(c, q, pos, table) for _ in range(3)]
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("rows_first", [False, True])
def test_offsets_beyond_32_bits(rows_first):
    """A pool of more than 2^32 elements per tensor: append, attention and read at its far end."""
    nkv, page, hd = 8, 64, 128
    n_pages = (1 << 32) // (nkv * page * hd) + 40
    shape = (n_pages, page, nkv, hd) if rows_first else (n_pages, nkv, page, hd)
    k, v = (torch.empty(shape, dtype=torch.uint8, device="cuda") for _ in range(2))
    if rows_first:
        k, v = k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3)
    ke, ve = (torch.empty(n_pages, nkv, page, dtype=torch.uint8, device="cuda") for _ in range(2))
    cache = kl.PagedCache(k, v, ke, ve)
    table = i32([[n_pages - 1, n_pages - 2, n_pages - 7]])
    kr, vr = rows_like(150, nkv, hd, torch.bfloat16, 71)
    kl.kl_paged_append(cache, kr, vr, i32([0]), table, row_starts=i32([0, 150]))
    ko, vo = (torch.zeros(150, nkv, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kl.kl_paged_read(cache, ko, vo, i32([0]), table, row_starts=i32([0, 150]))
    small = kl.PagedCache.allocate(3, nkv, page, hd, kl.KL_KV_E4M3)
    near = i32([[2, 0, 1]])
    kl.kl_paged_append(small, kr, vr, i32([0]), near, row_starts=i32([0, 150]))
    k2, v2 = torch.zeros_like(ko), torch.zeros_like(vo)
    kl.kl_paged_read(small, k2, v2, i32([0]), near, row_starts=i32([0, 150]))
    same = torch.equal(ko, k2) and torch.equal(vo, v2)
    assert same
    # half a step of e4m3: 2^-4 of a number, or 2^-10 of the row's scale below the smallest normal one; the scale is less
    # than the row's largest magnitude / 224
    x = kr.float()
    close = (ko.float() - x).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -10 / 224 * x.abs().amax(2, keepdim=True)
    assert bool(close.all())
    q = torch.randn(1, 32, hd, device="cuda").to(torch.bfloat16)
    ws = torch.empty(kl.kl_paged_workspace_bytes(cache, 32, 1, 3), dtype=torch.uint8, device="cuda")
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    kl.kl_paged_attention(cache, q, a, i32([149]), table, ws)
    kl.kl_paged_attention(small, q, b, i32([149]), near, ws)
    torch.cuda.synchronize()
    same = torch.equal(a, b)
    assert same and a.abs().max().item() > 0


# ---- selection

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hd,nq,nkv,page,n_select,keep", [(128, 32, 8, 16, 5, (1, 1)), (64, 6, 2, 4, 1, (0, 0)), (256, 12, 1, 64, 17, (0, 3)),
                                                          (128, 20, 2, 8, 300, (2, 2)), (64, 8, 8, 16, 2, (1, 1))])
@pytest.mark.parametrize("ties", [False, True])
def test_select(dtype, hd, nq, nkv, page, n_select, keep, ties):
    positions = [page * 300 - 1, 0, -1, page * 17 + 1, page, page * 999 + 2, n_select * page - 1, n_select * page]
    counts = [p // page + 1 if p >= 0 else 0 for p in positions]
    n_pages = sum(counts)
    table = ref.scattered_table([p + 1 for p in positions], page, n_pages, seed=81)
    g = torch.Generator().manual_seed(82)
    b = torch.randn(n_pages, nkv, 2, hd, generator=g)
    q = torch.randn(len(positions), nq, hd, generator=g)
    if ties:   # whole numbers: many pages of exactly equal scores
        b, q = b.sign(), (q * 0.7).round()
    b = b.sort(2).values.to(torch.bfloat16)
    q = q.to(dtype)
    cache = kl.PagedCache(None, None, bounds=b.cuda(), page_size=page, kv_type=kl.KL_KV_BF16)
    ws = torch.empty(kl.kl_paged_workspace_bytes(cache, nq, len(positions), table.shape[1]), dtype=torch.uint8, device="cuda").fill_(0xff)
    got = torch.full((len(positions), nkv, n_select), 99, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kl.kl_paged_select(cache, q.cuda(), i32(positions), table.cuda(), got, ws, keep_first=keep[0], keep_last=keep[1], status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    want = ref.select_ref(b, q, positions, table, page, keep[0], keep[1], n_select)
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("q_power,b_power", [(-124, 0), (-130, 20), (-118, 100), (-60, -70), (-75, -75), (100, 20), (0, -133)])
def test_select_at_the_ends_of_the_exponents(dtype, q_power, b_power):
    """Queries, bounds and products that 16-bit halves or 32-bit sums cannot hold."""
    hd, nq, nkv, page, n_select, count = 128, 8, 2, 16, 20, 300
    g = torch.Generator().manual_seed(86)
    b = (torch.randn(count, nkv, 2, hd, generator=g) * 2.0 ** (b_power // 2) * 2.0 ** (b_power - b_power // 2)).sort(2).values.to(torch.bfloat16)
    q = (torch.randn(1, nq, hd, generator=g) * 2.0 ** (q_power // 2) * 2.0 ** (q_power - q_power // 2)).to(dtype)
    table = ref.scattered_table([count * page], page, count, seed=87)
    cache = kl.PagedCache(None, None, bounds=b.cuda(), page_size=page, kv_type=kl.KL_KV_BF16)
    ws = torch.empty(kl.kl_paged_workspace_bytes(cache, nq, 1, table.shape[1]), dtype=torch.uint8, device="cuda").fill_(0xff)
    got = torch.full((1, nkv, n_select), 99, dtype=torch.int32, device="cuda")
    kl.kl_paged_select(cache, q.cuda(), i32([count * page - 1]), table.cuda(), got, ws, keep_first=0, keep_last=0)
    torch.cuda.synchronize()
    assert torch.equal(got.cpu(), ref.select_ref(b, q, [count * page - 1], table, page, 0, 0, n_select))


def test_select_long_table():
    """More pages than one block keeps in registers, infinite bounds, NaN bounds and -0."""
    page, hd, n_pages = 4, 64, 40000
    g = torch.Generator().manual_seed(91)
    b = torch.randn(n_pages, 1, 2, hd, generator=g).sort(2).values
    b[100, 0, 1, 3] = math.inf
    b[200, 0, 0, 7] = math.nan
    b[300] = -0.0
    b[301] = 0.0
    b = b.to(torch.bfloat16)
    q = torch.randn(2, 2, hd, generator=g).abs().to(torch.bfloat16)
    q[1] = -q[1]
    positions = [n_pages * page - 2, 33000 * page]
    table = torch.stack([torch.randperm(n_pages, generator=g), torch.randperm(n_pages, generator=g)]).to(torch.int32)
    cache = kl.PagedCache(None, None, bounds=b.cuda(), page_size=page, kv_type=kl.KL_KV_E4M3)
    ws = torch.empty(kl.kl_paged_workspace_bytes(cache, 2, 2, n_pages), dtype=torch.uint8, device="cuda")
    got = torch.zeros(2, 1, 1000, dtype=torch.int32, device="cuda")
    kl.kl_paged_select(cache, q.cuda(), i32(positions), table.cuda(), got, ws, keep_first=0, keep_last=1)
    torch.cuda.synchronize()
    assert torch.equal(got.cpu(), ref.select_ref(b, q, positions, table, page, 0, 1, 1000))


# ---- errors seen on the device

def test_bad_pages_and_positions_set_the_status_word():
    c = ref.Cache(6, 2, 16, 128, True, bounds=True, seed=101)
    q = torch.randn(1, 4, 128).cuda()
    out = torch.zeros_like(q)
    ws = torch.empty(kl.kl_paged_workspace_bytes(c.handle, 4, 1, 3), dtype=torch.uint8, device="cuda")
    sel = torch.zeros(1, 2, 2, dtype=torch.int32, device="cuda")
    k, v = rows_like(3, 2, 128, torch.bfloat16, 102)
    good, starts = i32([[0, 1, 2]]), i32([0, 3])

    def calls(pos, table, st, row_starts=starts):
        yield lambda: kl.kl_paged_append(c.handle, k, v, pos, table, row_starts=row_starts, status=st)
        yield lambda: kl.kl_paged_read(c.handle, torch.zeros(3, 2, 128, device="cuda"), torch.zeros(3, 2, 128, device="cuda"), pos, table,
                                       row_starts=row_starts, status=st)
        yield lambda: kl.kl_paged_attention(c.handle, q, out, pos, table, ws, status=st)
        yield lambda: kl.kl_paged_select(c.handle, q, pos, table, sel, ws, status=st)

    cases = [(i32([40]), i32([[0, 1, 6]]), starts), (i32([40]), i32([[0, 1, -1]]), starts), (i32([48]), good, starts),
             (i32([2 ** 31 - 1]), good, starts)]
    for pos, table, rs in cases:
        for i in range(4):
            st = torch.zeros(1, dtype=torch.int32, device="cuda")
            list(calls(pos, table, st, rs))[i]()
            torch.cuda.synchronize()
            assert st.item() == kl.KL_ERR_OUT_OF_RANGE, (pos, table, i)
    for rs in (i32([0, 4]), i32([2, 1]), i32([-1, 3])):
        for i in range(2):
            st = torch.zeros(1, dtype=torch.int32, device="cuda")
            list(calls(i32([0]), good, st, rs))[i]()
            torch.cuda.synchronize()
            assert st.item() == kl.KL_ERR_OUT_OF_RANGE, (rs, i)
    # sticky: nothing happens until the caller clears the word
    st = i32([kl.KL_ERR_OUT_OF_RANGE])
    before = [t.clone() for t in (c.k, c.v, c.ke, c.ve, c.bounds, out, sel)]
    for f in calls(i32([4]), good, st):
        f()
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, (c.k, c.v, c.ke, c.ve, c.bounds, out, sel)))
    st.zero_()
    for f in calls(i32([4]), good, st):
        f()
    torch.cuda.synchronize()
    assert st.item() == 0 and bool(out.abs().max() > 0)


# ---- as they are used together

@pytest.mark.parametrize("e4m3", [False, True])
def test_a_generation_with_all_of_them(e4m3):
    """A prompt goes in, then twenty tokens: append, select, attention over the chosen pages, on a stream of its own."""
    nkv, G, hd, page, n_select = 2, 4, 128, 4, 6
    lengths = [30, 3, 57]
    c = ref.Cache(60, nkv, page, hd, e4m3, bounds=True, seed=111)
    steps = 20
    table = ref.scattered_table([n + steps for n in lengths], page, 60, seed=112)
    starts = [0, 30, 33, 90]
    k, v = rows_like(90, nkv, hd, torch.bfloat16, 113)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    tab = table.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(kl.kl_paged_workspace_bytes(c.handle, nkv * G, 3, table.shape[1]), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    kl.kl_paged_append(c.handle, k, v, i32([0, 0, 0]), tab, row_starts=i32(starts), status=status, stream=st)
    sel = torch.zeros(3, nkv, n_select, dtype=torch.int32, device="cuda")
    for t in range(steps):
        kn, vn = rows_like(3, nkv, hd, torch.bfloat16, 200 + t)
        q = torch.randn(3, nkv * G, hd, generator=torch.Generator().manual_seed(300 + t)).to(torch.bfloat16).cuda()
        pos = torch.tensor([n + t for n in lengths], dtype=torch.int32)
        out, pd = torch.zeros_like(q), pos.cuda()
        torch.cuda.synchronize()
        kl.kl_paged_append(c.handle, kn, vn, pd, tab, status=status, stream=st)
        kl.kl_paged_select(c.handle, q, pd, tab, sel, ws, status=status, stream=st)
        kl.kl_paged_attention(c.handle, q, out, pd, tab, ws, selected=sel, status=status, stream=st)
        st.synchronize()
        assert status.item() == 0
        # the bounds are those of the pages' contents
        held = c.values("k")
        for s in range(3):
            for lp in range(int(pos[s]) // page + 1):
                rows = held[int(table[s, lp]), :, :min(page, int(pos[s]) + 1 - lp * page)]
                b = c.bounds[int(table[s, lp])].cpu().double()
                assert torch.equal(b[:, 0], rows.amin(1)) and torch.equal(b[:, 1], rows.amax(1))
        want_sel = ref.select_ref(c.bounds.cpu(), q.cpu(), pos.tolist(), table, page, 1, 1, n_select)
        assert torch.equal(sel.cpu(), want_sel)
        want, _, mass, reach = ref.attention_ref(held, c.values("v"), q.cpu(), pos.tolist(), table, page, 1 / math.sqrt(hd), 0, want_sel)
        tol = 2.0 ** -8 * want.abs() + (2 * (reach * (hd + 8) * 2.0 ** -24 + 2.0 ** -21 + 2.0 ** -16)[..., None] + 100 * 2.0 ** -24) * mass + 1e-30
        assert bool(((out.cpu().double() - want).abs() <= tol).all())


def test_captured_and_replayed():
    """A step captured once and replayed as the positions advance on the device; a second graph on a workspace of its own
    replayed on another stream at the same time gives its own results."""
    nkv, nq, hd, page = 2, 8, 128, 16
    graphs = []
    for i in range(2):
        c = ref.Cache(300, nkv, page, hd, i == 1, bounds=True, seed=121 + i)
        table = ref.scattered_table([2000, 700], page, 300, seed=123)
        x = dict(c=c, table=table, tab=table.cuda(), pos=i32([1500, 30]), q=torch.zeros(2, nq, hd, dtype=torch.bfloat16, device="cuda"),
                 kr=torch.zeros(2, nkv, hd, dtype=torch.bfloat16, device="cuda"), vr=torch.zeros(2, nkv, hd, dtype=torch.bfloat16, device="cuda"),
                 out=torch.zeros(2, nq, hd, dtype=torch.bfloat16, device="cuda"), sel=torch.zeros(2, nkv, 20, dtype=torch.int32, device="cuda"),
                 ws=torch.empty(kl.kl_paged_workspace_bytes(c.handle, nq, 2, table.shape[1]), dtype=torch.uint8, device="cuda"))

        def step(x=x):
            st = torch.cuda.current_stream()
            x["pos"] += 1
            kl.kl_paged_append(x["c"].handle, x["kr"], x["vr"], x["pos"], x["tab"], stream=st)
            kl.kl_paged_select(x["c"].handle, x["q"], x["pos"], x["tab"], x["sel"], x["ws"], stream=st)
            kl.kl_paged_attention(x["c"].handle, x["q"], x["out"], x["pos"], x["tab"], x["ws"], selected=x["sel"], stream=st)
        x["graph"] = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(x["graph"]):
            step()
        x["stream"] = torch.cuda.Stream()
        graphs.append(x)
    for t in range(4):
        for i, x in enumerate(graphs):
            g = torch.Generator().manual_seed(500 + 10 * t + i)
            for name in ("q", "kr", "vr"):
                x[name].copy_(torch.randn(x[name].shape, generator=g).mul_(0.1))
        torch.cuda.synchronize()
        for x in graphs:
            with torch.cuda.stream(x["stream"]):
                x["graph"].replay()
        torch.cuda.synchronize()
        for x in graphs:
            c, pos = x["c"], [1501 + t, 31 + t]
            assert x["pos"].tolist() == pos
            sel = ref.select_ref(c.bounds.cpu(), x["q"].cpu(), pos, x["table"], page, 1, 1, 20)
            assert torch.equal(x["sel"].cpu(), sel)
            want, _, mass, reach = ref.attention_ref(c.values("k"), c.values("v"), x["q"].cpu(), pos, x["table"], page, 1 / math.sqrt(hd), 0, sel)
            tol = 2.0 ** -8 * want.abs() + (2 * (reach * (hd + 8) * 2.0 ** -24 + 2.0 ** -21 + 2.0 ** -16)[..., None] + 400 * 2.0 ** -24) * mass + 1e-30
            assert bool(((x["out"].cpu().double() - want).abs() <= tol).all())
