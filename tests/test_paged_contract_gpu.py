"""Properties the paged operators promise beyond ordinary batches."""
import ctypes as C
import math

import pytest
import torch

from paper_2410_23668_b200 import binding as kl, build, inputs as gen
from tests import helpers, paged_ref as ref
from tests.test_paged_decode_gpu import Setup
from tests.test_paged_gpu import check_attention, i32, rows_like

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build_library()


def one_hot_rows(c, table, length, seed):
    """Keys with one column and values with one row that is not zero, powers of two: position p has its key in column p and
    its value in the columns d with d % length == p, so that every product sum of attention has a single term."""
    g = torch.Generator().manual_seed(seed)
    for x in (c.k, c.v):
        x.zero_()
    for p in range(length):
        phys, r = int(table[0, p // c.page]), p % c.page
        c.k[phys, :, r, p] = (2.0 ** torch.randint(-1, 1, (c.nkv,), generator=g)).to(torch.bfloat16).cuda()
        c.v[phys, :, r, p::length] = 1.0


@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("page", [4, 16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("reach", [0.125, 48.0])
def test_bf16_caches_keep_24_bits(hd, page, dtype, reach):
    """fp32 queries and the probabilities take part with 24 bits.  Tolerance, in units of 2^-24 of the result: with s the score
    (|s| <= reach), its three partial products are added with 2 each at most, the factor scale * log2(e) is rounded once and multiplied
    once: 8 |s|; the difference to the maximum, |s| log2(e) again at most twice as large: 2 |s|; a query in three parts leaves 1 |s|; the
    exponential 4; three parts of the probability added with 2 each: 6; numerator and denominator alike; N terms of the denominator, the
    reciprocal and the product N + 3.  bf16 outputs: half a step more, 2^-8."""
    n, nkv, G, scale = 2, 2, 16, reach
    c = ref.Cache(4, nkv, page, hd, False, seed=1)
    table = ref.scattered_table([n], page, 4, seed=2)
    one_hot_rows(c, table, n, 3)
    worst = 0.0
    for seed in range(8):
        q = ((torch.rand(1, nkv * G, hd, generator=torch.Generator().manual_seed(10 + seed)) * 2 - 1)).to(dtype).cuda()
        out = torch.zeros_like(q)
        ws = torch.empty(kl.kl_paged_workspace_bytes(c.handle, nkv * G, 1, table.shape[1]), dtype=torch.uint8, device="cuda")
        kl.kl_paged_attention(c.handle, q, out, i32([n - 1]), table.cuda(), ws, scale=scale)
        torch.cuda.synchronize()
        want = ref.attention_ref(c.values("k"), c.values("v"), q.cpu(), [n - 1], table, page, scale)[0]
        s = float(torch.tensor(scale, dtype=torch.float64))
        tol = ((2 * (11 * s + 4) + 6 + n + 3) * 2.0 ** -24 + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)) * want.abs() + 1e-37
        worst = max(worst, float(((out.cpu().double() - want).abs() / tol).max()))
    assert worst <= 1.0, worst


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd", [64, 128, 256])
def test_long_sums_on_bf16_caches_have_no_drift(hd, dtype):
    """Values that are all 1: the result is 1, however many tiles a warp adds up.  Additions to nearest have no direction; what is left
    is the 48 additions within a tile of 16 positions, single precision, half a unit off on average: 48 * 2^-24 of the mean of
    many results.  (Sums that are cut off instead lose half a unit per product and tile: 1.2e-5 here.)"""
    n, nkv, G, page, ctx = 32, 4, 4, 16, 65536
    g = torch.Generator(device="cuda").manual_seed(hd)
    k = torch.randn(ctx // page, nkv, page, hd, generator=g, device="cuda").to(torch.bfloat16)
    c = kl.PagedCache(k, torch.ones_like(k))
    table = torch.arange(ctx // page, dtype=torch.int32, device="cuda").expand(n, -1).contiguous()   # the sequences share their pages
    q = torch.randn(n, nkv * G, hd, generator=g, device="cuda").to(dtype)
    out = torch.zeros_like(q)
    ws = torch.empty(kl.kl_paged_workspace_bytes(c, nkv * G, n, ctx // page), dtype=torch.uint8, device="cuda")
    kl.kl_paged_attention(c, q, out, i32([ctx - 1] * n), table, ws)
    torch.cuda.synchronize()
    off = out.double() - 1
    if dtype == torch.bfloat16:   # rounded to 1 unless off by a quarter of the step below it
        assert bool((off == 0).all())
    else:
        assert abs(float(off.mean())) <= 48 * 2.0 ** -24, float(off.mean())


@pytest.mark.parametrize("e4m3,dtype,hd", [(False, torch.bfloat16, 128), (False, torch.float32, 64), (True, torch.bfloat16, 128), (True, torch.bfloat16, 64),
                                           (True, torch.float32, 256)])
@pytest.mark.parametrize("page", [4, 8, 16, 24])
@pytest.mark.parametrize("listed", [False, True])
def test_a_window_needs_no_pages_before_it(e4m3, dtype, hd, page, listed):
    """A program that slides a window along gives back the pages behind it: their table entries name no page."""
    nkv, nq, window = 2, 6, 50
    positions = [180 + i for i in range(0, 2 * page + 1, max(1, page // 8))] + [20, window - 1, window]
    lengths = [p + 1 for p in positions]
    n_pages = sum(-(-x // page) for x in lengths)
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, seed=1)
    table = ref.scattered_table(lengths, page, n_pages, seed=2)
    q = (torch.randn(len(positions), nq, hd, generator=torch.Generator().manual_seed(3)) * (0.02 if e4m3 else 1.0)).to(dtype).cuda()
    sel = None
    if listed:   # every page, those before the window among them
        sel = torch.arange(table.shape[1], dtype=torch.int32).expand(len(positions), nkv, -1).contiguous()
    first = torch.tensor([max(0, x - window) // page for x in lengths])
    gone = torch.arange(table.shape[1])[None, :] < first[:, None]
    assert gone.any()
    want = check_attention(c, q, torch.tensor(positions, dtype=torch.int32), table, window=window, selected=sel)
    got = check_attention(c, q, torch.tensor(positions, dtype=torch.int32), table.masked_fill(gone, -1), window=window, selected=sel)
    assert torch.equal(got, want)


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_window_that_blocks_share(e4m3):
    page, hd, nkv, nq, window = 16, 128, 2, 4, 5000
    positions = [19999, 31, 7000]
    lengths = [p + 1 for p in positions]
    n_pages = sum(-(-x // page) for x in lengths)
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, seed=4)
    table = ref.scattered_table(lengths, page, n_pages, seed=5)
    q = (torch.randn(3, nq, hd, generator=torch.Generator().manual_seed(6)) * (0.02 if e4m3 else 1.0)).to(torch.bfloat16).cuda()
    check_attention(c, q, torch.tensor(positions, dtype=torch.int32), table, window=window)


@pytest.mark.parametrize("static", [False, True])
def test_sampling_leaves_empty_slots_alone(static):
    shape, n = gen.TINY, 5
    logits = torch.randn(n, shape.vocab, generator=torch.Generator().manual_seed(1)).cuda()
    tok, pos = i32([7, 8, 9, 10, 11]), i32([3, -1, 0, -2 ** 31, 2 ** 20])
    dec = helpers.make_decoder(shape, n, 16, 0)
    for t in range(3):
        if static:
            kl.kl_argmax_advance_static(logits, tok, pos, n)
        else:
            dec.kl_argmax_advance(logits, tok, pos, n)
        torch.cuda.synchronize()
        best = logits.cpu().argmax(1).tolist()
        assert tok.tolist() == [best[0], 8, best[2], 10, best[4]]
        assert pos.tolist() == [4 + t, -1, 1 + t, -2 ** 31, 2 ** 20 + 1 + t]
    dec.close()


@pytest.mark.parametrize("fill", [-1, 0])
def test_replayed_steps_keep_empty_slots_empty(fill):
    """A capture of the step and the sampling, replayed: an empty slot stays one, whatever its row of the page table holds."""
    shape, contexts = gen.TINY, [30, -1, 12]
    a, b = (Setup(shape, contexts, 16, kl.KL_KV_E4M3, n_select=3) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    a.table[1] = fill
    b.table[1] = -1
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        st = torch.cuda.current_stream()
        a.step(stream=st)
        a.dec.kl_argmax_advance(a.logits, a.tok, a.pos, 3, stream=st)
    for t in range(4):
        graph.replay()
        b.step()
        b.dec.kl_argmax_advance(b.logits, b.tok, b.pos, 3)
        b.pos[1] = -1
        torch.cuda.synchronize()
        assert a.dec.kl_last_status() == 0 and b.dec.kl_last_status() == 0
        assert a.pos.tolist() == [31 + t, -1, 13 + t]
        for i in (0, 2):
            assert torch.equal(a.logits[i], b.logits[i]) and a.tok[i] == b.tok[i]
        for x, y in zip(a.caches, b.caches):
            assert all(torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for s, t in zip(x.tensors, y.tensors))
    del graph
    a.dec.close()
    b.dec.close()


def programmatic_edges(graph):
    """(edges, how many of them let a kernel start before the one in front of it has ended)"""
    cu = C.CDLL("libcuda.so.1")
    get = cu.cuGraphGetEdges_v2
    get.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(C.c_size_t)]
    n = C.c_size_t()
    assert get(graph.raw_cuda_graph(), None, None, None, C.byref(n)) == 0
    a, b = ((C.c_void_p * n.value)() for _ in range(2))
    data = (C.c_uint8 * (8 * n.value))()   # CUgraphEdgeData: the type is its third byte, 1 = programmatic
    assert get(graph.raw_cuda_graph(), a, b, data, C.byref(n)) == 0
    return n.value, sum(data[8 * i + 2] == 1 for i in range(n.value))


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("n_select", [0, 3])
def test_plain_stream_order_holds_for_the_whole_paged_step(wide, n_select):
    """kl_set_dependent_launch(0): every kernel of the step starts when the one before it has ended, those of the paged operators too."""
    shape, contexts = gen.TINY, [30, 12]
    s = Setup(shape, contexts, 16, kl.KL_KV_BF16, n_select)
    if wide:   # attention over all positions joins with a kernel of its own
        table = torch.full((2, 4096), -1, dtype=torch.int32, device="cuda")
        table[:, :s.table.shape[1]] = s.table
        s.table = table
        s.ws = torch.empty(s.dec.kl_paged_step_bytes(s.caches[0], 2, 4096, n_select), dtype=torch.uint8, device="cuda").fill_(0xff)
    made, logits = {}, {}
    torch.cuda.synchronize()
    for on in (True, False):
        s.dec.kl_set_dependent_launch(on)
        graph = torch.cuda.CUDAGraph(keep_graph=True)
        before = s.dec.kl_launch_count()
        with torch.cuda.graph(graph):
            s.step(stream=torch.cuda.current_stream())
        made[on] = s.dec.kl_launch_count() - before
        edges, early = programmatic_edges(graph)
        assert edges == made[on] - 1 and early == (edges if on else 0)
        graph.instantiate()
        graph.replay()
        torch.cuda.synchronize()
        assert s.dec.kl_last_status() == 0
        logits[on] = s.logits.clone()
        del graph
    assert made[True] == made[False] and torch.equal(logits[True], logits[False])
    s.dec.close()


def test_step_refuses_caches_of_the_host():
    s = Setup(gen.TINY, [30, 12], 16, kl.KL_KV_BF16)
    k = torch.zeros(4, gen.TINY.n_kv_heads, 16, gen.TINY.head_dim, dtype=torch.bfloat16)
    made = s.dec.kl_launch_count()
    for caches in ([kl.PagedCache(k, k.clone())] * gen.TINY.n_layers, s.caches[:-1] + [kl.PagedCache(k, k.clone())]):
        with pytest.raises(kl.KlError) as e:
            s.dec.kl_decode_step_paged(s.tok, s.pos, caches, s.table, s.logits, s.ws)
        assert e.value.code == kl.KL_ERR_INVALID_ARG
    assert s.dec.kl_launch_count() == made
    s.dec.close()


def test_bounds_hold_where_bf16_has_no_number():
    """e4m3 rows of the smallest scales stand for numbers that bf16 does not hold (down to 2^-136): their bounds are rounded outwards."""
    nkv, hd, page, n = 2, 64, 8, 13
    g = torch.Generator().manual_seed(1)
    x = torch.randn(n, 2, nkv, hd, generator=g) * 2.0 ** -134
    x[page:] *= 2.0 ** 20                                   # a page of scales that leave bf16 numbers only
    x[:, :, :, 0] = x[:, :, :, 0].sign() * 2.0 ** -124      # the largest of the first page's rows
    x = x.cuda()
    c = ref.Cache(3, nkv, page, hd, True, bounds=True, seed=2)
    table = ref.scattered_table([n + 5], page, 3, seed=3, extra=0)
    c.bounds.zero_()
    for k0, k1 in ((0, 4), (4, n)):   # a page goes on
        kl.kl_paged_append(c.handle, x[k0:k1, 0], x[k0:k1, 1], i32([k0]), table.cuda(), row_starts=i32([0, k1 - k0]))
    ko, vo = (torch.zeros(n, nkv, hd, device="cuda") for _ in range(2))
    kl.kl_paged_read(c.handle, ko, vo, i32([0]), table.cuda(), row_starts=i32([0, n]))
    torch.cuda.synchronize()
    inexact = 0
    for lp in range(2):
        phys = int(table[0, lp])
        held = c.values("k")[phys, :, :min(page, n - lp * page)]
        assert torch.equal(ko[lp * page:lp * page + held.shape[1]].cpu().double().transpose(0, 1), held)   # fp32 holds them all
        b = c.bounds[phys].cpu().double()
        lo, hi = held.amin(1), held.amax(1)
        assert bool((b[:, 0] <= lo).all()) and bool((b[:, 1] >= hi).all())
        step = 2.0 ** -133   # between the bf16 numbers at zero
        assert bool((lo - b[:, 0] < step).all()) and bool((b[:, 1] - hi < step).all())
        exact = (lo / step == (lo / step).round()) | (lo.abs() > 2.0 ** -120)
        assert torch.equal(b[:, 0][exact], lo[exact])
        inexact += int((~exact).sum())
    assert inexact > 50


SPREADS = ["one large, equal small ones", "one large, small ones of both signs", "falling by halves", "cancelling", "wide"]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("spread", SPREADS)
@pytest.mark.parametrize("power", [-20, -23, -25, -27])
def test_select_hard_spreads(dtype, hd, spread, power):
    """Pages whose scores differ only by terms that a 32-bit sum loses: the choice is that of the exact scores, and the scores the
    workspace holds ([n_seqs][n_kv_heads][pages] of score, bound) are off by no more than the bound beside them."""
    nkv, G, page, pages, n_select = 2, 3, 4, 300, 40
    g = torch.Generator().manual_seed(1000 * hd + 10 * SPREADS.index(spread) - power)
    c = ref.Cache(pages, nkv, page, hd, False, bounds=True, seed=1)
    q = torch.zeros(1, nkv * G, hd)
    b = torch.zeros(pages, nkv, hd)
    small = 2.0 ** power
    if spread == "one large, equal small ones":
        q[:] = small
        b[:] = (torch.rand(pages, nkv, hd, generator=g) < torch.rand(pages, nkv, 1, generator=g)).float()
    elif spread == "one large, small ones of both signs":
        q[:] = small * (1 + torch.rand(q.shape, generator=g))
        b[:] = torch.randint(-1, 2, b.shape, generator=g).float()
    elif spread == "falling by halves":
        q[:] = 2.0 ** -(torch.arange(hd) % 30).float() * torch.sign(torch.randn(q.shape, generator=g))
        b[:] = 1 + torch.rand(b.shape, generator=g) * small
    elif spread == "cancelling":
        q[:] = 1.0
        q[..., 1::2] = -1.0
        b[:] = 1.0 + 0.25 * torch.rand(pages, nkv, 1, generator=g)
        b[..., ::2] += torch.randint(0, 2, (pages, nkv, hd // 2), generator=g) * 2.0 ** -7
    else:
        q[:] = torch.randn(q.shape, generator=g) * torch.exp(4 * torch.randn(q.shape, generator=g))
        b[:] = torch.randn(b.shape, generator=g) * torch.exp(4 * torch.randn(b.shape, generator=g))
    if spread.startswith("one large"):
        at = int(torch.randint(0, hd, (1,), generator=g))
        q[..., at] = 1.0
        b[..., at] = 1.0
    q = q.to(dtype)
    b = b.to(torch.bfloat16)
    c.bounds.copy_(torch.stack([b, b], 2))   # lo = hi: the score is a plain product sum
    table = ref.scattered_table([pages * page], page, pages, seed=2)
    sel = torch.full((1, nkv, n_select), 9, dtype=torch.int32, device="cuda")
    ws = torch.empty(kl.kl_paged_workspace_bytes(c.handle, nkv * G, 1, table.shape[1]), dtype=torch.uint8, device="cuda").fill_(0xff)
    kl.kl_paged_select(c.handle, q.cuda(), i32([pages * page - 1]), table.cuda(), sel, ws)
    torch.cuda.synchronize()
    assert torch.equal(sel.cpu(), ref.select_ref(c.bounds.cpu(), q, [pages * page - 1], table, page, 1, 1, n_select))
    held = ws[:nkv * table.shape[1] * 8].view(torch.float32).view(nkv, table.shape[1], 2)[:, :pages].cpu().double()
    v = b[table[0, :pages].long()].double()
    exact = torch.stack([torch.einsum("gd,pd->gp", q[0, h * G:(h + 1) * G].double(), v[:, h]).amax(0) for h in range(nkv)])
    off = (held[..., 0] - exact).abs() / held[..., 1]
    assert bool((off <= 1.0).all()), float(off.max())
    reach = torch.stack([torch.einsum("gd,pd->gp", q[0, h * G:(h + 1) * G].double().abs(), v[:, h].abs()).amax(0) for h in range(nkv)])
    # hd / 16 products of 16 terms for lo and as many for hi (fp32 queries: twice), each addition off by a unit of 32 bits at most
    need = hd * 2.0 ** -22 if dtype == torch.bfloat16 else hd * 2.0 ** -21 + 2.0 ** -16
    assert bool((held[..., 1] >= need * reach).all())


def test_step_refuses_more_pages_than_a_list_can_name():
    """Refused before anything is launched, whatever the workspace claims to hold."""
    s = Setup(gen.TINY, [30, 12], 16, kl.KL_KV_BF16, 3)
    layers = (kl.PagedCacheDesc * len(s.caches))(*(c.desc for c in s.caches))
    made = s.dec.kl_launch_count()
    for n_select in (1, 2 ** 31, 2 ** 32 - 1):
        rc = kl.lib().kl_decode_step_paged(s.dec.handle, s.tok.data_ptr(), s.pos.data_ptr(), C.addressof(layers), s.table.data_ptr(), s.table.stride(0),
                                           s.table.shape[1], n_select, s.logits.data_ptr(), 2, s.ws.data_ptr(), 1 << 62, None)
        assert rc == kl.KL_ERR_INVALID_ARG
    assert s.dec.kl_launch_count() == made
    s.dec.close()


@pytest.mark.parametrize("e4m3", [False, True])
def test_sequences_share_the_pages_of_a_prefix(e4m3):
    """Three sequences with the same first pages: read, select and attention see the prefix in each, append writes their own pages."""
    page, hd, nkv, nq, prefix, own = 16, 128, 2, 8, 8, [3, 1, 5]
    lengths = [(prefix + x) * page - 5 for x in own]
    n_pages = prefix + sum(own)
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, bounds=True, seed=1)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(2)).to(torch.int32)
    table = torch.full((3, prefix + max(own)), -1, dtype=torch.int32)
    table[:, :prefix] = order[:prefix]
    at = prefix
    for s, x in enumerate(own):
        table[s, prefix:prefix + x] = order[at:at + x]
        at += x
    tab = table.cuda()
    k, v = rows_like(prefix * page, nkv, hd, torch.bfloat16, 3)
    kl.kl_paged_append(c.handle, k, v, i32([0]), tab[:1].contiguous(), row_starts=i32([0, prefix * page]))
    shared = [t[order[:prefix].long().cuda()].view(torch.uint8).clone() for t in (c.k, c.v, c.bounds)]
    starts = [0]
    for x in lengths:
        starts.append(starts[-1] + x - prefix * page)
    k, v = rows_like(starts[-1], nkv, hd, torch.bfloat16, 4)
    kl.kl_paged_append(c.handle, k, v, i32([prefix * page] * 3), tab, row_starts=i32(starts))
    torch.cuda.synchronize()
    assert all(torch.equal(x, t[order[:prefix].long().cuda()].view(torch.uint8)) for x, t in zip(shared, (c.k, c.v, c.bounds)))
    pos = [x - 1 for x in lengths]
    q = (torch.randn(3, nq, hd, generator=torch.Generator().manual_seed(5)) * 0.2).to(torch.bfloat16).cuda()
    check_attention(c, q, torch.tensor(pos, dtype=torch.int32), table)
    sel = torch.zeros(3, nkv, 6, dtype=torch.int32, device="cuda")
    ws = torch.empty(kl.kl_paged_workspace_bytes(c.handle, nq, 3, table.shape[1]), dtype=torch.uint8, device="cuda")
    kl.kl_paged_select(c.handle, q, i32(pos), tab, sel, ws)
    torch.cuda.synchronize()
    want = ref.select_ref(c.bounds.cpu(), q.cpu(), pos, table, page, 1, 1, 6)
    assert torch.equal(sel.cpu(), want)
    check_attention(c, q, torch.tensor(pos, dtype=torch.int32), table, selected=want)
    n = prefix * page
    ko, vo = (torch.zeros(3 * n, nkv, hd, device="cuda") for _ in range(2))
    kl.kl_paged_read(c.handle, ko, vo, i32([0, 0, 0]), tab, row_starts=i32([0, n, 2 * n, 3 * n]))
    torch.cuda.synchronize()
    for got, held in ((ko, c.values("k")), (vo, c.values("v"))):
        rows = held[order[:prefix].long()].transpose(1, 2).reshape(n, nkv, hd)
        assert torch.equal(got.cpu().double(), rows.repeat(3, 1, 1))


@pytest.mark.parametrize("n_select", [0, 3])
def test_steps_on_a_shared_prefix_equal_steps_on_copies(n_select):
    """Two sequences that share the pages of a prefix, and the same two with a copy of it each: the same logits, bit for bit."""
    shape, page, prefix = gen.TINY, 16, 3
    logits = []
    for shared in (False, True):
        s = Setup(shape, [prefix * page + 5, prefix * page + 2], page, kl.KL_KV_E4M3, n_select)
        for c in s.caches:   # the second sequence's prefix is the first one's
            for t in c.tensors:
                t.view(torch.uint8)[s.table[1, :prefix].long()] = t.view(torch.uint8)[s.table[0, :prefix].long()]
        if shared:
            s.table[1, :prefix] = s.table[0, :prefix]
        run = []
        for t in range(3):
            s.step()
            torch.cuda.synchronize()
            assert s.dec.kl_last_status() == 0
            run.append(s.logits.clone())
            s.dec.kl_argmax_advance(s.logits, s.tok, s.pos, 2)
        logits.append(run)
        s.dec.close()
    assert all(torch.equal(x, y) for x, y in zip(*logits))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows", [torch.bfloat16, torch.float32])
def test_rows_of_700_sequences(e4m3, rows):
    """More sequences than a block of append or read holds at once, some without rows, some of them empty slots."""
    nkv, hd, page, n = 2, 64, 8, 700
    g = torch.Generator().manual_seed(1)
    cnt = torch.randint(0, 12, (n,), generator=g).tolist()
    pos = torch.randint(0, 20, (n,), generator=g).tolist()
    for s in range(0, n, 7):
        pos[s] = -1
    cnt[:3], cnt[-3:] = [0, 0, 5], [0, 9, 0]
    starts = [2]   # rows in front of the first sequence
    for x in cnt:
        starts.append(starts[-1] + x)
    total = starts[-1] + 3
    lengths = [max(p, 0) + x if p >= 0 else 0 for p, x in zip(pos, cnt)]
    n_pages = sum(-(-x // page) for x in lengths)
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, bounds=True, seed=2)
    table = ref.scattered_table(lengths, page, n_pages, seed=3)
    before = {x: getattr(c, x).cpu().clone() for x in ("k", "v", "ke", "ve", "bounds") if getattr(c, x) is not None}
    k, v = rows_like(total, nkv, hd, rows, 4)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kl.kl_paged_append(c.handle, k, v, i32(pos), table.cuda(), row_starts=i32(starts), status=status)
    torch.cuda.synchronize()
    seq = torch.tensor([s for s in range(n) for _ in range(cnt[s] if pos[s] >= 0 else 0)])
    row = torch.tensor([starts[s] + i for s in range(n) for i in range(cnt[s] if pos[s] >= 0 else 0)])
    at = torch.tensor([pos[s] + i for s in range(n) for i in range(cnt[s] if pos[s] >= 0 else 0)])
    phys, off = table[seq, at // page].long(), at % page
    expected = {}
    for which, x in (("k", k), ("v", v)):
        x = x.cpu()[row]
        if e4m3:
            y = x.double()
            e = torch.tensor([ref.row_exponent(float(m)) for m in y.abs().amax(-1).flatten()]).view(len(row), nkv)
            held = ref.e4m3_round(y * torch.pow(torch.tensor(2.0, dtype=torch.float64), -e)[..., None]) * torch.pow(torch.tensor(2.0, dtype=torch.float64), e)[..., None]
            before[which + "e"][phys, :, off] = (e + 127).to(torch.uint8)
            assert torch.equal(getattr(c, which + "e").cpu(), before[which + "e"])
        else:
            held = x.to(torch.bfloat16).double()
        expected[which] = held
        assert torch.equal(c.values(which)[phys, :, off], held)
        rest = torch.ones(n_pages, page, dtype=torch.bool)
        rest[phys, off] = False
        for t, old in ((getattr(c, which), before[which]),):
            assert torch.equal(t.cpu().view(torch.uint8).transpose(1, 2)[rest], old.view(torch.uint8).transpose(1, 2)[rest])
    b = before["bounds"].double()
    for i in range(len(row)):
        p, y = int(phys[i]), expected["k"][i]
        if off[i] == 0:
            b[p, :, 0], b[p, :, 1] = math.inf, -math.inf
        b[p, :, 0], b[p, :, 1] = torch.minimum(b[p, :, 0], y), torch.maximum(b[p, :, 1], y)
    assert torch.equal(c.bounds.cpu().double(), b)
    for out_type in (torch.bfloat16, torch.float32):
        ko, vo = (torch.full((total, nkv, hd), 5.0, dtype=out_type, device="cuda") for _ in range(2))
        kl.kl_paged_read(c.handle, ko, vo, i32(pos), table.cuda(), row_starts=i32(starts), status=status)
        torch.cuda.synchronize()
        for which, o in (("k", ko), ("v", vo)):
            want = torch.full((total, nkv, hd), 5.0, dtype=torch.float64)
            want[row] = expected[which]
            assert torch.equal(o.cpu().double(), want)
    assert status.item() == 0


def test_attention_of_a_batch_in_another_order():
    """More sequences than blocks of the grid, in two orders: each is right, and equal calls give equal bits."""
    page, hd, nkv, nq, n = 16, 64, 2, 8, 500
    g = torch.Generator().manual_seed(51)
    lengths = [int(x) for x in torch.randint(0, 120, (n,), generator=g)]
    n_pages = sum(-(-x // page) for x in lengths)
    c = ref.Cache(n_pages, nkv, page, hd, False, seed=52)
    table = ref.scattered_table(lengths, page, n_pages, seed=53)
    q = torch.randn(n, nq, hd, generator=g).cuda()
    pos = torch.tensor(lengths, dtype=torch.int32) - 1
    for order in (torch.arange(n), torch.randperm(n, generator=g)):
        a, b = (check_attention(c, q[order.cuda()].contiguous(), pos[order], table[order].contiguous()) for _ in range(2))
        assert torch.equal(a, b)


def test_append_and_attention_on_a_stream_of_their_own():
    """Rows, positions and tables stay alive until the stream has read them: what is written is what was handed in."""
    page, hd, nkv, nq = 8, 128, 2, 8
    lengths = [30, 3, 57]
    c = ref.Cache(20, nkv, page, hd, True, bounds=True, seed=1)
    table = ref.scattered_table(lengths, page, 20, seed=2)
    starts, zero, tab = i32([0, 30, 33, 90]), i32([0, 0, 0]), table.cuda()
    k, v = rows_like(90, nkv, hd, torch.bfloat16, 3)
    q = (torch.randn(3, nq, hd, generator=torch.Generator().manual_seed(4)) * 0.2).to(torch.bfloat16).cuda()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    kl.kl_paged_append(c.handle, k, v, zero, tab, row_starts=starts, stream=st)
    st.synchronize()
    for s in range(3):
        for i in range(lengths[s]):
            got = c.k[int(table[s, i // page]), :, i % page].cpu()
            for h in range(nkv):
                x = k[int([0, 30, 33][s]) + i, h].cpu().double()
                assert torch.equal(ref.e4m3_values(got[h]), ref.e4m3_round(x * 2.0 ** -ref.row_exponent(float(x.abs().max()))))
    check_attention(c, q, torch.tensor(lengths, dtype=torch.int32) - 1, table, stream=st)
