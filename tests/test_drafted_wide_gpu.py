"""The operators for drafted tokens, and sampling, where sizes, addresses or company are unusual: pools and logits beyond 32 bits of
elements, calls at the same time, pages that sequences share, thousands of sequences, groups of many query heads, long runs of tokens.
Tolerances are those of the files whose checks are used."""
import numpy as np
import pytest
import torch

from paper_2410_23668_b200 import binding as kl, build
from tests import paged_ref as ref
from tests.test_drafted_gpu import check_tree, freqs, i32, starts_of
from tests.test_sample_gpu import one_row

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build_library()


@pytest.mark.parametrize("e4m3", [False, True])
def test_pools_beyond_32_bits_give_the_same_bits(e4m3):
    nkv, nq, page, hd, many = 4, 8, 16, 128, 600_000   # 4.9e9 elements
    seqs = [(300, 5), (0, 3), (1000, 9)]
    lengths = [b + t for b, t in seqs]
    small = ref.Cache(90, nkv, page, hd, e4m3, seed=1)
    table = ref.scattered_table(lengths, page, 90, seed=2)
    far = many - 90
    k, v = (torch.empty(many, nkv, page, hd, dtype=small.k.dtype, device="cuda") for _ in range(2))
    ke, ve = (torch.empty(many, nkv, page, dtype=torch.uint8, device="cuda") if e4m3 else None for _ in range(2))
    for to, of in ((k, small.k), (v, small.v), (ke, small.ke), (ve, small.ve)):
        if to is not None:
            to[far:] = of
    big = kl.PagedCache(k, v, ke, ve, None)
    far_table = torch.where(table >= 0, table + far, table)
    g = torch.Generator().manual_seed(3)
    n = sum(t for _, t in seqs)
    kr, vr = (torch.randn(n, nkv, hd, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.randn(n, nq, hd, generator=g).to(torch.bfloat16).cuda()
    ws = torch.empty(kl.kl_paged_tree_workspace_bytes(big, nq), dtype=torch.uint8, device="cuda")
    got = []
    for c, t in ((small.handle, table), (big, far_table)):
        qo, out, status = torch.zeros_like(q), torch.zeros_like(q), i32([0])
        args = (i32([b for b, _ in seqs]), t.cuda())
        kl.kl_paged_append_rotated(c, kr, vr, *args, freqs(hd).cuda(), row_starts=i32(starts_of(seqs)), q=q, q_out=qo, status=status)
        kl.kl_paged_tree_attention(c, qo, out, *args, ws, row_starts=i32(starts_of(seqs)), status=status)
        assert status.item() == 0
        got.append((qo, out))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and bool(got[0][1].isfinite().all())
    for to, of in ((k, small.k), (v, small.v), (ke, small.ke), (ve, small.ve)):
        if to is not None:
            assert torch.equal(to[far:].view(torch.uint8), of.contiguous().view(torch.uint8))


def test_logits_beyond_32_bits():
    vocab, stride, n = 5000, 1_100_000_000, 3
    space = torch.empty((n - 1) * stride + vocab, device="cuda")
    x = space.as_strided((n, vocab), (stride, 1))
    r = np.random.default_rng(4)
    rows = (r.standard_normal((n, vocab)) * 2).astype(np.float32)
    x.copy_(torch.from_numpy(rows))
    u = r.random(n).astype(np.float32)
    tokens = i32([-5] * n)
    kl.kl_sample(x, torch.from_numpy(u).cuda(), tokens, top_p=torch.full((n,), 0.9, device="cuda"))
    for i in range(n):
        want, _, near = one_row(rows[i], u[i], p=0.9)
        assert near > 2.0 ** -43 and int(tokens[i]) == want


@pytest.mark.parametrize("e4m3", [False, True])
def test_calls_at_the_same_time(e4m3):
    """Two streams, a workspace each, one cache: every call gives what it gives alone."""
    nkv, nq, page, hd = 4, 16, 16, 128
    sets = [[(2000, 7), (900, 3)], [(1500, 2), (33, 30), (700, 1)]]
    lengths = [b + t for s in sets for b, t in s]
    n_pages = sum(-(-x // page) for x in lengths) + 1
    c = ref.Cache(n_pages, nkv, page, hd, e4m3, seed=5)
    tables = ref.scattered_table(lengths, page, n_pages, seed=6)
    tables = [tables[:2].cuda(), tables[2:].cuda()]
    g = torch.Generator().manual_seed(7)
    q = [torch.randn(sum(t for _, t in s), nq, hd, generator=g).to(torch.bfloat16).cuda() for s in sets]
    at = [(i32([b for b, _ in s]), i32(starts_of(s))) for s in sets]
    logits = torch.randn(40, 50000, generator=g).cuda()
    u = [torch.rand(40, generator=g).cuda() for _ in sets]
    ws = [torch.empty(kl.kl_paged_tree_workspace_bytes(c.handle, nq), dtype=torch.uint8, device="cuda") for _ in sets]

    def step(i, out, tokens, stream=None):
        kl.kl_paged_tree_attention(c.handle, q[i], out, at[i][0], tables[i], ws[i], row_starts=at[i][1], stream=stream)
        kl.kl_sample(logits, u[i], tokens, stream=stream)

    alone = []
    for i in range(2):
        alone.append((torch.zeros_like(q[i]), torch.zeros(40, dtype=torch.int32, device="cuda")))
        step(i, *alone[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[(torch.zeros_like(q[i]), torch.zeros(40, dtype=torch.int32, device="cuda")) for _ in range(20)] for i in range(2)]
    torch.cuda.synchronize()
    for k in range(20):
        for i in range(2):
            step(i, *got[i][k], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for out, tokens in got[i]:
            assert torch.equal(out, alone[i][0]) and torch.equal(tokens, alone[i][1])


@pytest.mark.parametrize("e4m3", [False, True])
def test_sequences_that_share_their_first_pages(e4m3):
    seqs = [(200, 6), (200, 6), (137, 9)]
    c = ref.Cache(40, 2, 16, 128, e4m3, seed=8)
    table = ref.scattered_table([b + t for b, t in seqs], 16, 40, seed=9)
    table[1, :12] = table[0, :12]
    table[2, :8] = table[0, :8]
    q = torch.randn(21, 8, 128, generator=torch.Generator().manual_seed(10)).to(torch.bfloat16).cuda()
    check_tree(c, q, seqs, table, "tree", seed=11)


@pytest.mark.parametrize("e4m3,hd", [(False, 128), (True, 64), (False, 256)])
def test_thousands_of_sequences(e4m3, hd):
    g = np.random.default_rng(12)
    seqs = [(-1 if i % 17 == 3 else int(g.integers(0, 40)), 1) for i in range(3000)]
    lengths = [max(b, 0) + 1 for b, _ in seqs]
    n_pages = sum(-(-x // 8) for x in lengths) + 1
    c = ref.Cache(n_pages, 1, 8, hd, e4m3, seed=13)
    table = ref.scattered_table(lengths, 8, n_pages, seed=14)
    q = torch.randn(3000, 2, hd, generator=torch.Generator().manual_seed(15)).to(torch.bfloat16).cuda()
    check_tree(c, q, seqs, table, "causal", single=True)


@pytest.mark.parametrize("e4m3,hd,nq,seqs", [(False, 128, 300, [(200, 3), (5, 1)]), (True, 128, 600, [(150, 2)]), (False, 256, 130, [(90, 3)]), (False, 64, 71, [(300, 9)])])
def test_groups_of_many_heads(e4m3, hd, nq, seqs):
    c = ref.Cache(40, 1, 16, hd, e4m3, seed=16)
    table = ref.scattered_table([b + t for b, t in seqs], 16, 40, seed=17)
    n = sum(t for _, t in seqs)
    q = torch.randn(n, nq, hd, generator=torch.Generator().manual_seed(18)).to(torch.bfloat16).cuda()
    check_tree(c, q, seqs, table, "tree", seed=19)


@pytest.mark.parametrize("e4m3,hd,window", [(False, 64, 0), (True, 128, 0), (False, 128, 700)])
def test_a_long_run_of_tokens(e4m3, hd, window):
    seqs = [(100, 1500), (0, 400)]
    c = ref.Cache(140, 1, 16, hd, e4m3, seed=20)
    table = ref.scattered_table([b + t for b, t in seqs], 16, 140, seed=21)
    q = torch.randn(1900, 2, hd, generator=torch.Generator().manual_seed(22)).to(torch.bfloat16).cuda()
    check_tree(c, q, seqs, table, "causal", window=window, sinks=4 if window else 0)


@pytest.mark.parametrize("e4m3,hd,nq,seed", [(False, 128, 8, 0), (True, 128, 8, 1), (False, 64, 16, 2), (True, 256, 8, 3), (False, 128, 12, 4)])
def test_units_of_one_and_of_two_runs_of_rows(e4m3, hd, nq, seed):
    """Tokens times heads on either side of 128 and 256, next to one another, so that shares begin inside units of either kind."""
    g = np.random.default_rng(seed)
    G = nq // 2
    around = [max(1, x // G + d) for x in (32, 64, 128, 256, 384) for d in (-1, 0, 1)]
    seqs = [(int(g.integers(0, 1500)), t) for t in around] + [(1900, 1), (0, 1), (-1, 4), (640, 300 // G + 1)]
    lengths = [max(b, 0) + t for b, t in seqs]
    n_pages = sum(-(-x // 16) for x in lengths) + 1
    c = ref.Cache(n_pages, 2, 16, hd, e4m3, seed=30 + seed)
    table = ref.scattered_table(lengths, 16, n_pages, seed=31)
    q = torch.randn(sum(t for _, t in seqs), nq, hd, generator=torch.Generator().manual_seed(32)).to(torch.bfloat16).cuda()
    check_tree(c, q, seqs, table, "tree", seed=33)


@pytest.mark.parametrize("e4m3,hd,nq,page", [(False, 128, 8, 8), (True, 128, 16, 24), (False, 64, 2, 4), (True, 64, 6, 16), (False, 256, 4, 20), (True, 256, 16, 1024)])
@pytest.mark.parametrize("window,sinks", [(7, 3), (40, 17), (333, 64), (500, 1 << 30)])
def test_single_tokens_with_first_positions(e4m3, hd, nq, page, window, sinks):
    """Pages of every kind; windows that begin in the page, the group of rows, the tile of the last first position, and far behind it."""
    seqs = [(b, 1) for b in (0, 2, 6, 9, 15, 22, 41, 60, 100, 399, 700, 1301)] + [(-1, 1)]
    lengths = [max(b, 0) + t for b, t in seqs]
    n_pages = sum(-(-x // page) for x in lengths) + 1
    c = ref.Cache(n_pages, 2, page, hd, e4m3, seed=40)
    table = ref.scattered_table(lengths, page, n_pages, seed=41)
    q = torch.randn(len(seqs), nq, hd, generator=torch.Generator().manual_seed(42)).to(torch.bfloat16).cuda()
    check_tree(c, q, seqs, table, "causal", window=window, sinks=sinks, single=True)
