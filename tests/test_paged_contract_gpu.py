"""Properties the paged operators promise beyond ordinary batches."""
import pytest
import torch

from paper_2410_23668_b200 import binding as kl, build
from tests import paged_ref as ref
from tests.test_paged_gpu import i32

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
