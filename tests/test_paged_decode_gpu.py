"""kl_decode_step_paged against the decode step in 64 bits, and against the step on a contiguous cache."""
import dataclasses

import pytest
import torch

from paper_2410_23668_b200 import binding as kl, inputs as gen
from tests import helpers, paged_ref as ref

pytestmark = pytest.mark.gpu

WIDE = gen.ModelShape(2, 512, 8, 2, 128, 768, 640, 1e-5, 500000.0)   # head size 128, four query heads per kv head
BIAS = dataclasses.replace(gen.TINY, n_layers=2, qkv_bias=True)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Setup:
    """A model, prefilled pages of a ragged batch, and the same prefix for the plain decoder."""

    def __init__(self, shape, contexts, page, kv_type, n_select=0, max_batch=None, seed=0, table_pages=None):
        self.shape, self.page, self.n_select, self.contexts = shape, page, n_select, contexts
        self.layers = [gen.make_layer(shape, l, seed) for l in range(shape.n_layers)]
        self.glob = gen.make_globals(shape, seed)
        self.dec = helpers.make_decoder(shape, max_batch or max(2, len(contexts)), 16, seed)
        self.plain = ref.PlainDecoder(shape, self.layers, self.glob, page, kv_type == kl.KL_KV_E4M3, n_select)
        n_pages = sum(-(-(c + 8) // page) for c in contexts if c >= 0) + 1
        table = ref.scattered_table([max(0, c + 8) if c >= 0 else 0 for c in contexts], page, n_pages, seed=3)
        self.table = table.cuda() if table_pages is None else table[:, :table_pages].contiguous().cuda()
        self.caches = [kl.PagedCache.allocate(n_pages, shape.n_kv_heads, page, shape.head_dim, kv_type, bounds=True) for _ in range(shape.n_layers)]
        starts = [0]
        for c in contexts:
            starts.append(starts[-1] + max(0, c))
        self.rows = [[None] * shape.n_layers for _ in contexts]
        for l in range(shape.n_layers):
            g = torch.Generator().manual_seed(100 + l)
            k, v = (torch.randn(max(1, starts[-1]), shape.n_kv_heads, shape.head_dim, generator=g).to(torch.bfloat16) for _ in range(2))
            if starts[-1]:
                kl.kl_paged_append(self.caches[l], k.cuda(), v.cuda(), i32([0 if c >= 0 else -1 for c in contexts]), table.cuda(), row_starts=i32(starts))
            for b, c in enumerate(contexts):
                part = [torch.stack([self.plain.held(r.double()) for r in t[starts[b]:starts[b + 1]]], 1) if c > 0 else
                        torch.zeros(shape.n_kv_heads, 0, shape.head_dim, dtype=torch.float64) for t in (k, v)]
                self.rows[b][l] = tuple(part)
        need = self.dec.kl_paged_step_bytes(self.caches[0], len(contexts), self.table.shape[1], n_select)
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(0xff)
        n = len(contexts)
        self.tok = i32(gen.make_tokens(shape, n, seed).tolist())
        self.pos = i32(contexts)
        self.logits = torch.full((n, shape.vocab), 9.0, device="cuda")
        self.hidden = torch.zeros(n, shape.hidden, device="cuda")

    def step(self, stream=None):
        self.dec.kl_decode_step_paged(self.tok, self.pos, self.caches, self.table, self.logits, self.ws, self.n_select, stream=stream)


@pytest.mark.parametrize("shape,contexts,page,kv_type,n_select", [
    (gen.TINY, [37, 0, 64, 130, 15], 16, kl.KL_KV_BF16, 0),
    (gen.TINY, [37, -1, 64, 130, 16], 8, kl.KL_KV_E4M3, 0),
    (WIDE, [100, 3], 24, kl.KL_KV_E4M3, 0),
    (WIDE, [129], 16, kl.KL_KV_BF16, 0),
    (WIDE, [100, 40, 0], 8, kl.KL_KV_BF16, 4),
    (gen.TINY, [70, 90], 4, kl.KL_KV_E4M3, 6),
    (BIAS, [20, 33], 16, kl.KL_KV_BF16, 0),
])
def test_steps_match_the_plain_decoder(shape, contexts, page, kv_type, n_select):
    s = Setup(shape, contexts, page, kv_type, n_select)
    live = [b for b, c in enumerate(contexts) if c >= 0]
    for t in range(3):
        tok, pos = s.tok.tolist(), s.pos.tolist()
        launches = s.dec.kl_launch_count()
        s.step()
        s.dec.kl_read_hidden(s.hidden, len(contexts))
        torch.cuda.synchronize()
        assert s.dec.kl_last_status() == 0
        assert s.dec.kl_launch_count() - launches == 3 + shape.n_layers * (10 + (2 if n_select else 0))   # short tables: no join
        lg, hd = s.logits.cpu().numpy(), s.hidden.cpu().numpy()
        assert torch.isfinite(s.logits).all()
        nxt = list(tok)
        for b in live:
            hidden, logits = s.plain.step(s.rows[b], tok[b], pos[b])
            assert helpers.rel_l2(hd[b], hidden.numpy()) <= helpers.REL_L2_TOL
            assert helpers.rel_l2(lg[b], logits.numpy()) <= helpers.REL_L2_TOL
            assert abs(lg[b] - logits.numpy()).max() <= helpers.ABS_LOGIT_TOL
            nxt[b] = int(logits.argmax())
        s.dec.kl_argmax_advance(s.logits, s.tok, s.pos, len(contexts))
        torch.cuda.synchronize()
        assert [s.tok.tolist()[b] for b in live] == [nxt[b] for b in live]
        assert [s.pos.tolist()[b] for b in live] == [pos[b] + 1 for b in live]
        for b in range(len(contexts)):
            if b not in live:
                s.pos[b] = -1
    # the rows written are those the plain decoder holds, up to a rounding of values that agree to ~1e-5
    for l, c in enumerate(s.caches):
        for b in live:
            n = contexts[b] + 3
            ko, vo = (torch.zeros(n, shape.n_kv_heads, shape.head_dim, device="cuda") for _ in range(2))
            kl.kl_paged_read(c, ko, vo, i32([0]), s.table[b:b + 1].contiguous(), row_starts=i32([0, n]))
            torch.cuda.synchronize()
            for got, want in zip((ko, vo), s.rows[b][l]):
                got, want = got.cpu().double().transpose(0, 1), want
                assert torch.equal(got[:, :contexts[b]], want[:, :contexts[b]])
                step = 2.0 ** -3 if kv_type == kl.KL_KV_E4M3 else 2.0 ** -7
                assert bool(((got - want).abs() <= step * want.abs() + 1e-3 * want.abs().amax()).all())
    s.dec.close()


def test_same_as_the_contiguous_cache():
    shape, contexts, page, n = gen.TINY, [50, 7, 33], 16, 3
    s = Setup(shape, contexts, page, kl.KL_KV_BF16)
    max_ctx = 64
    dec = helpers.make_decoder(shape, n, max_ctx, 0)
    cache = torch.zeros(gen.kv_cache_shape(shape, n, max_ctx), dtype=torch.bfloat16, device="cuda")
    for l in range(shape.n_layers):
        for b, c in enumerate(contexts):
            for i in range(2):
                cache[l, i, b, :, :c] = s.rows[b][l][i].to(torch.bfloat16).cuda()
    logits, tok, pos = torch.zeros_like(s.logits), s.tok.clone(), s.pos.clone()
    for t in range(4):
        s.step()
        dec.kl_decode_step(tok, pos, cache, logits, n)
        torch.cuda.synchronize()
        assert s.dec.kl_last_status() == 0 and dec.kl_last_status() == 0
        for b in range(n):
            assert helpers.rel_l2(s.logits[b].cpu().numpy(), logits[b].cpu().double().numpy()) <= 1e-3
        s.dec.kl_argmax_advance(s.logits, s.tok, s.pos, n)
        dec.kl_argmax_advance(logits, tok, pos, n)
        torch.cuda.synchronize()
        assert torch.equal(tok, s.tok) and torch.equal(pos, s.pos)
    s.dec.close()
    dec.close()


@pytest.mark.parametrize("kv_type", [kl.KL_KV_BF16, kl.KL_KV_E4M3])
def test_a_wider_table_gives_the_same_step(kv_type):
    """Behind a wide table attention may share its pairs between blocks and takes a launch more per layer."""
    shape, contexts = gen.TINY, [50, -1, 7]
    a, b = (Setup(shape, contexts, 16, kv_type) for _ in range(2))
    wide = torch.full((3, 4096), -1, dtype=torch.int32, device="cuda")
    wide[:, :b.table.shape[1]] = b.table
    b.table = wide
    b.ws = torch.empty(b.dec.kl_paged_step_bytes(b.caches[0], 3, 4096, 0), dtype=torch.uint8, device="cuda").fill_(0xff)
    made = [s.dec.kl_launch_count() for s in (a, b)]
    a.step()
    b.step()
    torch.cuda.synchronize()
    assert [s.dec.kl_launch_count() - m for s, m in zip((a, b), made)] == [3 + shape.n_layers * 10, 3 + shape.n_layers * 11]
    for i in (0, 2):
        assert helpers.rel_l2(a.logits[i].cpu().numpy(), b.logits[i].cpu().double().numpy()) <= 1e-3
    for s in (a, b):
        assert s.dec.kl_last_status() == 0
        s.dec.close()


def test_captured_step_replays_like_eager_ones():
    shape, contexts = gen.TINY, [30, 12]
    a, b = (Setup(shape, contexts, 16, kl.KL_KV_E4M3, n_select=3) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        st = torch.cuda.current_stream()
        a.step(stream=st)
        a.dec.kl_argmax_advance(a.logits, a.tok, a.pos, 2, stream=st)
    for t in range(5):
        graph.replay()
        b.step()
        b.dec.kl_argmax_advance(b.logits, b.tok, b.pos, 2)
        torch.cuda.synchronize()
        assert torch.equal(a.tok, b.tok) and torch.equal(a.pos, b.pos) and torch.equal(a.logits, b.logits)
    assert a.dec.kl_last_status() == 0
    del graph
    a.dec.close()
    b.dec.close()


def test_a_bad_entry_makes_the_step_a_no_op():
    shape, contexts = gen.TINY, [30, 12]
    s = Setup(shape, contexts, 16, kl.KL_KV_BF16)
    good_table, pages = s.table.clone(), s.caches[0].desc.n_pages

    def unchanged():
        before = [t.clone() for c in s.caches for t in (c.tensors[0], c.tensors[1], c.tensors[4])] + [s.logits.clone()]
        s.step()
        torch.cuda.synchronize()
        assert s.dec.kl_last_status() == kl.KL_ERR_OUT_OF_RANGE
        after = [t for c in s.caches for t in (c.tensors[0], c.tensors[1], c.tensors[4])] + [s.logits]
        assert all(torch.equal(x, y) for x, y in zip(before, after))

    for entry in (-1, pages, 2 ** 31 - 1):
        s.table[0, 0] = entry
        unchanged()
        s.table.copy_(good_table)
    s.pos[1] = s.table.shape[1] * 16   # behind the page table
    unchanged()
    s.pos[1] = 12
    s.tok[0] = shape.vocab
    unchanged()
    s.tok[0] = 3
    s.step()
    torch.cuda.synchronize()
    assert s.dec.kl_last_status() == 0 and bool((s.logits != 9.0).all())
    s.dec.close()


def test_refusals():
    s = Setup(gen.TINY, [5, 5], 16, kl.KL_KV_BF16)

    def refused(code, **over):
        args = dict(caches=s.caches, table=s.table, ws=s.ws, n_select=0)
        args.update(over)
        with pytest.raises(kl.KlError) as e:
            s.dec.kl_decode_step_paged(s.tok, s.pos, args["caches"], args["table"], s.logits, args["ws"], args["n_select"])
        assert e.value.code == code

    refused(kl.KL_ERR_INVALID_ARG, n_select=1)
    refused(kl.KL_ERR_INVALID_ARG, ws=s.ws[:256])
    refused(kl.KL_ERR_INVALID_ARG, caches=s.caches[:1])
    other = kl.PagedCache.allocate(4, 2, 32, 64)
    refused(kl.KL_ERR_INVALID_ARG, caches=s.caches[:-1] + [other])                       # another page size, no bounds
    plain = [kl.PagedCache.allocate(8, 2, 16, 64) for _ in range(gen.TINY.n_layers)]
    refused(kl.KL_ERR_INVALID_ARG, caches=plain, n_select=3, ws=torch.empty(1 << 26, dtype=torch.uint8, device="cuda"))
    one = helpers.make_decoder(gen.TINY, 1, 16, 0)                          # no batched path
    with pytest.raises(kl.KlError) as e:
        one.kl_decode_step_paged(s.tok[:1], s.pos[:1], s.caches, s.table[:1], s.logits[:1], s.ws)
    assert e.value.code == kl.KL_ERR_UNSUPPORTED_SHAPE
    one.close()
    s.dec.close()
