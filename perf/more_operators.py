"""What the operators of drafted tokens on a paged cache are measured on: cases, their inputs, a plain form, the library's calls.

A program that checks several drafted tokens of a sequence in one pass (a chain or a tree of them) needs three operators next to
the framework's single-token ones:

  rotate   rows of new keys and values go to the positions of their sequences, the keys turned by their angles on the way (a
           drafted token's angle goes by its depth in the tree, its place by its number), as bf16 or as e4m3 codes with one
           power-of-two scale per (position, head), page bounds kept; queries are turned in the same call
  tree     attention of all new tokens of every sequence over the cached positions (all of them, or the last `window` and a few
           first ones) and over those new tokens that a bit mask names (their ancestors and themselves)
  sample   one token per row of logits from a given random number: temperature, top-k, top-p, min-p, each per row

Case keys: op; for rotate and tree: kv ("bf16" or "e4m3"), hd (head size), nq and nkv (heads), page (rows of a page), seqs, ctx
(cached positions of the longest sequence), ragged (lengths and token counts spread, some slots empty), tokens (new tokens of a
sequence), drafted (a tree of tokens or a prompt's consecutive ones), window, sinks; for sample: rows, vocab, top_k, top_p, min_p
(0, 1, 0: off), temperature, mixed (every row its own settings around these).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

E4M3_MAX = 448.0
THETA = 500000.0


# ---- cases

def listed():
    h8, h70 = dict(hd=128, nq=32, nkv=8), dict(hd=128, nq=64, nkv=8)   # head layouts of the 8B and the 70B decoder
    return [
        # one sequence generating: its new row and its queries, latency alone
        dict(name="rotate 1 row bf16", op="rotate", kv="bf16", **h8, page=16, seqs=1, ctx=4095, ragged=False, tokens=1, drafted=False),
        # a serving batch's drafted trees, some slots of the batch empty
        dict(name="rotate 32 x 8 drafted e4m3", op="rotate", kv="e4m3", **h8, page=16, seqs=32, ctx=8000, ragged=True, tokens=8, drafted=True),
        # seven chunks of prompts of uneven lengths written at once
        dict(name="rotate 7 x ~1170 e4m3", op="rotate", kv="e4m3", **h8, page=64, seqs=7, ctx=7800, ragged=True, tokens=1950, drafted=False),
        # one conversation with five drafted tokens: latency counts
        dict(name="tree 1 x 5 at 700 bf16", op="tree", kv="bf16", **h8, page=16, seqs=1, ctx=700, ragged=False, tokens=5, drafted=True, window=0, sinks=0),
        # the batch the framework decodes by default, eight drafted tokens each
        dict(name="tree 32 x 8 at 4096 bf16", op="tree", kv="bf16", **h8, page=16, seqs=32, ctx=4096, ragged=False, tokens=8, drafted=True, window=0, sinks=0),
        # a large tree behind one long document
        dict(name="tree 1 x 64 at 65536 e4m3", op="tree", kv="e4m3", **h8, page=64, seqs=1, ctx=65536, ragged=False, tokens=64, drafted=True, window=0, sinks=0),
        # a ragged serving batch of the larger decoder, trees of different sizes
        dict(name="tree 24 x <=32 at <=16384 bf16", op="tree", kv="bf16", **h70, page=16, seqs=24, ctx=16384, ragged=True, tokens=32, drafted=True, window=0, sinks=0),
        # endless chats, one new token each: a window and the first four positions
        dict(name="sinks 32 x 1 window 2044", op="tree", kv="e4m3", **h8, page=16, seqs=32, ctx=20000, ragged=True, tokens=1, drafted=False, window=2044, sinks=4),
        # one sequence generating with the usual settings
        dict(name="sample 1 x 128256", op="sample", rows=1, vocab=128256, top_k=50, top_p=0.9, min_p=0.0, temperature=0.8, mixed=False),
        # a serving batch, every request with settings of its own
        dict(name="sample 32 x 128256 mixed", op="sample", rows=32, vocab=128256, top_k=40, top_p=0.95, min_p=0.05, temperature=0.9, mixed=True),
        # the nodes of a batch's trees, nucleus sampling
        dict(name="sample 256 x 32000 top-p", op="sample", rows=256, vocab=32000, top_k=0, top_p=0.9, min_p=0.0, temperature=1.0, mixed=False),
        # a large batch that draws from everything likely enough
        dict(name="sample 160 x 128256 min-p", op="sample", rows=160, vocab=128256, top_k=0, top_p=1.0, min_p=0.02, temperature=1.3, mixed=False),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["rotate", "tree", "tree", "sample"])
    if op == "sample":
        vocab = _spread(rng, 50, 160000)
        rows = _spread(rng, 1, max(1, min(512, 20_000_000 // vocab)))
        return dict(op=op, rows=rows, vocab=vocab, top_k=rng.choice([0, 0, 1, _spread(rng, 2, 2000)]), top_p=rng.choice([1.0, 1.0, 0.5, 0.9, 0.95, 0.99]),
                    min_p=rng.choice([0.0, 0.0, 0.02, 0.1]), temperature=round(rng.uniform(0.3, 1.6), 2), mixed=rng.random() < 0.5)
    hd = rng.choice([64, 128, 128, 256])
    nkv = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 3, 4, 6, 8, 12])
    case = dict(op=op, kv=rng.choice(["bf16", "e4m3"]), hd=hd, nq=nkv * group, nkv=nkv, page=rng.choice([4, 8, 16, 16, 24, 32, 64, 64, 128]),
                seqs=_spread(rng, 1, 48), ctx=0, ragged=rng.random() < 0.6, tokens=0, drafted=True)
    if op == "rotate":
        case["drafted"] = rng.random() < 0.5
        most = max(1, min(64 if case["drafted"] else 8192, (1 << 23) // (nkv * (group + 2) * hd * case["seqs"])))
        case["tokens"] = _spread(rng, 1, most)
        case["ctx"] = _spread(rng, 1, 9000)
        return case
    case["drafted"] = rng.random() < 0.7
    case["tokens"] = rng.choice([1, _spread(rng, 1, 64), _spread(rng, 1, 64)])
    # at most 134 million cached numbers each of keys and values, and 10^11 operations
    most = min((1 << 27) // (nkv * hd), 10**11 // (4 * hd * nkv * group * case["tokens"])) // case["seqs"]
    case["ctx"] = _spread(rng, 1, max(1, min(100000, most)))
    case["window"] = rng.choice([0, 0, _spread(rng, 1, case["ctx"])])
    case["sinks"] = rng.choice([0, 1, 4, 17]) if case["window"] else 0
    return case


# ---- sizes that follow from a case alone

def _plan(c):
    """(cached positions, new tokens) of every sequence; no tokens for an empty slot."""
    base, count = [], []
    for i in range(c["seqs"]):
        if not c["ragged"] or i == 0:
            base.append(c["ctx"])
            count.append(c["tokens"])
        elif i % 9 == 8:
            base.append(0)
            count.append(0)
        else:
            base.append((i * 40503 * 2654435761 >> 8) % (c["ctx"] + 1))
            count.append(1 + (i * 2654435761 >> 7) % c["tokens"])
    return base, count


def _geometry(c):
    base, count = _plan(c)
    pages = [-(-(b + t) // c["page"]) for b, t in zip(base, count)]
    return base, count, pages, max(1, max(pages)), sum(pages) + 2


def work(c):
    if c["op"] == "sample":
        return {"bytes": c["rows"] * (c["vocab"] * 4 + 4 + 8), "flops": 4 * c["rows"] * c["vocab"]}
    base, count, _, _, _ = _geometry(c)
    nq, nkv, hd = c["nq"], c["nkv"], c["hd"]
    row = nkv * (2 * hd if c["kv"] == "bf16" else hd + 1)   # bytes of one position, keys or values
    rows = sum(count)
    if c["op"] == "rotate":
        return {"bytes": rows * (2 * row + 2 * nkv * hd * 2 + 2 * nq * hd * 2), "flops": 3 * rows * (nkv + nq) * hd}
    seen = pairs = 0   # cached positions that some token sees; pairs of a token and what it sees
    for b, t in zip(base, count):
        if t:
            cached = min(b, c["window"] + c["sinks"] - 1) if c["window"] else b
            seen += cached + t
            pairs += t * cached + t * (t + 1) // 2
    return {"bytes": 2 * seen * row + 2 * rows * nq * hd * 2, "flops": 4 * pairs * nq * hd}


# ---- inputs

def prepare(c, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=g, device=dev, dtype=dtype)

    st = {"case": c}
    if c["op"] == "sample":
        n, v = c["rows"], c["vocab"]
        # rows between undecided and almost sure, a few tokens forbidden
        x = normal(n, v, dtype=torch.float32) * (1.2 + 2.3 * torch.rand(n, 1, generator=g, device=dev))
        x[torch.rand(n, v, generator=g, device=dev) < 0.01] = -math.inf
        st["logits"] = x
        st["uniforms"] = torch.rand(n, generator=g, device=dev)
        one = torch.ones(n, device=dev)
        pick = torch.rand(4, n, generator=g, device=dev) if c["mixed"] else torch.full((4, n), 0.5, device=dev)
        st["temperature"] = c["temperature"] * (0.7 + 0.6 * pick[0])
        k = torch.full((n,), c["top_k"], device=dev, dtype=torch.int32)
        st["top_k"] = torch.where(pick[1] > 0.3, k, 0).to(torch.int32)
        st["top_p"] = torch.where(pick[2] > 0.3, c["top_p"] * one, one)
        st["min_p"] = torch.where(pick[3] > 0.3, c["min_p"] * one, 0 * one)
        st["tokens"] = torch.zeros(n, device=dev, dtype=torch.int32)
        st["logprobs"] = torch.zeros(n, device=dev)
        return st

    base, count, pages, table, n_pages = _geometry(c)
    n, nq, nkv, hd, page = c["seqs"], c["nq"], c["nkv"], c["hd"], c["page"]
    rows = sum(count)
    # every sequence's pages lie scattered over the pool; table entries behind its last page name no page
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    counts = torch.tensor(pages, device=dev)
    first = torch.cumsum(counts, 0) - counts
    slot = torch.arange(table, device=dev)[None, :]
    st["page_table"] = torch.where(slot < counts[:, None], order[(first[:, None] + slot).clamp(max=n_pages - 1)], torch.full_like(order[:1], -1)).contiguous()
    shape = (n_pages, nkv, page, hd)
    if c["kv"] == "bf16":
        st["k"], st["v"] = normal(*shape), normal(*shape)
        st["k_exp"] = st["v_exp"] = None
    else:   # codes as a row of largest value 1.75 * 2^e .. 3.5 * 2^e leaves them; scales vary from row to row
        st["k"] = (normal(*shape) * 96).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        st["v"] = (normal(*shape) * 96).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        st["k_exp"] = torch.randint(119, 123, shape[:3], generator=g, device=dev, dtype=torch.uint8)
        st["v_exp"] = torch.randint(117, 124, shape[:3], generator=g, device=dev, dtype=torch.uint8)
    st["positions"] = torch.tensor([b if t else -1 for b, t in zip(base, count)], device=dev, dtype=torch.int32)
    starts = [sum(count[:i]) for i in range(n + 1)]
    single = rows == n and max(count) == 1
    st["rows"] = rows
    st["row_starts"] = None if single else torch.tensor(starts, device=dev, dtype=torch.int32)

    st["row_positions"] = st["mask"] = None
    if c["drafted"]:   # every token's parent is one of the few before it; the first follows the last cached position
        words = -(-max(count) // 32)
        back = torch.randint(1, 4, (max(count),), generator=g, device=dev).tolist()
        parent = [max(0, i - b) if i else -1 for i, b in enumerate(back)]
        depth, seen = [], []
        for i, p in enumerate(parent):
            depth.append(depth[p] + 1 if i else 0)
            seen.append((seen[p] if i else 0) | 1 << i)
        word = [[(m >> 32 * w & 0xffffffff) - (1 << 32 if m >> 32 * w & 0x80000000 else 0) for w in range(words)] for m in seen]
        st["row_positions"] = torch.tensor([b + d for b, t in zip(base, count) for d in depth[:t]], device=dev, dtype=torch.int32)
        st["mask"] = torch.tensor([w for t in count for w in word[:t]], device=dev, dtype=torch.int32)

    if c["op"] == "rotate":
        a, b = normal(n_pages, nkv, hd), normal(n_pages, nkv, hd)
        st["bounds"] = torch.stack([torch.minimum(a, b), torch.maximum(a, b)], 2).contiguous()
        # the projections' output: rows of one fused tensor, of a loudness of their own
        fused = normal(rows, nq + 2 * nkv, hd) * torch.exp(0.5 * normal(rows, nq + 2 * nkv, 1))
        st["q"], st["k_rows"], st["v_rows"] = fused[:, :nq], fused[:, nq:nq + nkv], fused[:, nq + nkv:]
        st["q_out"] = torch.zeros(rows, nq, hd, device=dev, dtype=torch.bfloat16)
        st["freqs"] = THETA ** (-torch.arange(0, hd, 2, device=dev, dtype=torch.float64) / hd)
        return st
    st["q"] = normal(rows, nq, hd) * 2
    st["out"] = torch.zeros_like(st["q"])
    return st


# ---- one pass

def run(st):
    if own:
        return _run_own(st)
    return {"rotate": _rotate, "tree": _tree, "sample": _sample}[st["case"]["op"]](st)


def _run_own(st):
    from paper_2410_23668_b200 import binding as kl
    c, stream = st["case"], torch.cuda.current_stream()
    if c["op"] == "sample":
        kl.kl_sample(st["logits"], st["uniforms"], st["tokens"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"],
                     logprobs=st["logprobs"], stream=stream)
        return [st["tokens"], st["logprobs"]]
    if "cache" not in st:   # the handle and the workspace that a program keeps
        st["cache"] = kl.PagedCache(st["k"], st["v"], st["k_exp"], st["v_exp"], bounds=st.get("bounds"))
        if c["op"] == "tree":
            st["workspace"] = torch.empty(kl.kl_paged_tree_workspace_bytes(st["cache"], c["nq"]), dtype=torch.uint8, device="cuda")
    if c["op"] == "rotate":
        kl.kl_paged_append_rotated(st["cache"], st["k_rows"], st["v_rows"], st["positions"], st["page_table"], st["freqs"], row_starts=st["row_starts"],
                                   row_positions=st["row_positions"], q=st["q"], q_out=st["q_out"], stream=stream)
        return _pool(st)
    kl.kl_paged_tree_attention(st["cache"], st["q"], st["out"], st["positions"], st["page_table"], st["workspace"], row_starts=st["row_starts"],
                               row_positions=st["row_positions"], mask=st["mask"], window=c["window"], n_sinks=c["sinks"], stream=stream)
    return [st["out"]]


def _pool(st):
    """The cache as an append leaves it (the codes are e4m3 numbers, their scales' exponents whole numbers), and the turned queries."""
    return [t for t in (st["k"], st["v"], st["k_exp"], st["v_exp"], st["bounds"], st["q_out"]) if t is not None]


# ---- plain forms

def _scale(exponent):
    """2^(exponent - 127), to the bit: the exponent field of a 32-bit number, or 2^-127 as the subnormal it is."""
    e = exponent.to(torch.int32)
    return torch.where(e > 0, e << 23, 1 << 22).view(torch.float32)


def _rows_of(st):
    """(sequence, number among its sequence's new tokens, position) of every row."""
    pos = st["positions"].long()
    r = torch.arange(st["rows"], device=pos.device)
    if st["row_starts"] is None:
        return r, torch.zeros_like(r), pos
    starts = st["row_starts"].long()
    seq = torch.searchsorted(starts[1:].contiguous(), r, right=True)
    return seq, r - starts[seq], pos[seq] + r - starts[seq]


def _turn(x, c, s):
    """Pairs (i, i + half) of x's last axis turned by angles of cosine c and sine s."""
    a, b = x.chunk(2, -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _rotate(st):
    c = st["case"]
    seq, _, at = _rows_of(st)
    page, off = st["page_table"].long()[seq, at // c["page"]], at % c["page"]
    turn = at if st["row_positions"] is None else st["row_positions"].long()
    # angles of far positions, and keys next to a border between two codes or two scales: in 64 bits
    angle = turn.double()[:, None, None] * st["freqs"]
    cos, sin = torch.cos(angle), torch.sin(angle)
    st["q_out"].copy_(_turn(st["q"].float(), cos.float(), sin.float()))
    for name, x in (("k", _turn(st["k_rows"].double(), cos, sin)), ("v", st["v_rows"].float())):
        if c["kv"] == "bf16":
            held = x.to(torch.bfloat16)
            st[name][page, :, off] = held
            held = held.float()
        else:
            mant, ex = torch.frexp(x.abs().amax(-1))   # largest = mant * 2^ex, mant in [1/2, 1)
            ex = torch.where(mant > 0, ex - torch.where(mant > 0.875, 8, 9), -127).clamp(min=-127)
            scale = _scale(ex + 127)[..., None]
            code = (x / scale).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float32).to(torch.float8_e4m3fn)
            st[name].view(torch.uint8)[page, :, off] = code.view(torch.uint8)
            st[name + "_exp"][page, :, off] = (ex + 127).to(torch.uint8)
            held = code.float() * scale
        if name == "k":
            touched, back = torch.unique(page, return_inverse=True)
            fresh = torch.zeros(touched.numel(), device=page.device).index_add_(0, back, (off == 0).float()) > 0
            lo, hi = st["bounds"][touched, :, 0].float(), st["bounds"][touched, :, 1].float()
            lo = torch.where(fresh[:, None, None], math.inf, lo).index_reduce_(0, back, held, "amin")
            hi = torch.where(fresh[:, None, None], -math.inf, hi).index_reduce_(0, back, held, "amax")
            st["bounds"][touched] = torch.stack([lo, hi], 2).to(torch.bfloat16)
    return _pool(st)


def _tree(st):
    c = st["case"]
    n, nq, nkv, hd, page, most = c["seqs"], c["nq"], c["nkv"], c["hd"], c["page"], c["tokens"]
    seq, i, at = _rows_of(st)
    table, dev = st["page_table"].long().clamp(min=0), seq.device
    turn = at if st["row_positions"] is None else st["row_positions"].long()
    base = st["positions"].long().clamp(min=0)
    key = torch.arange(table.shape[1] * page, device=dev)
    # what every row sees, [rows, positions]
    old = key < base[seq][:, None]
    if c["window"]:
        old &= (key < c["sinks"]) | (key > turn[:, None] - c["window"])
    j = key - base[seq][:, None]
    if st["mask"] is None:
        new = (j >= 0) & (j <= i[:, None])
        if c["window"]:
            new &= i[:, None] - j < c["window"]
    else:
        bits = st["mask"].long().gather(1, (j // 32).clamp(0, st["mask"].shape[1] - 1))
        new = (j >= 0) & (j < 32 * st["mask"].shape[1]) & ((bits >> (j % 32)) & 1 > 0)
    seen = torch.zeros(n, most, len(key), dtype=torch.bool, device=dev)
    seen[seq, i] = old | new

    head = torch.arange(nkv, device=dev)[None, :, None]

    def gather(name):
        if st["k_exp"] is None:
            return st[name][table[:, None], head].float().flatten(2, 3)
        x = st[name].view(torch.uint8)[table[:, None], head].view(torch.float8_e4m3fn).float()
        return (x * _scale(st[name + "_exp"][table[:, None], head])[..., None]).flatten(2, 3)

    q = torch.zeros(n, most, nq, hd, device=dev)
    q[seq, i] = st["q"].float()
    s = torch.einsum("nthgd,nhkd->nhtgk", q.view(n, most, nkv, nq // nkv, hd), gather("k")) / math.sqrt(hd)
    s.masked_fill_(~seen[:, None, :, None], -math.inf)
    s.sub_(s.amax(4, keepdim=True).clamp(min=-3e38)).exp_()
    total = s.sum(4, keepdim=True)
    o = torch.einsum("nhtgk,nhkd->nhtgd", s, gather("v"))
    o = torch.where(total > 0, o / total.clamp(min=1e-38), 0.0).permute(0, 2, 1, 3, 4).reshape(n, most, nq, hd)
    return [o[seq, i].to(torch.bfloat16)]


def _sample(st):
    # weights, their sums and what is compared with them in 64 bits: a token next to a border stays or goes as a whole
    x = st["logits"].double()
    top = x.amax(1, keepdim=True)
    y = torch.where(x == top, 0.0, (x - top) / st["temperature"].double()[:, None])
    y, order = torch.sort(y, dim=1, descending=True, stable=True)   # equal logits: the lower token first
    w = torch.exp(y)
    rank = torch.arange(x.shape[1], device=x.device)
    k = st["top_k"].long()[:, None]
    keep = (rank < k) | (k <= 0)
    w = torch.where(keep, w, 0.0)
    p = st["top_p"].double()[:, None]
    before = torch.cumsum(w, 1) - w
    keep &= (before < p * w.sum(1, keepdim=True)) | (p >= 1) | (rank == 0)
    keep &= (w >= st["min_p"].double()[:, None]) | (rank == 0)
    w = torch.where(keep, w, 0.0)
    by_token = torch.zeros_like(w).scatter_(1, order, w)            # drawn in the tokens' own order
    c = torch.cumsum(by_token, 1)
    total = c[:, -1:]
    token = (c <= st["uniforms"].double()[:, None] * total).sum(1, keepdim=True)
    token = torch.minimum(token, (c < total).sum(1, keepdim=True))
    logprob = torch.log(by_token.gather(1, token) / total)[:, 0]
    return [token[:, 0].to(torch.int32), logprob.float()]


# ---- the definitions in 64 bits, sequence after sequence and row after row

def _e4m3_numbers():
    """Every finite e4m3 number that is not negative, in order of its code."""
    return torch.tensor([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127], dtype=torch.float64)


def _nearest_e4m3(x):
    """The e4m3 number nearest to every |x| (the one of even code when two are), with x's sign."""
    num = _e4m3_numbers().to(x.device)
    a = x.abs().clamp(max=E4M3_MAX)
    hi = torch.searchsorted(num, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = num[hi] - a, a - num[lo]
    pick_hi = (up < down) | ((up == down) & (hi % 2 == 0))
    return torch.copysign(torch.where(pick_hi, num[hi], num[lo]), x)


def _power_of_two(e):
    """2^e in 64 bits, to the bit."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def exact(c, seed):
    if c["op"] == "sample":
        return _exact_sample(c, seed)
    base, count, _, _, _ = _geometry(c)
    if c["op"] == "tree" and sum(t * b for t, b in zip(count, base)) * c["nq"] * c["hd"] > 4e12:
        return None
    st = prepare(c, seed)
    dev, page, hd = "cuda", c["page"], c["hd"]
    table = st["page_table"].tolist()
    turn = None if st["row_positions"] is None else st["row_positions"].tolist()
    if c["op"] == "rotate":
        rows, pages, offs, turns = [], [], [], []
        for s in range(c["seqs"]):
            for i in range(count[s]):
                p = base[s] + i
                rows.append(len(rows))
                pages.append(table[s][p // page])
                offs.append(p % page)
                turns.append(turn[len(turns)] if turn else p)
        pages, offs = (torch.tensor(v, device=dev, dtype=torch.long) for v in (pages, offs))
        freqs = st["freqs"].cpu().numpy()
        angle = np.array(turns, dtype=np.float64)[:, None] * freqs
        z = torch.from_numpy(np.cos(angle) + 1j * np.sin(angle)).to(dev)[:, None]

        def turned(x):   # a pair as one complex number
            x = x.double()
            y = torch.complex(x[..., :hd // 2].contiguous(), x[..., hd // 2:].contiguous()) * z
            return torch.cat([y.real, y.imag], -1)

        out = {}
        for name in ("k", "v"):
            x = turned(st["k_rows"]) if name == "k" else st["v_rows"].double()
            out[name] = st[name].double()
            if c["kv"] == "e4m3":
                big = x.abs().amax(-1)
                e = torch.round(torch.log2(big.clamp(min=1e-60) / E4M3_MAX))   # one too small where the largest does not fit
                e = torch.where(big > E4M3_MAX * _power_of_two(e), e + 1, e)
                e = torch.where(big <= E4M3_MAX * _power_of_two(e - 1), e - 1, e).clamp(min=-127.0)
                code = _nearest_e4m3(x * _power_of_two(-e)[..., None])
                out[name + "_exp"] = st[name + "_exp"].clone()
                out[name + "_exp"][pages, :, offs] = (e + 127).to(torch.uint8)
                out[name][pages, :, offs] = code
                x = code * _power_of_two(e)[..., None]
            else:
                out[name][pages, :, offs] = x
            if name == "k":
                held = x
        bounds = st["bounds"].double()
        cut = torch.cat([torch.ones(1, dtype=torch.bool, device=dev), pages[1:] != pages[:-1]])
        block, names = torch.cumsum(cut, 0) - 1, pages[cut]
        dense = torch.full((len(names), page, *held.shape[1:]), math.inf, dtype=torch.float64, device=dev)
        dense[block, offs] = held
        low = dense.min(1).values
        dense[dense == math.inf] = -math.inf
        high = dense.max(1).values
        begun = torch.isinf(dense[:, 0, 0, 0])   # pages that held rows before
        bounds[names, :, 0] = torch.where(begun[:, None, None], torch.minimum(low, bounds[names, :, 0]), low)
        bounds[names, :, 1] = torch.where(begun[:, None, None], torch.maximum(high, bounds[names, :, 1]), high)
        return [out[k] for k in ("k", "v", "k_exp", "v_exp") if k in out] + [bounds, turned(st["q"])]

    out = torch.zeros(st["rows"], c["nq"], hd, dtype=torch.float64, device=dev)
    group, r0 = c["nq"] // c["nkv"], 0
    mask = None if st["mask"] is None else st["mask"].cpu().numpy().astype(np.uint32)
    for s in range(c["seqs"]):
        b, t = base[s], count[s]
        if not t:
            continue
        at = torch.arange(b + t, device=dev)
        tab = torch.tensor(table[s], device=dev)
        p, r = tab[at // page], at % page
        sees = np.zeros((t, b + t), dtype=bool)
        for i in range(t):
            me = turn[r0 + i] if turn else b + i
            sees[i, :b] = True
            if c["window"]:
                sees[i, :max(0, min(b, me - c["window"] + 1))] = False
                sees[i, :min(b, c["sinks"])] = True
            for j in range(t):
                if mask is None:
                    sees[i, b + j] = j <= i and (not c["window"] or i - j < c["window"])
                else:
                    sees[i, b + j] = bool(mask[r0 + i, j // 32] >> np.uint32(j % 32) & np.uint32(1))
        hidden = ~torch.from_numpy(sees).to(dev)
        for h in range(c["nkv"]):
            if c["kv"] == "bf16":
                k, v = st["k"][p, h, r].double(), st["v"][p, h, r].double()
            else:
                k, v = (st[x].view(torch.uint8)[p, h, r].view(torch.float8_e4m3fn).double()
                        * _power_of_two(st[x + "_exp"][p, h, r].long() - 127)[:, None] for x in ("k", "v"))
            for a in range(h * group, (h + 1) * group):
                score = (st["q"][r0:r0 + t, a].double() @ k.T / math.sqrt(hd)).masked_fill(hidden, -math.inf)
                alone = hidden.all(1, keepdim=True)
                out[r0:r0 + t, a] = torch.where(alone, 0.0, torch.softmax(score.masked_fill(alone, 0.0), 1)) @ v
        r0 += t
    return [out]


def _exact_sample(c, seed):
    st = prepare(c, seed)
    x = st["logits"].cpu().numpy().astype(np.float64)
    u, t, p, q = (st[k].cpu().numpy().astype(np.float64) for k in ("uniforms", "temperature", "top_p", "min_p"))
    k = st["top_k"].cpu().numpy()
    tokens, logprobs = [], []
    for r in range(c["rows"]):
        w = np.exp((x[r] - x[r].max()) / t[r])
        ranked = np.lexsort((np.arange(len(w)), -x[r]))
        if k[r] > 0:
            ranked = ranked[:k[r]]
        if p[r] < 1:
            mass = np.cumsum(w[ranked])
            ranked = ranked[:1 + int(np.sum(mass[:-1] < p[r] * mass[-1]))]
        stay = np.sort(ranked[(w[ranked] >= q[r]) | (np.arange(len(ranked)) == 0)])
        mass = np.cumsum(w[stay])
        at = min(int(np.sum(mass <= u[r] * mass[-1])), int(np.sum(mass < mass[-1])))
        tokens.append(int(stay[at]))
        logprobs.append(math.log(w[stay[at]] / mass[-1]))
    return [torch.tensor(tokens, dtype=torch.int32), torch.tensor(logprobs, dtype=torch.float64)]
