"""What the paged key-value cache operators are measured on: cases, their inputs, a plain form, the library's calls.

Four operators work on one cache of pages (page p, kv head h, row r of the page, column d):

  append     rows of new keys and values go to the positions of their sequences, as bf16 or as e4m3 codes with one
             power-of-two scale per (position, head); the page's bounds (smallest and largest key per column, what the
             cache stands for) are brought up to date
  read       positions of a sequence come back as contiguous bf16 rows
  select     every (sequence, kv head) picks the pages whose bounds allow the largest score
  attention  one new token per sequence over all of its positions, the last `window` of them, or selected pages

Case keys: op, kv ("bf16" or "e4m3"), hd (head size), nq and nkv (heads), page (rows of a page), seqs, ctx (longest
sequence), ragged (lengths spread over 0..ctx, or all of them ctx), and per operator rows, prompt, window, n_select.
"""
from __future__ import annotations

import math

import torch

own = False

E4M3_MAX = 448.0


# ---- cases

def listed():
    h8, h70 = dict(hd=128, nq=32, nkv=8), dict(hd=128, nq=64, nkv=8)   # head layouts of the 8B and the 70B decoder
    return [
        # one sequence generating: its new row, latency alone
        dict(name="append 1 row bf16", op="append", kv="bf16", **h8, page=16, seqs=1, ctx=4096, ragged=False, prompt=False, rows=1),
        # a serving batch generating, some slots of the batch empty
        dict(name="append 32 rows e4m3", op="append", kv="e4m3", **h8, page=16, seqs=32, ctx=4096, ragged=True, prompt=False, rows=32),
        # seven prompts of uneven lengths written at once, their first pages partly filled already
        dict(name="append 8191 rows e4m3", op="append", kv="e4m3", **h8, page=64, seqs=7, ctx=9000, ragged=True, prompt=True, rows=8191),
        # a shared prefix read back for the next chunk of a prompt
        dict(name="read 1 x 4096 bf16", op="read", kv="bf16", **h8, page=16, seqs=1, ctx=4096, ragged=False, prompt=True, rows=4096),
        # the prefixes of several sequences, long and uneven
        dict(name="read 5 x ~13000 e4m3", op="read", kv="e4m3", **h8, page=64, seqs=5, ctx=20000, ragged=True, prompt=True, rows=65537),
        # one sequence, short and ordinary context: latency counts
        dict(name="attn 1 x 333 bf16", op="attention", kv="bf16", **h8, page=16, seqs=1, ctx=333, ragged=False, window=0, n_select=0),
        # the batch the framework decodes by default
        dict(name="attn 32 x 4096 bf16", op="attention", kv="bf16", **h8, page=16, seqs=32, ctx=4096, ragged=False, window=0, n_select=0),
        # one long document
        dict(name="attn 1 x 65536 e4m3", op="attention", kv="e4m3", **h8, page=64, seqs=1, ctx=65536, ragged=False, window=0, n_select=0),
        # a ragged serving batch of the larger decoder
        dict(name="attn 32 x <=32768 e4m3", op="attention", kv="e4m3", **h70, page=16, seqs=32, ctx=32768, ragged=True, window=0, n_select=0),
        # the selected pages of long sequences only
        dict(name="attn 8 x 32 of 1024 pages", op="attention", kv="bf16", **h8, page=64, seqs=8, ctx=65536, ragged=False, window=0, n_select=32),
        # choosing those pages
        dict(name="select 1 x 65536", op="select", kv="e4m3", **h8, page=64, seqs=1, ctx=65536, ragged=False, n_select=32),
        dict(name="select 32 x <=65536", op="select", kv="bf16", **h70, page=16, seqs=32, ctx=65536, ragged=True, n_select=64),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["append", "read", "attention", "attention", "select"])
    hd = rng.choice([64, 128, 128, 256])
    nkv = rng.choice([1, 2, 4, 8])
    nq = nkv * rng.choice([1, 2, 3, 4, 6, 8, 12])
    case = dict(op=op, kv=rng.choice(["bf16", "e4m3"]), hd=hd, nq=nq, nkv=nkv, page=rng.choice([4, 8, 16, 16, 24, 32, 64, 64, 128]),
                seqs=_spread(rng, 1, 64), ctx=0, ragged=rng.random() < 0.6)
    if op in ("append", "read"):
        rows = _spread(rng, 1, max(1, (1 << 25) // (nkv * hd)))
        case["seqs"] = min(case["seqs"], rows)
        case["prompt"] = op == "read" or rng.random() < 0.6
        case["rows"] = rows if case["prompt"] else case["seqs"]
        case["ctx"] = (rows if case["prompt"] else _spread(rng, 1, 8192)) + _spread(rng, 1, 500)
        return case
    if op == "select":   # bounds of at most 67 million columns
        pages = _spread(rng, 64, max(64, min(32768, (1 << 26) // (nkv * hd * case["seqs"]))))
        case["ctx"] = pages * case["page"] - rng.randrange(case["page"])
        case["n_select"] = _spread(rng, 8, pages // 2)
    else:
        most = (1 << 27) // (nkv * hd * case["seqs"])   # keys and values of at most 134 million numbers each
        case["ctx"] = _spread(rng, 1, max(1, min(131072, most)))
        kind = rng.choice(["all", "all", "window", "select"])
        case["window"] = _spread(rng, 1, case["ctx"]) if kind == "window" else 0
        case["n_select"] = _spread(rng, 2, 128) if kind == "select" else 0
    return case


# ---- sizes that follow from a case alone

def _lengths(c):
    """Positions every sequence holds (for append: after it), as a list."""
    n, ctx = c["seqs"], c["ctx"]
    if c["op"] in ("append", "read"):
        return [s + r for s, r in zip(*_rows(c))]
    if not c["ragged"]:
        return [ctx] * n
    out = []
    for i in range(n):   # a fixed scatter over 1..ctx; the first sequence is the longest, every ninth slot is empty
        out.append(ctx if i == 0 else 0 if i % 9 == 8 else 1 + (i * 40503 * 2654435761 >> 8) % ctx)
    return out


def _rows(c):
    """(first position, rows) of every sequence's rows in an append or a read; no rows for an empty slot."""
    n = c["seqs"]
    if not c["prompt"]:
        pos = [(c["ctx"] - 1) if not c["ragged"] or i == 0 else (i * 40503 * 2654435761 >> 8) % c["ctx"] for i in range(n)]
        rows = [0 if c["ragged"] and i % 9 == 8 else 1 for i in range(n)]
        return pos, rows
    weight = [1 + (i * 7919) % 5 if c["ragged"] else 1 for i in range(n)]
    rows = [c["rows"] * w // sum(weight) for w in weight]
    rows[0] += c["rows"] - sum(rows)
    most = max(0, c["ctx"] - max(rows))
    start = [(i * 2654435761 >> 7) % (most + 1) if c["ragged"] else 0 for i in range(n)]
    return start, rows


def _pages(c, length):
    return -(-length // c["page"])


def _geometry(c):
    lens = _lengths(c)
    table = max(1, max(_pages(c, n) for n in lens))
    return lens, table, sum(_pages(c, n) for n in lens) + 2


def work(c):
    lens, _, _ = _geometry(c)
    nq, nkv, hd = c["nq"], c["nkv"], c["hd"]
    row = nkv * (2 * hd if c["kv"] == "bf16" else hd + 1)   # bytes of one position, keys or values
    if c["op"] in ("append", "read"):
        rows = sum(_rows(c)[1])
        return {"bytes": 2 * rows * (row + 2 * nkv * hd), "flops": 2 * rows * nkv * hd}
    if c["op"] == "select":
        pages = sum(_pages(c, n) for n in lens)
        picked = sum(min(_pages(c, n), c["n_select"]) for n in lens)
        return {"bytes": pages * nkv * 4 * hd + len(lens) * nq * hd * 2 + picked * nkv * 4 + pages * 4, "flops": 2 * pages * nq * hd}
    if c["n_select"]:
        keys = sum(min(n, c["n_select"] * c["page"]) for n in lens)
    else:
        keys = sum(min(n, c["window"]) if c["window"] else n for n in lens)
    return {"bytes": 2 * keys * row + 2 * len(lens) * nq * hd * 2, "flops": 4 * keys * nq * hd}


# ---- inputs

def prepare(c, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    lens, table, n_pages = _geometry(c)
    n, nq, nkv, hd, page = c["seqs"], c["nq"], c["nkv"], c["hd"], c["page"]

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=g, device=dev, dtype=dtype)

    st = {"case": c, "n": n}
    # every sequence's pages lie scattered over the pool; table entries behind its last page name no page
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    counts = torch.tensor([_pages(c, x) for x in lens], device=dev)
    first = torch.cumsum(counts, 0) - counts
    slot = torch.arange(table, device=dev)[None, :]
    inside = slot < counts[:, None]
    st["page_table"] = torch.where(inside, order[(first[:, None] + slot).clamp(max=n_pages - 1)], torch.full_like(order[:1], -1)).contiguous()

    shape = (n_pages, nkv, page, hd)
    st["bounds"] = None
    if c["op"] != "select":   # select reads the pages' bounds alone
        if c["kv"] == "bf16":
            st["k"], st["v"] = normal(*shape), normal(*shape)
            st["k_exp"] = st["v_exp"] = None
        else:   # codes as a row of largest value 1.75 * 2^e .. 3.5 * 2^e leaves them; scales vary from row to row
            st["k"] = (normal(*shape) * 96).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
            st["v"] = (normal(*shape) * 96).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
            st["k_exp"] = torch.randint(119, 123, shape[:3], generator=g, device=dev, dtype=torch.uint8)
            st["v_exp"] = torch.randint(117, 124, shape[:3], generator=g, device=dev, dtype=torch.uint8)
    else:
        a, b = normal(n_pages, nkv, hd), normal(n_pages, nkv, hd)
        st["bounds"] = torch.stack([torch.minimum(a, b) - 1, torch.maximum(a, b) + 1], 2).contiguous()

    if c["op"] in ("append", "read"):
        start, rows = _rows(c)
        st["positions"] = torch.tensor([p if r else -1 for p, r in zip(start, rows)], device=dev, dtype=torch.int32)
        st["rows"] = sum(rows) if c["prompt"] else n
        st["row_starts"] = None
        if c["prompt"]:
            st["row_starts"] = torch.tensor([sum(rows[:i]) for i in range(n + 1)], device=dev, dtype=torch.int32)
        if c["op"] == "append":
            a, b = normal(n_pages, nkv, hd), normal(n_pages, nkv, hd)
            st["bounds"] = torch.stack([torch.minimum(a, b), torch.maximum(a, b)], 2).contiguous()
            # the projections' output: rows of one fused tensor, of a loudness of their own
            fused = normal(st["rows"], 2, nkv, hd) * torch.exp(0.5 * normal(st["rows"], 2, nkv, 1))
            st["k_rows"], st["v_rows"] = fused[:, 0], fused[:, 1]
        else:
            st["k_out"] = torch.zeros(st["rows"], nkv, hd, device=dev, dtype=torch.bfloat16)
            st["v_out"] = torch.zeros_like(st["k_out"])
        return st
    st["positions"] = torch.tensor([x - 1 for x in lens], device=dev, dtype=torch.int32)
    st["q"] = normal(n, nq, hd) * 2
    st["selected"] = None
    if c["op"] == "select":
        st["selected"] = torch.zeros(n, nkv, c["n_select"], device=dev, dtype=torch.int32)
    else:
        st["out"] = torch.zeros_like(st["q"])
        if c["n_select"]:   # distinct pages in ascending order, the newest among them
            draw_ = torch.rand(n, nkv, table, generator=g, device=dev).masked_fill_(~inside[:, None, :], -1.0)
            draw_ += (slot == counts[:, None] - 1)[:, None, :]
            top = draw_.topk(min(c["n_select"], table), dim=2)
            picked = top.indices.masked_fill(top.values < 0, table).sort(2).values
            picked = torch.where(picked == table, -1, picked).to(torch.int32)
            st["selected"] = torch.nn.functional.pad(picked, (0, c["n_select"] - picked.shape[2]), value=-1).contiguous()
    return st


# ---- one pass

def run(st):
    if own:
        return _run_own(st)
    return {"append": _append, "read": _read, "select": _select, "attention": _attention}[st["case"]["op"]](st)


def _run_own(st):
    from paper_2410_23668_b200 import binding as kl
    c = st["case"]
    if "cache" not in st:   # the handle and the workspace that a program keeps
        if c["op"] == "select":   # it reads the bounds alone: the pages' rows need no memory
            kind = kl.KL_KV_E4M3 if c["kv"] == "e4m3" else kl.KL_KV_BF16
            st["cache"] = kl.PagedCache(None, None, bounds=st["bounds"], page_size=c["page"], kv_type=kind)
        else:
            st["cache"] = kl.PagedCache(st["k"], st["v"], st["k_exp"], st["v_exp"], bounds=st["bounds"])
        if c["op"] in ("select", "attention"):
            need = kl.kl_paged_workspace_bytes(st["cache"], c["nq"], st["n"], st["page_table"].shape[1])
            st["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    cache, stream = st["cache"], torch.cuda.current_stream()
    if c["op"] == "append":
        kl.kl_paged_append(cache, st["k_rows"], st["v_rows"], st["positions"], st["page_table"], row_starts=st["row_starts"], stream=stream)
        return _pool(st)
    if c["op"] == "read":
        kl.kl_paged_read(cache, st["k_out"], st["v_out"], st["positions"], st["page_table"], row_starts=st["row_starts"], stream=stream)
        return [st["k_out"], st["v_out"]]
    if c["op"] == "select":
        kl.kl_paged_select(cache, st["q"], st["positions"], st["page_table"], st["selected"], st["workspace"], keep_first=1, keep_last=1, stream=stream)
        return [st["selected"]]
    kl.kl_paged_attention(cache, st["q"], st["out"], st["positions"], st["page_table"], st["workspace"], window=c["window"],
                          selected=st["selected"], stream=stream)
    return [st["out"]]


def _pool(st):
    """The cache as an append leaves it: the codes are e4m3 numbers, their scales' exponents whole numbers."""
    return [t for t in (st["k"], st["v"], st["k_exp"], st["v_exp"], st["bounds"]) if t is not None]


# ---- plain forms

def _scale(exponent):
    """2^(exponent - 127), to the bit: the exponent field of a 32-bit number, or 2^-127 as the subnormal it is."""
    e = exponent.to(torch.int32)
    return torch.where(e > 0, e << 23, 1 << 22).view(torch.float32)


def _places(st):
    """(page, row of the page, whether there is such a row) of every row handed in or out."""
    c, pos = st["case"], st["positions"].long()
    r = torch.arange(st["rows"], device=pos.device)
    if st["row_starts"] is None:
        seq, at, live = r, pos, pos >= 0
    else:
        starts = st["row_starts"].long()
        seq = torch.searchsorted(starts[1:].contiguous(), r, right=True)
        at = pos[seq] + r - starts[seq]
        live = pos[seq] >= 0
    at = at.clamp(min=0)
    return st["page_table"].long()[seq, at // c["page"]], at % c["page"], live


def _append(st):
    c = st["case"]
    page, off, live = _places(st)
    page, off = page[live], off[live]
    for name, rows in (("k", st["k_rows"][live]), ("v", st["v_rows"][live])):
        if c["kv"] == "bf16":
            st[name][page, :, off] = rows
            held = rows.float()
        else:
            x = rows.float()
            mant, ex = torch.frexp(x.abs().amax(-1))   # largest = mant * 2^ex, mant in [1/2, 1)
            ex = torch.where(mant > 0, ex - torch.where(mant > 0.875, 8, 9), -127).clamp(min=-127)
            scale = _scale(ex + 127)[..., None]
            code = (x / scale).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
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


def _read(st):
    page, off, live = _places(st)
    out = []
    for name in ("k", "v"):
        x = st[name].view(torch.uint8 if st["k_exp"] is not None else torch.bfloat16)[page, :, off]
        if st["k_exp"] is not None:
            x = x.view(torch.float8_e4m3fn).float() * _scale(st[name + "_exp"][page, :, off])[..., None]
        out.append(torch.where(live[:, None, None], x.float(), st[name + "_out"].float()).to(torch.bfloat16))
    return out


def _select(st):
    c = st["case"]
    n, nkv, hd, k = st["n"], c["nkv"], c["hd"], c["n_select"]
    table = st["page_table"]
    count = (torch.div(st["positions"], c["page"], rounding_mode="floor") + 1).long()   # pages of every sequence
    slot = torch.arange(table.shape[1], device=table.device)
    # scores in 64 bits, rounded to 32 at the end: two pages may be next to each other at the border
    b = st["bounds"][table.long().clamp(min=0)].double()                                # [n, P, nkv, 2, hd]
    q = st["q"].double().view(n, nkv, -1, hd)
    s = torch.einsum("nhgd,nphd->nhgp", q.clamp(min=0), b[:, :, :, 1]) + torch.einsum("nhgd,nphd->nhgp", q.clamp(max=0), b[:, :, :, 0])
    s = s.amax(2).float()
    inside = (slot[None, :] < count[:, None])[:, None]
    forced = ((slot[None, :] < 1) | (slot[None, :] >= count[:, None] - 1))[:, None]
    s = s.masked_fill(forced, math.inf).masked_fill(~inside, -math.inf)
    order = torch.sort(s, dim=2, descending=True, stable=True).indices[:, :, :k]        # equal scores: the lower page first
    order = torch.where(inside.expand_as(s).gather(2, order), order, table.shape[1]).sort(2).values
    order = torch.where(order == table.shape[1], -1, order)
    return [torch.nn.functional.pad(order, (0, k - order.shape[2]), value=-1).to(torch.int32)]


def _attention(st):
    c = st["case"]
    n, nkv, hd, page = st["n"], c["nkv"], c["hd"], c["page"]
    table = st["page_table"].long()
    if st["selected"] is not None:
        logical = st["selected"].long()                                                 # [n, nkv, P]
        named = logical >= 0
        physical = table[torch.arange(n, device=table.device)[:, None, None], logical.clamp(min=0)]
    else:
        logical = torch.arange(table.shape[1], device=table.device).expand(n, nkv, -1)
        physical, named = table[:, None].expand(n, nkv, -1), logical >= 0
    physical = physical.clamp(min=0)
    head = torch.arange(nkv, device=table.device)[None, :, None]
    pos = st["positions"].long()[:, None, None, None]
    at = logical[..., None] * page + torch.arange(page, device=table.device)             # position of every gathered row
    seen = named[..., None] & (at <= pos)
    if c["window"]:
        seen &= at > pos - c["window"]
    seen = seen.flatten(2)                                                               # [n, nkv, N]

    def gather(name):
        if st["k_exp"] is None:
            return st[name][physical, head].float().flatten(2, 3)
        x = st[name].view(torch.uint8)[physical, head].view(torch.float8_e4m3fn).float()
        return (x * _scale(st[name + "_exp"][physical, head])[..., None]).flatten(2, 3)

    q = st["q"].float().view(n, nkv, -1, hd)
    s = torch.einsum("nhgd,nhkd->nhgk", q, gather("k")) / math.sqrt(hd)
    s = s.masked_fill(~seen[:, :, None], -math.inf)
    m = s.amax(3, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - m)
    total = p.sum(3, keepdim=True)
    o = torch.einsum("nhgk,nhkd->nhgd", p, gather("v"))
    return [torch.where(total > 0, o / total.clamp(min=1e-38), 0.0).reshape(n, c["nq"], hd).to(torch.bfloat16)]


# ---- the definitions in 64 bits, sequence after sequence

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
    st = prepare(c, seed)
    dev, page = "cuda", c["page"]
    pos, table = st["positions"].tolist(), st["page_table"].tolist()
    if c["op"] in ("append", "read"):
        starts = st["row_starts"].tolist() if st["row_starts"] is not None else list(range(st["n"] + 1))
        rows, pages, offs = [], [], []
        for s in range(st["n"]):
            for i in range(starts[s + 1] - starts[s] if pos[s] >= 0 else 0):
                rows.append(starts[s] + i)
                pages.append(table[s][(pos[s] + i) // page])
                offs.append((pos[s] + i) % page)
        rows, pages, offs = (torch.tensor(v, device=dev, dtype=torch.long) for v in (rows, pages, offs))
    if c["op"] == "append":
        out = {}
        for name in ("k", "v"):
            x = st[name + "_rows"][rows].double()
            out[name] = st[name].double()
            if c["kv"] == "e4m3":
                big = x.abs().amax(-1)
                e = torch.round(torch.log2(big.clamp(min=1e-60) / E4M3_MAX))   # one too small where the largest does not fit
                e = torch.where(big > E4M3_MAX * _power_of_two(e), e + 1, e).clamp(min=-127.0)
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
        if len(pages):   # every touched page as a block of its own, places without a new row left at infinity
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
        return [out[k] for k in ("k", "v", "k_exp", "v_exp") if k in out] + [bounds]
    if c["op"] == "read":
        back = []
        for name in ("k", "v"):
            o = st[name + "_out"].double()
            x = st[name][pages, :, offs] if c["kv"] == "bf16" else st[name].view(torch.uint8)[pages, :, offs].view(torch.float8_e4m3fn)
            x = x.double()
            if c["kv"] == "e4m3":
                x = x * _power_of_two(st[name + "_exp"][pages, :, offs].long() - 127)[..., None]
            o[rows] = x
            back.append(o)
        return back
    group = c["nq"] // c["nkv"]
    if c["op"] == "select":
        out = torch.full((st["n"], c["nkv"], c["n_select"]), -1, dtype=torch.int32)
        for s in range(st["n"]):
            count = pos[s] // page + 1 if pos[s] >= 0 else 0
            if not count:
                continue
            b = st["bounds"][torch.tensor(table[s][:count], device=dev)].double()
            for h in range(c["nkv"]):
                best = torch.full((count,), -math.inf, dtype=torch.float64, device=dev)
                for q in st["q"][s, h * group:(h + 1) * group].double():
                    best = torch.maximum(best, torch.maximum(q * b[:, h, 0], q * b[:, h, 1]).sum(1))
                score = best.float().tolist()
                rest = sorted(range(1, count - 1), key=lambda p: (-score[p], p))
                keep = sorted(({0, count - 1} | set(rest[:max(0, c["n_select"] - len({0, count - 1}))])))
                out[s, h, :len(keep)] = torch.tensor(keep, dtype=torch.int32)
        return [out]
    out = torch.zeros(st["n"], c["nq"], c["hd"], dtype=torch.float64, device=dev)
    for s in range(st["n"]):
        if pos[s] < 0:
            continue
        first = max(0, pos[s] - c["window"] + 1) if c["window"] else 0
        everything = torch.arange(first, pos[s] + 1, device=dev)
        tab = torch.tensor(table[s], device=dev)
        for h in range(c["nkv"]):
            at = everything
            if st["selected"] is not None:
                chosen = st["selected"][s, h]
                chosen = chosen[chosen >= 0].long()
                at = (chosen[:, None] * page + torch.arange(page, device=dev)).flatten()
                at = at[at <= pos[s]]
            p, r = tab[at // page], at % page
            if c["kv"] == "bf16":
                k, v = st["k"][p, h, r].double(), st["v"][p, h, r].double()
            else:
                k, v = (st[x].view(torch.uint8)[p, h, r].view(torch.float8_e4m3fn).double()
                        * _power_of_two(st[x + "_exp"][p, h, r].long() - 127)[:, None] for x in ("k", "v"))
            score = st["q"][s, h * group:(h + 1) * group].double() @ k.T / math.sqrt(c["hd"])
            out[s, h * group:(h + 1) * group] = torch.softmax(score, 1) @ v
    return [out]
