"""Plain 64-bit restatements of the paged cache operators, and builders of small caches.  No arithmetic is shared with
the library: e4m3 numbers come from a table built from the format's definition."""
from __future__ import annotations

import math

import torch

from paper_2410_23668_b200 import binding as kl

E4M3 = torch.tensor([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127], dtype=torch.float64)


def e4m3_values(codes: torch.Tensor) -> torch.Tensor:
    """Value of every code byte (0x7f, 0xff: NaN)."""
    table = torch.cat([E4M3, torch.tensor([math.nan], dtype=torch.float64)])
    table = torch.cat([table, -table])
    return table[codes.view(torch.uint8).cpu().long()]


def e4m3_round(x: torch.Tensor) -> torch.Tensor:
    """Nearest e4m3 number (the even code between two), saturating; NaN stays."""
    x = x.double()
    a = x.abs().clamp(max=448.0).nan_to_num(0.0)
    hi = torch.searchsorted(E4M3, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = E4M3[hi] - a, a - E4M3[lo]
    y = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), E4M3[hi], E4M3[lo])
    return torch.where(x.isnan(), x, torch.copysign(y, x))


def row_exponent(big: float) -> int:
    """Smallest e >= -127 with big <= 448 * 2^e."""
    e = -127
    while big > 448.0 * 2.0 ** e:
        e += 1
    return e


class Cache:
    """A pool on the device next to its values in 64 bits on the host."""

    def __init__(self, n_pages, nkv, page, hd, e4m3, bounds=False, rows_first=False, seed=0, poison=False):
        self.n_pages, self.nkv, self.page, self.hd, self.e4m3 = n_pages, nkv, page, hd, e4m3
        g = torch.Generator().manual_seed(seed)
        shape = (n_pages, nkv, page, hd)

        def make():
            if e4m3:
                codes = torch.randint(0, 254, shape, generator=g)
                codes = torch.where(codes >= 127, codes + 1, codes).to(torch.uint8)   # no NaN
                if poison:
                    codes.fill_(0x7f)
                return codes
            t = torch.randn(shape, generator=g).to(torch.bfloat16)
            return torch.full_like(t, math.nan) if poison else t

        self.k0, self.v0 = make(), make()
        self.ke0 = torch.randint(110, 122, shape[:3], generator=g).to(torch.uint8) if e4m3 else None
        self.ve0 = torch.randint(110, 122, shape[:3], generator=g).to(torch.uint8) if e4m3 else None
        self.b0 = torch.randn(n_pages, nkv, 2, hd, generator=g).sort(2).values.to(torch.bfloat16) if bounds else None

        def put(t):
            if t is None:
                return None
            if rows_first and t.dim() == 4:
                return t.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
            return t.cuda()

        self.k, self.v = put(self.k0), put(self.v0)
        self.ke = None if self.ke0 is None else self.ke0.cuda()
        self.ve = None if self.ve0 is None else self.ve0.cuda()
        self.bounds = None if self.b0 is None else self.b0.cuda()
        self.handle = kl.PagedCache(self.k, self.v, self.ke, self.ve, self.bounds)

    def values(self, which: str) -> torch.Tensor:
        """What the device's pool stands for now, in 64 bits."""
        t = {"k": self.k, "v": self.v}[which].cpu()
        if not self.e4m3:
            return t.double()
        e = {"k": self.ke, "v": self.ve}[which].cpu().double()
        return e4m3_values(t) * torch.pow(torch.tensor(2.0, dtype=torch.float64), e - 127)[..., None]


def scattered_table(lengths, page, n_pages, seed=0, extra=2):
    """Page table with every sequence's pages scattered over the pool; entries behind a sequence's last page are -1."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    assert sum(need) <= n_pages
    order = torch.randperm(n_pages, generator=g).tolist()
    table = torch.full((len(lengths), max(need) + extra), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    return table


def attention_ref(k, v, q, positions, table, page, scale, window=0, selected=None):
    """out, lse, sum p |v|, largest scale * sum |q k| -- all in 64 bits; k, v: pools of values; q [n, nq, hd]."""
    n, nq, hd = q.shape
    nkv = k.shape[1]
    G = nq // nkv
    out = torch.zeros(n, nq, hd, dtype=torch.float64)
    mass = torch.zeros(n, nq, hd, dtype=torch.float64)
    lse = torch.full((n, nq), -math.inf, dtype=torch.float64)
    reach = torch.zeros(n, nq, dtype=torch.float64)
    for s in range(n):
        pos = int(positions[s])
        for h in range(nkv):
            if pos < 0:
                continue
            if selected is None:
                at = list(range(pos + 1))
            else:
                pages = pos // page + 1
                at = [p * page + r for p in selected[s][h].tolist()[:pages] if 0 <= p < pages for r in range(page) if p * page + r <= pos]
            if window:
                at = [p for p in at if p > pos - window]
            if not at:
                continue
            at = torch.tensor(at)
            phys, r = table[s].long()[at // page], at % page
            kk, vv = k[phys, h, r], v[phys, h, r]
            qq = q[s, h * G:(h + 1) * G].double()
            sc = scale * qq @ kk.T
            heads = slice(h * G, (h + 1) * G)
            p = torch.softmax(sc, 1)
            out[s, heads] = p @ vv
            mass[s, heads] = p @ vv.abs()
            lse[s, heads] = torch.logsumexp(sc, 1)
            reach[s, heads] = scale * (qq.abs() @ kk.abs().T).amax(1)
    return out, lse, mass, reach


def select_ref(bounds, q, positions, table, page, keep_first, keep_last, n_select):
    n, nq, hd = q.shape
    nkv = bounds.shape[1]
    G = nq // nkv
    out = torch.full((n, nkv, n_select), -1, dtype=torch.int32)
    for s in range(n):
        count = int(positions[s]) // page + 1 if positions[s] >= 0 else 0
        if not count:
            continue
        b = bounds[table[s, :count].long()].double()
        for h in range(nkv):
            best = None
            for x in q[s, h * G:(h + 1) * G].double():
                hi = torch.where(x >= 0, x * b[:, h, 1], x * b[:, h, 0]).sum(1).float()
                best = hi if best is None else torch.where(best.isnan(), hi, torch.where(hi.isnan(), best, torch.maximum(best, hi)))
            forced = [p for p in range(count) if p < keep_first or p >= count - keep_last]
            score = best.tolist()
            rest = sorted((p for p in range(count) if p not in set(forced)), key=lambda p: (math.isnan(score[p]), 0.0 if math.isnan(score[p]) else -score[p], p))
            keep = sorted(forced + rest[:max(0, n_select - len(forced))])[:n_select]
            out[s, h, :len(keep)] = torch.tensor(keep, dtype=torch.int32)
    return out


class PlainDecoder:
    """The decode step in 64 bits over a cache kept as lists of rows per (layer, sequence): what kl_decode_step_paged
    computes, written out.  e4m3: rows are stored as the values their codes stand for.  n_select: 0, or pages per kv head."""

    def __init__(self, shape, layers, glob, page, e4m3=False, n_select=0):
        self.s, self.page, self.e4m3, self.n_select = shape, page, e4m3, n_select
        self.layers = [{k: v.double() for k, v in l.items()} for l in layers]
        self.glob = {k: v.double() for k, v in glob.items()}

    def _norm(self, x, gain):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + self.s.rms_eps) * gain

    def _rope(self, x, pos):
        half = self.s.head_dim // 2
        f = pos * self.s.rope_theta ** (-2.0 * torch.arange(half, dtype=torch.float64) / self.s.head_dim)
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * f.cos() - b * f.sin(), b * f.cos() + a * f.sin()], -1)

    def held(self, x):
        """Row(s) [nkv, hd] as the cache stands for them."""
        if not self.e4m3:
            return x.float().to(torch.bfloat16).double()
        out = torch.empty_like(x)
        for h in range(x.shape[0]):
            e = row_exponent(float(x[h].abs().max()))
            out[h] = e4m3_round(x[h] * 2.0 ** -e) * 2.0 ** e
        return out

    def step(self, cache, token, pos):
        """One sequence; cache: per layer (k, v) tensors [nkv, rows, hd] of the rows before pos, extended in place.  Returns hidden, logits."""
        s, G = self.s, self.s.n_q_heads // self.s.n_kv_heads
        x = self.glob["embed"][token]
        for l, w in enumerate(self.layers):
            a = self._norm(x, w["norm1"])
            q, k, v = w["wq"] @ a, w["wk"] @ a, w["wv"] @ a
            if "bq" in w:
                q, k, v = q + w["bq"], k + w["bk"], v + w["bv"]
            q = self._rope(q.view(s.n_q_heads, s.head_dim), pos)
            k = self.held(self._rope(k.view(s.n_kv_heads, s.head_dim), pos))
            v = self.held(v.view(s.n_kv_heads, s.head_dim))
            kk, vv = (torch.cat([c, r[:, None]], 1) for c, r in zip(cache[l], (k, v)))
            cache[l] = (kk, vv)
            o = torch.empty(s.n_q_heads, s.head_dim, dtype=torch.float64)
            for h in range(s.n_kv_heads):
                at = torch.arange(pos + 1)
                pages = pos // self.page + 1
                if self.n_select and pages > self.n_select:
                    lo = torch.stack([kk[h, p * self.page:(p + 1) * self.page].amin(0) for p in range(pages)])
                    hi = torch.stack([kk[h, p * self.page:(p + 1) * self.page].amax(0) for p in range(pages)])
                    score = torch.stack([torch.maximum(y * lo, y * hi).sum(1) for y in q[h * G:(h + 1) * G]]).amax(0)
                    rest = sorted(range(1, pages - 1), key=lambda p: (-float(score[p]), p))[:self.n_select - 2]
                    at = torch.cat([at[p * self.page:(p + 1) * self.page] for p in sorted([0, pages - 1] + rest)])
                sc = q[h * G:(h + 1) * G] @ kk[h, at].T / math.sqrt(s.head_dim)
                o[h * G:(h + 1) * G] = torch.softmax(sc, 1) @ vv[h, at]
            x = x + w["wo"] @ o.flatten()
            a = self._norm(x, w["norm2"])
            g = w["wgate"] @ a
            x = x + w["wdown"] @ (g / (1 + torch.exp(-g)) * (w["wup"] @ a))
        return x, self.glob["lm_head"] @ self._norm(x, self.glob["norm_f"])
