"""Plain models of the operators on a paged cache: attention and the append step in fp64 on the CPU, the
bookkeeping of pages in Python lists, and the inputs that their tests share."""
from __future__ import annotations

import math
from dataclasses import dataclass, field

import torch

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
EPS32 = 2.0 ** -24


@dataclass
class Paged:
    """A cache on the CPU: lens[b] keys of sequence b, some[b] new tokens behind them."""
    k: torch.Tensor             # [P, Hkv, page, d] in the cache's type
    v: torch.Tensor
    table: torch.Tensor
    lens: list
    some: list
    kscale: float = 1.0
    vscale: float = 1.0
    starts: list = field(default_factory=list)

    def __post_init__(self):
        self.starts = [0]
        for m in self.some:
            self.starts.append(self.starts[-1] + m)

    def gpu(self):
        """k, v, table, lens, q_start as GPU tensors."""
        return (self.k.cuda(), self.v.cuda(), self.table.cuda(), ints(self.lens).cuda(), ints(self.starts).cuda())

    def keys(self, b):
        """fp64 K and V [Hkv, keys, d] of sequence b, its new tokens among them; None for missing pages."""
        page = self.k.shape[2]
        j = torch.arange(self.lens[b] + self.some[b])
        p = self.table[b].long()[j // page]
        there = p >= 0
        p = p.clamp(min=0)
        return (self.k[p, :, j % page].double().transpose(0, 1) * self.kscale,
                self.v[p, :, j % page].double().transpose(0, 1) * self.vscale, there)


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


def make(lens, some, Hkv, d, page, dtype="bf16", fp8=False, seed=0, spare=3, qk_std=1.0):
    """A cache whose pages lie in no order; keys and values N(0, 1)."""
    gen = torch.Generator().manual_seed(seed)
    cols = [-(-(l + m) // page) for l, m in zip(lens, some)]
    P = sum(cols) + spare
    table = torch.full((len(lens), max(max(cols), 1)), -1, dtype=torch.int32)
    order = torch.randperm(P, generator=gen).to(torch.int32)
    at = 0
    for b, n in enumerate(cols):
        table[b, :n] = order[at:at + n]
        at += n
    k = torch.randn(P, Hkv, page, d, generator=gen) * qk_std
    v = torch.randn(P, Hkv, page, d, generator=gen)
    if fp8:
        to = lambda x: (x * 32).to(torch.float8_e4m3fn)     # noqa: E731
        return Paged(to(k), to(v), table, lens, some, 1 / 32, 1 / 32)
    return Paged(k.to(DT[dtype]), v.to(DT[dtype]), table, lens, some)


def queries(c, Hq, dtype, seed=0, std=1.0, extra=0):
    gen = torch.Generator().manual_seed(seed + 1)
    return (torch.randn(c.starts[-1] + extra, Hq, c.k.shape[3], generator=gen) * std).to(DT[dtype])


def random_tree(some, words, seed=0, holes=True):
    """Bits [T, words] and the same as lists of visible tokens; without `holes` every token sees itself
    and its ancestors, with them any tokens at all, some rows none."""
    gen = torch.Generator().manual_seed(seed + 2)
    rows, lists = [], []
    for m in some:
        seen = torch.zeros(m, m, dtype=torch.bool)
        for i in range(m):
            if holes:
                seen[i] = torch.rand(m, generator=gen) < 0.4
                if i % 5 == 3:
                    seen[i] = False
            else:
                if i:
                    seen[i] = seen[int(torch.randint(0, i, (1,), generator=gen))]
                seen[i, i] = True
        for i in range(m):
            js = [j for j in range(m) if seen[i, j] and j < 64 * words]
            row = [0] * words
            for j in js:
                row[j // 64] |= 1 << (j % 64)
            rows.append([x - (1 << 64) if x >= 1 << 63 else x for x in row])
            lists.append(js)
    return torch.tensor(rows, dtype=torch.int64).view(len(rows), words), lists


def attention(c, q, scale, seen=None):
    """fp64 output [T, Hq, d] and a bound's ingredients: sum_j w_j |v_j| and, per row, the largest sum of
    absolute products of a visible score.  seen: per token the new tokens it sees (None: a chain)."""
    T, Hq, d = q.shape
    Hkv = c.k.shape[1]
    o = torch.zeros(T, Hq, d, dtype=torch.float64)
    mass = torch.zeros_like(o)
    size = torch.zeros(T, Hq, 1, dtype=torch.float64)
    for b, (l, m) in enumerate(zip(c.lens, c.some)):
        if m == 0:
            continue
        k, v, there = c.keys(b)
        for i in range(m):
            t = c.starts[b] + i
            js = range(i + 1) if seen is None else seen[t]
            at = torch.tensor(list(range(l)) + [l + j for j in js if j < m], dtype=torch.long)
            at = at[there[at]]
            if len(at) == 0:
                continue
            for h in range(Hq):
                g = h // (Hq // Hkv)
                x = k[g][at] @ q[t, h].double() * scale
                w = torch.softmax(x, 0)
                o[t, h] = w @ v[g][at]
                mass[t, h] = w @ v[g][at].abs()
                size[t, h] = (k[g][at].abs() @ q[t, h].double().abs()).max() * abs(scale)
    return o, mass, size


def attention_bound(c, dtype, o, mass, size):
    """How far the operator may be from fp64, element by element.

    Rounding of the output: u |o|.  Weights of f16/bf16 are rounded, each by at most u of itself; the sum
    they are divided by moves by as much: 2 u sum w |v|.  f16 holds no weight below 2^-25 of a weight
    of 1, which the largest at least is: keys * 2^-25 * max |v|.  A score's sum of d products (and its
    two scalings, and the argument and result of the exponential) is off by at most (d + 8) e size,
    e = 2^-24, which as a factor of a weight counts twice (numerator and sum); the sums over the keys
    add keys * e."""
    u = HALF_STEP[dtype]
    d = c.k.shape[3]
    n = max(l + m for l, m in zip(c.lens, c.some))
    bound = u * o.abs() + (2 * ((d + 8) * (size + 4) + n) * EPS32) * mass
    if dtype != "f32":
        bound = bound + 2.02 * u * mass
    if dtype == "f16":
        bound = bound + n * 2.0 ** -25 * float((c.v.double() * c.vscale).abs().nan_to_num(0, 0, 0).max())
    return bound + 1e-30


class Pages:
    """The bookkeeping of sequences and pages in Python lists."""

    def __init__(self, table, lens, P):
        self.P = P
        self.max_pages = table.shape[1]
        self.rows = [[int(p) for p in row if p >= 0] for row in table]
        self.lens = list(lens)

    @property
    def refs(self):
        n = [0] * self.P
        for row in self.rows:
            for p in row:
                n[p] += 1
        return n

    @property
    def table(self):
        return ints([row + [-1] * (self.max_pages - len(row)) for row in self.rows])

    def fork(self, parent):
        ok = [0 <= p < len(self.rows) for p in parent]
        self.rows, self.lens = ([list(self.rows[p]) if g else [] for p, g in zip(parent, ok)],
                                [self.lens[p] if g else 0 for p, g in zip(parent, ok)])

    def reserve(self, some, page):
        """The report of flashd_cache_reserve, and (sequence, from, to, keys) of each copied page."""
        for b, m in enumerate(some):
            total = min(self.lens[b] + m, self.max_pages * page)
            self.rows[b] = self.rows[b][:-(-total // page)]
        refs = self.refs
        last = [self.rows[b][l // page] if m > 0 and l % page and l // page < len(self.rows[b]) else -1
                for b, (l, m) in enumerate(zip(self.lens, some))]
        want = []
        beyond = 0
        for b, m in enumerate(some):
            total = self.lens[b] + m
            fits = min(total, self.max_pages * page)
            beyond += -(-(total - fits) // page)
            p = last[b]
            copy = p >= 0 and refs[p] > 1 and (last.count(p) < refs[p] or last.index(p) != b)
            want += [(b, "copy")] * copy
            want += [(b, "new")] * (-(-fits // page) - len(self.rows[b]) if m > 0 else 0)
        free = [p for p in range(self.P) if refs[p] == 0]
        missing = max(0, len(want) - len(free)) + beyond
        report = [missing] + [-1] * len(some)
        copies = []
        if missing == 0:
            for (b, what), p in zip(want, free):
                if what == "copy":
                    at = self.lens[b] // page
                    report[1 + b] = self.rows[b][at]
                    copies.append((b, self.rows[b][at], p, self.lens[b] % page))
                    self.rows[b][at] = p
                else:
                    self.rows[b].append(p)
        return report, copies


def append(c, q, k, v, positions, inv_freq, qw, kw, eps, interleaved):
    """fp64 q_out [T, Hq, d] and what becomes K and V of each token [T, Hkv, d] (before the division by
    the cache's scales), and per element the error bound's sizes."""
    T = q.shape[0]
    d = q.shape[2]
    rot = 0 if inv_freq is None else 2 * len(inv_freq)
    pos = torch.zeros(T, dtype=torch.float64)
    for b, (l, m) in enumerate(zip(c.lens, c.some)):
        pos[c.starts[b]:c.starts[b] + m] = torch.arange(l, l + m, dtype=torch.float64)
    if positions is not None:
        pos = positions.double()

    def turned(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
        size = x.abs().clone()
        y = x.clone()
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
            angle = (pos * float(inv_freq[i]))[:, None]
            y[..., a] = x[..., a] * torch.cos(angle) - x[..., b] * torch.sin(angle)
            y[..., b] = x[..., b] * torch.cos(angle) + x[..., a] * torch.sin(angle)
            size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
        return y, size

    # The norm: a sum of d squares, a mean, a root, a quotient and two products, (d / 2 + 6) e of the
    # value; cos and sin, of an angle whose turn is exact to 2^-53 of its number of turns and then rounded
    # to fp32 in (-1, 1] half turns: pi e and some e of their own; two products and a sum.
    rel = ((d / 2 + 6) + (math.pi + 4 + 3 if rot else 0)) * EPS32 + float(pos.abs().max() if T else 0) * 2.0 ** -52
    (qo, qs), (ko, ks) = turned(q, qw), turned(k, kw)
    return (qo, qs * rel), (ko, ks * rel), (v.double(), torch.zeros_like(v, dtype=torch.float64))
