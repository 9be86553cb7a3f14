"""The operators on a paged cache whose speed this library is judged by, and their plain forms.

A case is one pass through the entry points of `paper_2505_14201_amd.flashd` that work on a cache
kept in pages: `attn_fwd_tree` (attention of each sequence's new tokens over its cached keys, the
new tokens seeing each other as a chain or as a tree), `cache_append` (norm and rotation of projected
q and k, k and v written into the pages) and `cache_fork`, `cache_reserve`, `cache_commit` (sequences
branch, get pages and give them back, keep accepted tokens).  With `own` false the same results come from elementary
torch operations.

Fields of a case: op ("tree", "append", "branch", "accept"), dtype of q, k, v and o, kv ("same": the
cache has that type too, "fp8": e4m3), B sequences, heads Hq and Hkv, d, page (keys of a page), lengths
lo..hi of the sequences in the cache, spread evenly, n (the most new tokens of a sequence; the
others have at least half of that), tree (drafted as a tree, otherwise a chain), layers, rot and
interleaved (the rotation), keep (the most accepted tokens).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FP8_SCALE = 2.0 ** -5       # of N(0, 1) values: +-14 sigma fit e4m3
EPS = 1e-6


def _case(name, op="tree", dtype="bf16", kv="same", B=1, Hq=32, Hkv=8, d=128, page=64, lo=1, hi=1,
          n=1, tree=False, layers=1, rot=128, interleaved=False, keep=1):
    c = {"op": op, "dtype": dtype, "kv": kv, "B": B, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page,
         "lo": lo, "hi": hi, "n": n, "tree": tree, "layers": layers, "rot": rot,
         "interleaved": interleaved, "keep": keep}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One user's token in a short context: the latency of a single step.
        _case("token_short", page=16, lo=1000, hi=1000),
        # The step of a serving loop: a token for each of 64 sequences of very different lengths.
        _case("tokens_ragged", B=64, lo=500, hi=8192),
        # The same from a cache kept in fp8, four drafted tokens a sequence.
        _case("drafts_fp8", kv="fp8", B=64, lo=500, hi=8192, n=4, tree=True),
        # Checking drafted trees of up to 16 tokens: 64 query rows for each head of the cache.
        _case("trees_ragged", B=32, page=32, lo=500, hi=8192, n=16, tree=True),
        # Wide trees of a model with heads of 64 and one query head to a cached head.
        _case("trees_wide_f16", dtype="f16", B=8, Hq=16, Hkv=16, d=64, page=16, lo=100, hi=4000,
              n=61, tree=True),
        # One tree far into a context of 128 K: one sequence has to fill the chip.
        _case("tree_long", page=128, lo=131000, hi=131000, n=12, tree=True),
        # Chunks of prompts behind what is cached already: the largest call, products bound it.
        _case("prompt_chunks", B=4, lo=2000, hi=7000, n=1000),
        # A token each of 64 sequences: norm, rotation and cache write of a decode step.
        _case("append_tokens", op="append", B=64, lo=500, hi=8192),
        # Whole prompts at once.
        _case("append_prompts", op="append", B=8, lo=0, hi=0, n=2000),
        # Drafts into an fp8 cache, heads of 64, half of each rotated in neighbouring pairs.
        _case("append_fp8", op="append", dtype="f16", kv="fp8", B=32, Hkv=4, d=64, page=16, lo=100,
              hi=4000, n=16, tree=True, rot=32, interleaved=True),
        # 32 sequences branch in two; shared pages that are part filled are copied, 8 layers.
        _case("branch", op="branch", B=32, lo=100, hi=4000, layers=8),
        # What was accepted of 16 drafts moves together in all of 32 layers.
        _case("accept", op="accept", B=32, page=16, lo=100, hi=1000, n=16, tree=True, layers=32,
              keep=6),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _bounded(c):
    """The case with its batch, then its lengths cut until it costs no more than the largest listed."""
    w = work(c)
    while w["flops"] > 3.0e11 or w["bytes"] > 1.0e9:
        c = dict(c, B=c["B"] // 2) if c["B"] > 1 else dict(c, hi=c["hi"] // 2, lo=c["lo"] // 2,
                                                          n=max(1, c["n"] // 2), keep=1)
        w = work(c)
    return c


def draw(rng):
    op = rng.choices(["tree", "append", "branch", "accept"], [55, 21, 12, 12])[0]
    hq, hkv = rng.choice([(32, 8), (32, 32), (16, 16), (32, 4), (12, 12), (8, 1), (16, 2), (10, 2)])
    d = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
    c = _case("", op=op, dtype=dtype, kv="fp8" if dtype != "f32" and rng.random() < 0.25 else "same",
              B=_log(rng, 1, 96), Hq=hq, Hkv=hkv, d=d, page=rng.choice([16, 32, 64, 128, 256]))
    if op == "tree":
        c["hi"] = _log(rng, 1, 131072 if c["B"] <= 4 else 16384)
        c["lo"] = rng.randint(c["hi"] // 16, c["hi"])
        c["tree"] = rng.random() < 0.5
        c["n"] = _log(rng, 2, 100) if c["tree"] else rng.choice([1, 1, _log(rng, 2, 800)])
    elif op == "append":
        c["hi"] = _log(rng, 1, 8192)
        c["lo"] = rng.randint(0, c["hi"])
        c["n"] = rng.choice([1, _log(rng, 2, 24), _log(rng, 32, 2000)])
        c["rot"] = rng.choice([d, d, d // 2, 16])
        c["interleaved"] = rng.random() < 0.3
        c["tree"] = rng.random() < 0.3
    else:
        c["hi"] = _log(rng, 2, 8192)
        c["lo"] = rng.randint(0, c["hi"])
        c["layers"] = rng.choice([1, 4, 16, 28])
        c["n"] = _log(rng, 2, 48) if op == "accept" else 1
        c["keep"] = rng.randint(1, min(8, c["n"]))
        c["B"] = min(c["B"], 48)
        pool = lambda x: x["B"] * (x["hi"] + 3.0 * x["page"]) * hkv * d * x["layers"]    # noqa: E731
        while pool(c) > 2.5e8:
            c = dict(c, layers=max(1, c["layers"] // 2), hi=max(2, c["hi"] // 2), lo=c["lo"] // 2)
            if c["layers"] == 1 and c["hi"] == 2:
                c["B"] = max(1, c["B"] // 2)
    return _bounded(c)


def _spread(c):
    """The lengths in the cache and the numbers of new tokens of a case's sequences."""
    at = [math.modf((b + 1) * 0.6180339887498949)[0] for b in range(c["B"])]
    lens = [c["lo"] + int(round((c["hi"] - c["lo"]) * x)) for x in at]
    lens[0] = c["hi"]
    some = [max(1, c["n"] - int(c["n"] // 2 * x)) for x in at]
    some[-1] = c["n"]
    return lens, some


def _esz(c):
    return {"f32": 4, "f16": 2, "bf16": 2}[c["dtype"]]


def work(c):
    lens, some = _spread(c)
    esz = _esz(c)
    csz = 1 if c["kv"] == "fp8" else esz
    T, row = sum(some), c["Hkv"] * c["d"] * csz
    if c["op"] == "tree":
        # keys and values once, queries once, outputs once; the products of the visible pairs
        # (of a tree at least what a path of log2 n ancestors sees)
        inner = sum((m.bit_length() if c["tree"] else (m + 1) / 2) * m for m in some)
        pairs = sum(l * m for l, m in zip(lens, some)) + inner
        return {"bytes": 2 * row * sum(l + m for l, m in zip(lens, some)) + 2 * T * c["Hq"] * c["d"] * esz,
                "flops": 4 * c["Hq"] * c["d"] * pairs}
    if c["op"] == "append":
        return {"bytes": T * c["d"] * esz * (2 * c["Hq"] + 2 * c["Hkv"]) + 2 * T * row,
                "flops": 8 * T * c["d"] * (c["Hq"] + c["Hkv"])}
    # read once and written once, keys and values, in every layer
    if c["op"] == "branch":       # one of two branches copies what the last page holds
        rows = sum(l % c["page"] for l in lens)
    else:                         # the kept tokens past the first move (the first stays where it is)
        rows = sum(max(0, min(c["keep"], m) - 1) for m in some)
    tables = 8 * c["B"] * (c["hi"] // c["page"] + 2)
    return {"bytes": 4 * rows * row * c["layers"] + tables, "flops": 0}


def prepare(case, seed):
    """The tensors that a serving loop has in hand before the call."""
    c = dict(case)
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    cpu = torch.Generator().manual_seed(int(seed))
    dt = DTYPES[c["dtype"]]
    lens, some = _spread(c)
    B, T, page, d = c["B"], sum(some), c["page"], c["d"]
    start = [0]
    for m in some:
        start.append(start[-1] + m)

    def ints(x):
        return torch.as_tensor(x, dtype=torch.int32).to(dev)

    def normal(*shape):
        return torch.randn(*shape, device=dev, generator=gen, dtype=dt)

    # pages of the sequences, in no order; before "accept" and "branch" reserve() has yet to add some
    fresh = c["op"] in ("branch", "accept")
    cols = [-(-(l if fresh else l + m) // page) for l, m in zip(lens, some)]
    most = max(-(-(l + m) // page) for l, m in zip(lens, some))
    spare = 2 * B * (2 + c["n"] // page) if fresh else 3
    P = sum(cols) + spare
    order = torch.randperm(P, generator=cpu, dtype=torch.int64).to(torch.int32)
    table = torch.full((B, most), -1, dtype=torch.int32)
    refs = torch.zeros(P, dtype=torch.int32)
    at = 0
    for b, k in enumerate(cols):
        table[b, :k] = order[at:at + k]
        at += k
    refs[order[:at].long()] = 1

    s = {"c": c, "lens": ints(lens), "q_start": ints(start), "table": table.to(dev),
         "refs": refs.to(dev), "max_q": max(some), "kscale": FP8_SCALE if c["kv"] == "fp8" else 1.0}
    shape = (P, c["Hkv"], page, d) if c["op"] in ("tree", "append") else (c["layers"], P, c["Hkv"], page, d)
    for name in ("kcache", "vcache"):
        x = normal(*shape)
        s[name] = (x * (1 / FP8_SCALE)).to(torch.float8_e4m3fn) if c["kv"] == "fp8" else x
    s["vscale"] = s["kscale"]

    # drafted trees: each token continues an earlier one of its sequence, mostly a late one
    n = c["n"]
    parent = torch.zeros(B, n, dtype=torch.int64)
    seen = torch.zeros(B, n, n, dtype=torch.bool)
    seen[:, 0, 0] = True
    each = torch.arange(B)
    for i in range(1, n if c["tree"] else 0):
        far = torch.rand(B, generator=cpu).square() * min(i, 8)
        parent[:, i] = i - 1 - far.long().clamp(max=i - 1)
        seen[:, i] = seen[each, parent[:, i]]
        seen[:, i, i] = True
    s["tree"] = s["positions"] = None
    if c["tree"]:
        words = -(-n // 64)
        bits = torch.zeros(B, n, words * 64, dtype=torch.int64)
        bits[:, :, :n] = seen
        bits = (bits.view(B, n, words, 64) << torch.arange(64)).sum(-1)
        mine = torch.cat([bits[b, :m] for b, m in enumerate(some)])
        s["tree"] = mine.to(dev)
        depth = seen.sum(-1)
        s["positions"] = torch.cat([lens[b] + depth[b, :m] - 1 for b, m in enumerate(some)]).to(torch.int32).to(dev)

    if c["op"] == "tree":
        s["q"] = normal(T, c["Hq"], d)
        s["o"] = torch.zeros_like(s["q"])
        s["scale"] = 1.0 / math.sqrt(d)
    elif c["op"] == "append":
        # one projection's output holds q, k and v of a token side by side
        qkv = normal(T, c["Hq"] + 2 * c["Hkv"], d) * 3
        s["q"], s["k"], s["v"] = qkv.split([c["Hq"], c["Hkv"], c["Hkv"]], dim=1)
        s["q_out"] = torch.zeros(T, c["Hq"], d, dtype=dt, device=dev)
        s["q_weight"], s["k_weight"] = (1 + 0.1 * normal(2, d)).unbind(0)
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])).float().to(dev)
    elif c["op"] == "branch":
        # twice as many sequences: each goes on in two
        s["parent"] = torch.cat([torch.arange(B), torch.randperm(B, generator=cpu)]).to(torch.int32).to(dev)
        s["refs0"] = s["refs"].clone()
        s["table_out"] = torch.empty(2 * B, most, dtype=torch.int32, device=dev)
        s["lens_out"] = torch.empty(2 * B, dtype=torch.int32, device=dev)
        s["q_start"] = torch.arange(2 * B + 1, dtype=torch.int32, device=dev)
        s["report"] = torch.empty(2 * B + 1, dtype=torch.int32, device=dev)
    else:
        # the accepted tokens are a path from the root on
        keep = torch.full((B, c["keep"]), 0, dtype=torch.int32)
        n_keep = torch.zeros(B, dtype=torch.int32)
        for b, m in enumerate(some):
            k = min(c["keep"], m)
            late = 1 + torch.randperm(m - 1, generator=cpu)[:k - 1].sort().values if m > 1 else torch.zeros(0, dtype=torch.int64)
            keep[b, :k] = torch.cat([torch.zeros(1, dtype=torch.int64), late])[:k].to(torch.int32)
            n_keep[b] = k
        s["keep"], s["n_keep"] = keep.to(dev), n_keep.to(dev)
        s["lens_out"] = torch.empty(B, dtype=torch.int32, device=dev)
        s["report"] = torch.empty(B + 1, dtype=torch.int32, device=dev)
    return s


def _owner(s):
    """Sequence and place within it of every new token."""
    T = s["q"].shape[0]
    t = torch.arange(T, device=s["q"].device)
    b = torch.searchsorted(s["q_start"].long(), t, right=True) - 1
    return b, t - s["q_start"].long()[b]


def _plain_tree(s):
    c, q = s["c"], s["q"]
    B, G, n, d = c["B"], c["Hq"] // c["Hkv"], s["max_q"], c["d"]
    start, lens = s["q_start"].long(), s["lens"].long()
    some = start[1:] - start[:-1]
    at = (start[:-1, None] + torch.arange(n, device=q.device)).clamp(max=q.shape[0] - 1)      # [B, n]
    keys = s["table"].shape[1] * c["page"]
    pages = s["table"].long().clamp(min=0)

    def gathered(x):
        return x[pages].transpose(1, 2).reshape(B, c["Hkv"], keys, d).float()

    qq = q[at].float().view(B, n, c["Hkv"], G, d).permute(0, 2, 1, 3, 4).reshape(B, c["Hkv"], n * G, d)
    x = torch.matmul(qq, gathered(s["kcache"]).transpose(-1, -2)) * (s["scale"] * s["kscale"])
    rel = torch.arange(keys, device=q.device) - lens[:, None]                               # [B, keys]
    if s["tree"] is None:
        inner = rel[:, None, :] <= torch.arange(n, device=q.device)[:, None]
    else:
        words = s["tree"].shape[1]
        word = (rel // 64).clamp(0, words - 1)[:, None, :].expand(B, n, keys)
        inner = (s["tree"][at].gather(2, word) >> (rel % 64)[:, None, :]) & 1 > 0
        inner &= (rel < 64 * words)[:, None, :]
    seen = (rel < 0)[:, None, :] | (inner & (rel < some[:, None])[:, None, :])
    x = x.view(B, c["Hkv"], n, G, keys).masked_fill(~seen[:, None, :, None, :], float("-inf"))
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(B, c["Hkv"], n * G, keys), gathered(s["vcache"])).view(B, c["Hkv"], n, G, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o)) * s["vscale"]
    b, i = _owner(s)
    s["o"].copy_(o.permute(0, 2, 1, 3, 4).reshape(B, n, c["Hq"], d)[b, i])


def _plain_append(s):
    c = s["c"]
    b, i = _owner(s)
    key = s["lens"].long()[b] + i
    position = key if s["positions"] is None else s["positions"]
    angle = position.double()[:, None, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    half, rot = c["rot"] // 2, c["rot"]

    def turned(x, weight):
        x = x.float()
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
        y, rest = x[..., :rot], x[..., rot:]
        if c["interleaved"]:
            u, v = y[..., 0::2], y[..., 1::2]
            y = torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2)
        else:
            u, v = y[..., :half], y[..., half:]
            y = torch.cat([u * cos - v * sin, v * cos + u * sin], -1)
        return torch.cat([y, rest], -1)

    def stored(x, scale):
        to = s["kcache"].dtype
        return (x / scale).clamp(-448, 448).to(to) if c["kv"] == "fp8" else x.to(to)

    s["q_out"].copy_(turned(s["q"], s["q_weight"]))
    where = s["table"].long()[b, key // c["page"]], slice(None), key % c["page"]
    s["kcache"][where] = stored(turned(s["k"], s["k_weight"]), s["kscale"])
    s["vcache"][where] = stored(s["v"].float(), s["vscale"])


def _plain_fork(s):
    table, parent = s["table"], s["parent"].long()
    s["table_out"].copy_(table[parent])
    s["lens_out"].copy_(s["lens"][parent])
    refs = s["refs"]
    for_each = torch.ones_like(refs[:1])
    spare = refs.shape[0]                          # entries without a page are counted behind the last
    more = torch.zeros(spare + 1, dtype=torch.int32, device=refs.device)
    new, old = s["table_out"].flatten(), table.flatten()
    more.index_add_(0, torch.where(new < 0, spare, new), for_each.expand(new.numel()))
    more.index_add_(0, torch.where(old < 0, spare, old), -for_each.expand(old.numel()))
    refs += more[:-1]


def _plain_reserve(s, table, lens):
    c, refs = s["c"], s["refs"]
    page = c["page"]
    start, length = s["q_start"].long(), lens.long()
    some = start[1:] - start[:-1]
    # a sequence has exactly the pages of its keys: what lies behind goes back first
    col = torch.arange(table.shape[1], device=table.device)
    last = -(-(length + some) // page)
    gone = (table >= 0) & (col >= last[:, None])
    refs.index_add_(0, table.long().clamp(min=0).flatten(), -gone.flatten().to(torch.int32))
    table.masked_fill_(gone, -1)
    first = length // page
    part = length % page
    mine = table.long().gather(1, first.clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    page_of = mine.clamp(min=0)
    share = (some > 0) & (part > 0) & (mine >= 0) & (refs[page_of] > 1)
    # where nobody else holds the page, the first of those that share it keeps it
    each = torch.arange(length.shape[0], device=table.device)
    holders = torch.zeros_like(refs).index_add_(0, page_of, share.to(torch.int32))
    lowest = torch.full_like(refs, len(each)).long().scatter_reduce_(0, page_of, torch.where(share, each, len(each)), "amin")
    share &= (holders != refs)[page_of] | (lowest[page_of] != each)
    new = (table < 0) & (col >= first[:, None]) & (col < last[:, None]) & (some > 0)[:, None]
    wanted = torch.cat([share[:, None], new], 1)
    rank = (wanted.flatten().long().cumsum(0) - 1).view(wanted.shape)
    free = torch.sort((refs != 0).to(torch.int32), stable=True).indices
    missing = (wanted.sum() - (refs == 0).sum()).clamp(min=0)
    wanted &= missing == 0
    given = free[rank.clamp(0, free.numel() - 1)]
    share, new = wanted[:, 0], wanted[:, 1:]
    # shared pages that are part filled: their rows move to a page of the sequence's own
    b = share.nonzero()[:, 0]
    src, dst = mine[b], given[b, 0]
    held = (torch.arange(page, device=table.device) < part[b, None])[:, None, :, None]
    k, v, words = s["kcache"], s["vcache"], torch.int32
    k, v = k.view(words), v.view(words)            # whole rows as they are, whatever their type
    k[:, dst] = torch.where(held, k[:, src], k[:, dst])
    v[:, dst] = torch.where(held, v[:, src], v[:, dst])
    table.copy_(torch.where(new, given[:, 1:], table.long()))
    table[b, first[b]] = dst.to(torch.int32)
    refs.index_add_(0, src, -torch.ones_like(src, dtype=torch.int32))
    refs.copy_(refs + torch.zeros_like(refs).index_add_(0, given.flatten(), wanted.flatten().to(torch.int32)))
    s["report"][0] = missing
    s["report"][1:] = torch.where(share, mine, -torch.ones_like(mine))


def _plain_commit(s):
    table, page, lens = s["table"], s["c"]["page"], s["lens"].long()
    i = torch.arange(s["keep"].shape[1], device=table.device)
    b, i = (i < s["n_keep"][:, None]).nonzero().unbind(1)
    src, dst = lens[b] + s["keep"][b, i], lens[b] + i
    sp, dp = table.long()[b, src // page], table.long()[b, dst // page]
    k, v = s["kcache"].view(torch.int32), s["vcache"].view(torch.int32)     # whole rows as they are
    k[:, dp, :, dst % page] = k[:, sp, :, src % page]
    v[:, dp, :, dst % page] = v[:, sp, :, src % page]
    s["lens_out"].copy_(lens + s["n_keep"])


def run(s):
    op = s["c"]["op"]
    if own:
        from paper_2505_14201_amd import flashd
        if op == "tree":
            flashd.attn_fwd_tree(s["q"], s["kcache"], s["vcache"], s["o"], s["table"], s["lens"], s["q_start"],
                                 s["max_q"], s["scale"], tree=s["tree"], kscale=s["kscale"], vscale=s["vscale"])
            return {"o": s["o"]}
        if op == "append":
            flashd.cache_append(s["q"], s["k"], s["v"], s["q_out"], s["kcache"], s["vcache"], s["table"], s["lens"],
                                s["q_start"], positions=s["positions"], inv_freq=s["inv_freq"],
                                q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                                interleaved=s["c"]["interleaved"], kscale=s["kscale"], vscale=s["vscale"])
            return {"q": s["q_out"], "k": s["kcache"], "v": s["vcache"]}
        if op == "branch":
            s["refs"].copy_(s["refs0"])
            flashd.cache_fork(s["parent"], s["refs"], s["table"], s["lens"], s["table_out"], s["lens_out"])
            flashd.cache_reserve(s["kcache"], s["vcache"], s["refs"], s["table_out"], s["lens_out"], s["q_start"],
                                 s["report"])
            return {"k": s["kcache"], "v": s["vcache"], "refs": s["refs"], "table": s["table_out"],
                    "lens": s["lens_out"], "report": s["report"]}
        flashd.cache_reserve(s["kcache"], s["vcache"], s["refs"], s["table"], s["lens"], s["q_start"], s["report"])
        flashd.cache_commit(s["kcache"], s["vcache"], s["table"], s["lens"], s["q_start"], s["lens_out"],
                            keep=s["keep"], n_keep=s["n_keep"])
        return {"k": s["kcache"], "v": s["vcache"], "refs": s["refs"], "table": s["table"], "lens": s["lens_out"],
                "report": s["report"]}
    if op == "tree":
        _plain_tree(s)
        return {"o": s["o"]}
    if op == "append":
        _plain_append(s)
        return {"q": s["q_out"], "k": s["kcache"], "v": s["vcache"]}
    if op == "branch":
        s["refs"].copy_(s["refs0"])
        _plain_fork(s)
        _plain_reserve(s, s["table_out"], s["lens_out"])
        return {"k": s["kcache"], "v": s["vcache"], "refs": s["refs"], "table": s["table_out"],
                "lens": s["lens_out"], "report": s["report"]}
    _plain_reserve(s, s["table"], s["lens"])
    _plain_commit(s)
    return {"k": s["kcache"], "v": s["vcache"], "refs": s["refs"], "table": s["table"], "lens": s["lens_out"],
            "report": s["report"]}


def exact(case, seed):
    """The outputs that are computed numbers, in 64 bits, sequence by sequence and key by key as the
    operators are defined; None for copies and whole numbers."""
    s = prepare(case, seed)
    c = s["c"]
    lens, some = _spread(c)
    page = c["page"]
    if c["op"] in ("branch", "accept"):
        return None
    k, v = s["kcache"].double(), s["vcache"].double()
    if c["op"] == "tree":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        at = 0
        for b, (l, m) in enumerate(zip(lens, some)):
            j = torch.arange(l + m, device="cuda")
            p = s["table"][b].long()[j // page]
            kb, vb = k[p, :, j % page] * s["kscale"], v[p, :, j % page] * s["vscale"]      # [keys, Hkv, d]
            seen = torch.ones(m, l + m, dtype=torch.bool, device="cuda")
            if s["tree"] is None:
                seen[:, l:] = torch.tril(seen[:, l:])
            else:
                bits = s["tree"][at:at + m]
                seen[:, l:] = torch.stack([(bits[:, x // 64] >> (x % 64)) & 1 for x in range(m)], 1) > 0
            for h in range(c["Hq"]):
                g = h // (c["Hq"] // c["Hkv"])
                x = s["q"][at:at + m, h].double() @ kb[:, g].T.contiguous() * s["scale"]
                x.masked_fill_(~seen, -math.inf)
                x = torch.exp(x - torch.logsumexp(x, 1, keepdim=True))
                out[at:at + m, h] = torch.nan_to_num(x) @ vb[:, g].contiguous()
            at += m
        return {"o": out}
    q = torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda")
    t = torch.cat([torch.full((m,), b) for b, m in enumerate(some)]).cuda()
    key = torch.cat([torch.arange(l, l + m) for l, m in zip(lens, some)]).cuda()
    pos = key if s["positions"] is None else s["positions"].long()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       pos[:, None].double() * s["inv_freq"].double())[:, None]

    def turned(x, weight):
        x = x.double()
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * weight.double()
        r = c["rot"]
        z = x[..., :r].unflatten(-1, (r // 2, 2) if c["interleaved"] else (2, r // 2))
        z = torch.complex(*z.unbind(-1 if c["interleaved"] else -2)) * turn
        x[..., :r] = torch.stack([z.real, z.imag], -1 if c["interleaved"] else -2).flatten(-2)
        return x

    q.copy_(turned(s["q"], s["q_weight"]))
    where = s["table"].long()[t, key // page], slice(None), key % page
    most = 448.0 if c["kv"] == "fp8" else math.inf
    k[where] = (turned(s["k"], s["k_weight"]) / s["kscale"]).clamp(-most, most)
    v[where] = (s["v"].double() / s["vscale"]).clamp(-most, most)
    return {"q": q, "k": k, "v": v}
