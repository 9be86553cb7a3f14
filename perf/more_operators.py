"""More operators of a serving loop on a paged cache whose speed this library is judged by, and their
plain forms: what happens to a step's new tokens, and to the cache, after the attention.

A case is one pass through an entry point of `paper_2505_14201_amd.flashd`:

  verify   `draft_verify`: which of the drafted tokens of each sequence stay, by rejection sampling
           against the target's probabilities from given random numbers, and the token that follows
  score    `cache_score`: the attention weight that the new tokens give to each cached key is added
           to the key's score (lse: each query's log-sum-exp, which the attention has left)
  evict    `cache_evict`: of each sequence and kv head the keys with the largest scores stay, moved
           together in their order, in every layer

With `own` false the same results come from elementary torch operations.  `verify` is computed in 64
bits there: the boundaries between V tokens on the unit interval lie closer to each other than the
rounding of a sum in 32.

Fields of a case: op, dtype (of logits, or of q and the cache), B sequences, n (the most new tokens
of a sequence; the others have at least half of that), tree (drafted as a tree, otherwise a chain);
verify: V tokens, draft (type of the drafts' probabilities, "none": drafts were not sampled), heat
(a temperature for each sequence, some of them 0), keep (the most tokens that may stay);
score and evict: heads Hq and Hkv, d, page (keys of a page), lengths lo..hi of the sequences, spread
evenly; score: kv ("fp8": the cache is e4m3), decay (of the old scores; 0: they begin anew), votes
(new tokens have weights, some of them 0); evict: layers, budget (keys that stay), first and recent
(of them the first and last ones, whatever their scores).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FP8_SCALE = 2.0 ** -5       # of N(0, 1) values: +-14 sigma fit e4m3


def _verify(name, dtype="bf16", B=1, n=1, tree=False, V=32000, draft="none", heat=False, keep=0):
    c = {"op": "verify", "dtype": dtype, "B": B, "n": n, "tree": tree, "V": V, "draft": draft, "heat": heat,
         "keep": keep or n}
    return dict(c, name=name) if name else c


def _score(name, dtype="bf16", kv="same", B=1, Hq=32, Hkv=8, d=128, page=64, lo=1, hi=1, n=1, tree=False,
           decay=0.0, votes=False):
    c = {"op": "score", "dtype": dtype, "kv": kv, "B": B, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "lo": lo,
         "hi": hi, "n": n, "tree": tree, "decay": decay, "votes": votes}
    return dict(c, name=name) if name else c


def _evict(name, dtype="bf16", B=1, Hkv=8, d=128, page=64, lo=1, hi=1, layers=1, budget=1, first=0, recent=0):
    c = {"op": "evict", "dtype": dtype, "B": B, "Hkv": Hkv, "d": d, "page": page, "lo": lo, "hi": hi,
         "layers": layers, "budget": budget, "first": first, "recent": recent}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One user's chain of three drafts behind the last token: the latency of a step.
        _verify("verify_one", n=4),
        # 64 sequences, four drafts each, sampled from a smaller model whose probabilities were kept.
        _verify("verify_chains", B=64, n=5, V=131072, draft="f32"),
        # Trees of up to 16 tokens that a lookup proposed, an odd vocabulary, a temperature for each
        # sequence (with 0 the largest logit is what the target says).
        _verify("verify_trees_f16", dtype="f16", B=32, n=16, tree=True, V=50257, heat=True),
        # Trees whose tokens were sampled, siblings after each other: every refusal changes what is left.
        _verify("verify_trees_sampled", dtype="f32", B=8, n=31, tree=True, V=100003, draft="bf16", keep=8),
        # One user's token in a short context.
        _score("score_short", page=16, lo=1000, hi=1000),
        # A token for each of 64 sequences of very different lengths.
        _score("score_tokens", B=64, lo=500, hi=8192),
        # Trees of four drafts, an fp8 cache, and older votes count less and less.
        _score("score_drafts_fp8", kv="fp8", B=64, lo=500, hi=8192, n=4, tree=True, decay=0.97),
        # The last tokens of long prompts vote on what is kept of them, the latest the most.
        _score("score_votes", B=4, lo=10000, hi=32000, n=32, votes=True),
        # Every token of a chunk of a prompt votes: the products bound it.
        _score("score_prompts", B=4, lo=2000, hi=7000, n=1000),
        # A few keys of each of 16 sequences go to make room for the next ones, in one layer.
        _evict("evict_few", B=16, page=16, lo=1030, hi=1056, budget=1024, first=4, recent=64),
        # Of each of 8 prompts 1024 keys stay, in all of 8 layers.
        _evict("evict_prompts", B=8, lo=1500, hi=8000, layers=8, budget=1024, first=4, recent=32),
        # A long context is cut to a quarter.
        _evict("evict_long", page=128, lo=65536, hi=65536, layers=2, budget=16384, first=4, recent=256),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choices(["verify", "score", "evict"], [35, 40, 25])[0]
    if op == "verify":
        tree = rng.random() < 0.5
        c = _verify("", dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), B=_log(rng, 1, 96),
                    n=_log(rng, 2, 40) if tree else _log(rng, 1, 10), tree=tree, V=_log(rng, 200, 200000),
                    draft=rng.choice(["none", "none", "f32", "bf16", "f16"]), heat=rng.random() < 0.4)
        c["keep"] = rng.choice([c["n"], c["n"], rng.randint(1, c["n"])])
        while work(c)["bytes"] > 1.5e8:
            c["B"], c["V"] = max(1, c["B"] // 2), max(200, c["V"] * 2 // 3)
        return c
    hq, hkv = rng.choice([(32, 8), (32, 32), (16, 16), (32, 4), (12, 12), (8, 1), (16, 2), (10, 2)])
    d, page = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128, 256])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
    if op == "score":
        c = _score("", dtype=dtype, kv="fp8" if dtype != "f32" and rng.random() < 0.25 else "same", B=_log(rng, 1, 96),
                   Hq=hq, Hkv=hkv, d=d, page=page, tree=rng.random() < 0.4,
                   decay=rng.choice([0.0, 0.0, 1.0, 0.9]), votes=rng.random() < 0.3)
        c["hi"] = _log(rng, 1, 131072 if c["B"] <= 4 else 16384)
        c["lo"] = rng.randint(c["hi"] // 16, c["hi"])
        c["n"] = _log(rng, 2, 100) if c["tree"] else rng.choice([1, 1, _log(rng, 2, 800)])
        w = work(c)
        while w["flops"] > 1.5e11 or w["bytes"] > 6.0e8:
            c = dict(c, B=c["B"] // 2) if c["B"] > 1 else dict(c, hi=c["hi"] // 2, lo=c["lo"] // 2, n=max(1, c["n"] // 2))
            w = work(c)
        return c
    c = _evict("", dtype=dtype, B=min(48, _log(rng, 1, 96)), Hkv=hkv, d=d, page=page, layers=rng.choice([1, 1, 4, 12]))
    c["hi"] = _log(rng, 2, 32768 if c["B"] <= 4 else 8192)
    c["lo"] = rng.randint(c["hi"] // 8, c["hi"])
    pool = lambda x: x["B"] * (x["hi"] + 2.0 * page) * hkv * d * x["layers"]    # noqa: E731
    share = rng.random()
    c["budget"] = _log(rng, 1, c["hi"])
    while pool(c) > 2.5e8 or work(c)["bytes"] > 5.0e8:
        if c["layers"] > 1:
            c["layers"] //= 2
        elif c["B"] > 1:
            c["B"] //= 2
        else:
            c["hi"], c["lo"], c["budget"] = c["hi"] // 2, c["lo"] // 2, max(1, c["budget"] // 2)
    c["first"] = rng.choice([0, 0, 1, int(share * c["budget"])])
    c["recent"] = rng.choice([0, 1, rng.randint(0, c["budget"])])
    return c


def _spread(c):
    """The lengths in the cache and the numbers of new tokens of a case's sequences."""
    at = [math.modf((b + 1) * 0.6180339887498949)[0] for b in range(c["B"])]
    lens = [c.get("lo", 0) + int(round((c.get("hi", 0) - c.get("lo", 0)) * x)) for x in at]
    lens[0] = c.get("hi", 0)
    n = c.get("n", 0)
    some = [max(1, n - int(n // 2 * x)) for x in at]
    some[-1] = n
    return lens, some


def _esz(c):
    return {"f32": 4, "f16": 2, "bf16": 2}[c["dtype"]]


def work(c):
    lens, some = _spread(c)
    T, esz = sum(some), _esz(c)
    if c["op"] == "verify":
        # every row of logits once; of the drafts' probabilities the row where a sequence's drafts end
        drafted = 0 if c["draft"] == "none" else c["B"] * c["V"] * {"f32": 4, "f16": 2, "bf16": 2}[c["draft"]]
        return {"bytes": T * c["V"] * esz + drafted + 16 * T + 4 * c["B"] * (c["keep"] + 2), "flops": 4 * T * c["V"]}
    if c["op"] == "score":
        # keys once, queries once, old scores read and new ones written; the products of the visible
        # pairs (of a tree at least what a path of log2 n ancestors sees)
        row = c["Hkv"] * c["d"] * (1 if c["kv"] == "fp8" else esz)
        keys = sum(l + m for l, m in zip(lens, some))
        inner = sum((m.bit_length() if c["tree"] else (m + 1) / 2) * m for m in some)
        pairs = sum(l * m for l, m in zip(lens, some)) + inner
        return {"bytes": keys * (row + 4 * c["Hkv"]) + (4 * c["Hkv"] * sum(lens) if c["decay"] else 0)
                + T * c["Hq"] * (c["d"] * esz + 4), "flops": 2 * c["Hq"] * c["d"] * pairs}
    # scores once; the keys and values that stay behind the first ones, and their scores, move
    units, some = c["layers"] * c["Hkv"], [l for l in lens if l > c["budget"]]
    stay = len(some) * max(0, c["budget"] - c["first"])
    return {"bytes": units * (4 * sum(some) + stay * (4 * c["d"] * esz + 4)) + 8 * c["B"], "flops": 0}


def prepare(case, seed):
    """The tensors that a serving loop has in hand before the call."""
    c = dict(case)
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    cpu = torch.Generator().manual_seed(int(seed))
    dt = DTYPES[c["dtype"]]
    lens, some = _spread(c)
    B, T = c["B"], sum(some)
    start = [0]
    for m in some:
        start.append(start[-1] + m)

    def ints(x):
        return torch.as_tensor(x, dtype=torch.int32).to(dev)

    def normal(*shape, dtype=None):
        return torch.randn(*shape, device=dev, generator=gen, dtype=dtype or dt)

    s = {"c": c, "q_start": ints(start), "lens": ints(lens)}

    # drafted trees: each token continues an earlier one of its sequence, mostly a late one
    parent = s["tree"] = s["parent"] = None
    if c.get("tree"):
        n = c["n"]
        parent = torch.full((B, n), -1, dtype=torch.int64)
        for i in range(1, n):
            far = torch.rand(B, generator=cpu).square() * min(i, 8)
            parent[:, i] = i - 1 - far.long().clamp(max=i - 1)
        s["parent"] = ints(torch.cat([parent[b, :m] for b, m in enumerate(some)]))

    if c["op"] == "verify":
        V = c["V"]
        # a few likely tokens in front of a long tail, as a trained model's logits have them
        x = normal(T, V, dtype=torch.float32) * 1.5
        top = torch.randint(0, V // 12, (T, 12), device=dev, generator=gen) + torch.arange(12, device=dev) * (V // 12)
        x.scatter_add_(1, top, 6 + 4 * torch.rand(T, 12, device=dev, generator=gen))
        s["logits"] = x.to(dt)
        # the drafts come from another model's opinion on the token before them
        y = torch.softmax(x.add_(torch.randn(T, V, device=dev, generator=gen), alpha=0.6), 1)
        if c["draft"] != "none":
            y = y.to(DTYPES[c["draft"]])
        before = torch.arange(T) - 1
        if parent is not None:
            at = torch.tensor(start[:-1])[:, None] + parent.clamp(min=0)
            before = torch.cat([at[b, :m] for b, m in enumerate(some)])
        before = before.clamp(min=0).to(dev)
        s["tokens"] = torch.multinomial(y.float()[before], 1, generator=gen)[:, 0].to(torch.int32)
        s["draft"] = None if c["draft"] == "none" else y
        s["uniform"] = torch.rand(T, device=dev, generator=gen)
        s["temperature"] = None
        if c["heat"]:
            s["temperature"] = torch.tensor([0.7, 1.0, 0.0, 1.3])[torch.randint(0, 4, (B,), generator=cpu)].to(dev)
        s["keep"] = torch.empty(B, c["keep"], dtype=torch.int32, device=dev)
        s["n_keep"] = torch.empty(B, dtype=torch.int32, device=dev)
        s["next"] = torch.empty(B, dtype=torch.int32, device=dev)
        return s

    # pages of the sequences, in no order
    page, d, Hkv = c["page"], c["d"], c["Hkv"]
    cols = [-(-(l + m) // page) for l, m in zip(lens, some)]
    P, most = sum(cols) + 3, max(cols)
    order = torch.randperm(P, generator=cpu, dtype=torch.int64).to(torch.int32)
    table = torch.full((B, most), -1, dtype=torch.int32)
    refs = torch.zeros(P, dtype=torch.int32)
    at = 0
    for b, k in enumerate(cols):
        table[b, :k] = order[at:at + k]
        at += k
    refs[order[:at].long()] = 1
    s["table"], s["refs"] = table.to(dev), refs.to(dev)

    if c["op"] == "evict":
        shape = (c["layers"], P, Hkv, page, d)
        s["kcache"], s["vcache"] = normal(*shape), normal(*shape)
        # sums of weights: most keys have little, some very much
        s["score0"] = torch.exp(2.5 * normal(c["layers"], B, Hkv, most * page, dtype=torch.float32))
        s["score"] = torch.empty_like(s["score0"])
        s["lens_out"] = torch.empty(B, dtype=torch.int32, device=dev)
        return s

    fp8 = c["kv"] == "fp8"
    s["kscale"] = FP8_SCALE if fp8 else 1.0
    k = normal(P, Hkv, page, d)
    s["kcache"] = (k * (1 / FP8_SCALE)).to(torch.float8_e4m3fn) if fp8 else k
    s["q"] = normal(T, c["Hq"], d) * 1.5
    s["scale"] = 1.0 / math.sqrt(d)
    if parent is not None:
        n = c["n"]
        seen = torch.zeros(B, n, n, dtype=torch.bool)
        seen[:, 0, 0] = True
        each = torch.arange(B)
        for i in range(1, n):
            seen[:, i] = seen[each, parent[:, i]]
            seen[:, i, i] = True
        words = -(-n // 64)
        bits = torch.zeros(B, n, words * 64, dtype=torch.int64)
        bits[:, :, :n] = seen
        bits = (bits.view(B, n, words, 64) << torch.arange(64)).sum(-1)
        s["tree"] = torch.cat([bits[b, :m] for b, m in enumerate(some)]).to(dev)
    s["votes"] = None
    if c["votes"]:
        # the latest tokens count most, and some do not count
        w = torch.linspace(0.1, 1.0, T)
        w[::7] = 0.0
        s["votes"] = w.to(dev)
    s["score0"] = torch.rand(B, Hkv, most * page, device=dev, generator=gen)
    s["score"] = torch.zeros_like(s["score0"])
    # what the attention has left
    lse = torch.empty(T, c["Hq"], device=dev)
    for b, (at, to) in enumerate(zip(start, start[1:])):
        x = _scores(s, b, at, to, lens[b], torch.float32)
        lse[at:to] = torch.logsumexp(x, -1).permute(2, 0, 1).reshape(to - at, c["Hq"])
    s["lse"] = lse
    return s


def _scores(s, b, at, to, length, dtype):
    """Scores [Hkv, G, new tokens, keys] of a sequence, -inf where a token does not see a key."""
    c = s["c"]
    n, dev = to - at, s["q"].device
    j = torch.arange(length + n, device=dev)
    k = s["kcache"][s["table"][b].long()[j // c["page"]], :, j % c["page"]].to(dtype)     # [keys, Hkv, d]
    q = s["q"][at:to].to(dtype).view(n, c["Hkv"], -1, c["d"]).permute(1, 2, 0, 3)          # [Hkv, G, n, d]
    G = q.shape[1]
    x = torch.matmul(q.reshape(c["Hkv"], G * n, c["d"]), k.permute(1, 2, 0).contiguous())
    x = x.mul_(s["scale"] * s["kscale"]).view(c["Hkv"], G, n, length + n)
    i = torch.arange(n, device=dev)
    if s["tree"] is None:
        seen = i[:, None] >= i
    else:
        seen = (s["tree"][at:to][:, i // 64] >> (i % 64)) & 1 > 0
    x[..., length:].masked_fill_(~seen, -math.inf)
    return x


def _plain_score(s):
    c = s["c"]
    lens, some = _spread(c)
    at = 0
    for b, (l, m) in enumerate(zip(lens, some)):
        to = at + m
        lse = s["lse"][at:to].view(m, c["Hkv"], -1).permute(1, 2, 0)
        w = _scores(s, b, at, to, l, torch.float32).sub_(lse[..., None]).exp_()
        if s["votes"] is not None:
            w.mul_(s["votes"][at:to, None])
        w = w.sum((1, 2))
        s["score"][b, :, :l] = (s["score"][b, :, :l] * c["decay"] if c["decay"] else 0.0) + w[:, :l]
        s["score"][b, :, l:l + m] = w[:, l:]
        at = to


def _plain_verify(s):
    c = s["c"]
    B, n, V = c["B"], c["n"], c["V"]
    dev = s["logits"].device
    start, each = s["q_start"].long(), torch.arange(B, device=dev)
    some = start[1:] - start[:-1]
    heat = torch.ones(B, dtype=torch.float64, device=dev) if s["temperature"] is None else s["temperature"].double()
    cur = torch.zeros_like(each)
    s["keep"].fill_(-1)
    s["keep"][:, 0] = 0
    kept = torch.ones_like(each)

    def row_of(at):
        """The target's probabilities behind the tokens `at` of the sequences."""
        x = s["logits"][start[:-1] + at].double()
        top = x.amax(1, keepdim=True)
        p = torch.exp((x - top) / torch.where(heat > 0, heat, torch.ones_like(heat))[:, None])
        p = p / p.sum(1, keepdim=True)
        first = torch.zeros_like(p).scatter_(1, (x == top).int().argmax(1, keepdim=True), 1.0)
        return torch.where((heat > 0)[:, None], p, first)

    left = row_of(cur)
    for j in range(1, n):
        row = (start[:-1] + j).clamp(max=s["tokens"].shape[0] - 1)
        before = j - 1 if s["parent"] is None else s["parent"].long()[row]
        asked = (j < some) & (cur == before) & (kept < c["keep"])
        x = s["tokens"].long()[row][:, None]
        p = left.gather(1, x)[:, 0]
        if s["draft"] is None:
            q = torch.ones_like(p)
            rest = left.scatter(1, x, 0.0)
        else:
            whole = s["draft"][start[:-1] + cur].double()
            q = whole.gather(1, x)[:, 0]
            rest = (left - whole).clamp(min=0)
        yes = asked & (s["uniform"][row].double() * q < p)
        total = rest.sum(1, keepdim=True)
        rest = torch.where(total > 0, rest / total, left)
        cur = torch.where(yes, j, cur)
        s["keep"][each, torch.where(yes, kept, 0)] = torch.where(yes, j, 0).to(torch.int32)
        kept = kept + yes
        left = torch.where(yes[:, None], row_of(cur), torch.where(asked[:, None], rest, left))
    upto = left.cumsum(1)
    wanted = s["uniform"][start[:-1]].double()[:, None] * upto[:, -1:]
    s["next"].copy_(((upto > wanted) & (left > 0)).int().argmax(1))
    s["n_keep"].copy_(kept)


def _plain_evict(s):
    c = s["c"]
    page, layers, Hkv, most = c["page"], c["layers"], c["Hkv"], s["score"].shape[-1]
    lens = _spread(c)[0]
    y = torch.arange(layers, device=s["table"].device)[:, None, None]
    h = torch.arange(Hkv, device=y.device)[:, None]
    for b, l in enumerate(lens):
        m = min(c["budget"], most)
        s["lens_out"][b] = min(l, m)
        if l <= m:
            continue
        first = min(c["first"], m)
        recent = min(c["recent"], m - first)
        x = s["score"][:, b, :, :l].clone()
        x[..., :first] = math.inf
        x[..., l - recent:] = math.inf
        stay = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :m].sort(-1).values   # [layers, Hkv, m]
        to = torch.arange(m, device=y.device)
        src, dst = s["table"][b].long()[stay // page], s["table"][b].long()[to // page]
        for name in ("kcache", "vcache"):
            s[name][y, dst, h, to % page] = s[name][y, src, h, stay % page]
        s["score"][:, b, :, :m] = s["score"][:, b].gather(-1, stay)


def run(s):
    c = s["c"]
    if c["op"] == "verify":
        if own:
            from paper_2505_14201_amd import flashd
            flashd.draft_verify(s["logits"], s["tokens"], s["uniform"], s["q_start"], s["keep"], s["n_keep"], s["next"],
                                parent=s["parent"], draft=s["draft"], temperature=s["temperature"])
        else:
            _plain_verify(s)
        return {"keep": s["keep"], "n_keep": s["n_keep"], "next": s["next"]}
    if c["op"] == "score":
        if c["decay"]:
            s["score"].copy_(s["score0"])           # each pass adds to the same scores
        if own:
            from paper_2505_14201_amd import flashd
            flashd.cache_score(s["q"], s["kcache"], s["table"], s["lens"], s["q_start"], s["lse"], s["score"], s["scale"],
                               tree=s["tree"], row_weight=s["votes"], decay=c["decay"], kscale=s["kscale"])
        else:
            _plain_score(s)
        return {"score": s["score"]}
    s["score"].copy_(s["score0"])                   # each pass chooses by the same scores
    if own:
        from paper_2505_14201_amd import flashd
        flashd.cache_evict(s["kcache"], s["vcache"], s["refs"], s["table"], s["lens"], s["score"], s["lens_out"],
                           c["budget"], first=c["first"], recent=c["recent"])
    else:
        _plain_evict(s)
    return {"k": s["kcache"], "v": s["vcache"], "score": s["score"], "lens": s["lens_out"]}


def exact(case, seed):
    """Scores in 64 bits, head by head from the definition; None for copies and whole numbers."""
    if case["op"] != "score":
        return None
    s = prepare(case, seed)
    c = s["c"]
    lens, some = _spread(c)
    out = (s["score0"] if c["decay"] else s["score"]).double()
    G, at = c["Hq"] // c["Hkv"], 0
    for b, (l, m) in enumerate(zip(lens, some)):
        out[b, :, :l] *= c["decay"]
        out[b, :, l:l + m] = 0
        j = torch.arange(l + m, device="cuda")
        pages = s["table"][b].long()[j // c["page"]]
        hidden = torch.zeros(m, l + m, dtype=torch.bool, device="cuda")
        if s["tree"] is None:
            hidden[:, l:] = torch.triu(torch.ones(m, m, dtype=torch.bool, device="cuda"), 1)
        else:
            bits = s["tree"][at:at + m]
            hidden[:, l:] = torch.stack([(bits[:, x // 64] >> (x % 64)) & 1 for x in range(m)], 1) == 0
        votes = torch.ones(m, dtype=torch.float64, device="cuda") if s["votes"] is None else s["votes"][at:at + m].double()
        for h in range(c["Hkv"]):
            k = s["kcache"][pages, h, j % c["page"]].double() * s["kscale"]
            for g in range(G):
                x = s["q"][at:at + m, h * G + g].double() @ k.T.contiguous() * s["scale"]
                x = torch.exp(x - s["lse"][at:at + m, h * G + g, None].double())
                out[b, h, :l + m] += votes @ x.masked_fill_(hidden, 0.0)
        at += m
    return {"score": out}
