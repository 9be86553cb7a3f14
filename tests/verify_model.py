"""Plain model of flashd_draft_verify: token by token in fp64 on the CPU."""
import math

import torch


def row_of(logits, t, heat):
    """The target's probabilities behind row t; None where there are none."""
    x = logits[t].double()
    x = torch.where(x.isnan(), -math.inf, x).clamp(max=float(torch.finfo(torch.float32).max))
    top = x.max()
    if top == -math.inf:
        return None
    if not heat > 0:
        return torch.zeros_like(x).index_fill_(0, (x == top).nonzero()[0], 1.0)
    p = torch.exp((x - top) / heat)
    p[x == -math.inf] = 0
    return p / p.sum()


def verify(logits, tokens, uniform, starts, max_keep, parent=None, draft=None, temperature=None):
    """keep, n_keep, next as lists, and the least distance of a random number from the border it was held against."""
    keep, counts, then, near = [], [], [], math.inf
    for b in range(len(starts) - 1):
        s, n = starts[b], starts[b + 1] - starts[b]
        if n == 0:
            keep.append([-1] * max_keep)
            counts.append(0)
            then.append(-1)
            continue
        heat = 1.0 if temperature is None else float(temperature[b])
        cur, path, r = 0, [0], row_of(logits, s, heat)
        for j in range(1, n):
            if len(path) == max_keep or (j - 1 if parent is None else int(parent[s + j])) != cur:
                continue
            x = int(tokens[s + j])
            inside = 0 <= x < logits.shape[1]
            p = float(r[x]) if r is not None and inside else 0.0
            q = torch.zeros(logits.shape[1], dtype=torch.float64)
            if draft is not None:
                q = draft[s + cur].double()
                q = torch.where(q > 0, q, 0.0)
            elif inside:
                q[x] = 1.0
            at = float(q[x]) if inside else 1.0
            u = float(uniform[s + j])
            near = min(near, abs(u * at - p)) if p > 0 else near
            if u * at < p:
                cur = j
                path.append(j)
                r = row_of(logits, s + j, heat)
            elif r is not None:
                rest = (r - q).clamp(min=0)
                if rest.sum() > 0:
                    r = rest / rest.sum()
        keep.append(path + [-1] * (max_keep - len(path)))
        counts.append(len(path))
        if r is None:
            then.append(-1)
            continue
        upto = r.cumsum(0)
        place = float(uniform[s]) * float(upto[-1])
        over = ((upto > place) & (r > 0)).nonzero()
        then.append(int(over[0]) if len(over) else int((r > 0).nonzero()[-1]))
        near = min(near, float((upto - place).abs().min()))
    return keep, counts, then, near


def random_call(some, V, dtype, tree=False, draft=None, heat=False, seed=0, extra=0):
    """Arguments of a call on the CPU: drafts that are accepted as a rule, by a model that is not the target."""
    gen = torch.Generator().manual_seed(seed)
    starts = [0]
    for m in some:
        starts.append(starts[-1] + m)
    T = starts[-1] + extra
    x = torch.randn(T, V, generator=gen) * 2
    logits = x.to(dtype)
    y = torch.softmax(x + 0.7 * torch.randn(T, V, generator=gen), 1)
    if draft is not None:
        y = y.to(draft)
    parent = torch.full((T,), -1, dtype=torch.int32)
    tokens = torch.zeros(T, dtype=torch.int32)
    for s, m in zip(starts, some):
        for j in range(1, m):
            far = int(torch.randint(1, min(j, 4) + 1, (1,), generator=gen)) if tree else 1
            parent[s + j] = j - far
            tokens[s + j] = int(torch.multinomial(y[s + j - far].float(), 1, generator=gen))
    temperature = torch.tensor([[0.7, 0.0, 1.5, 1.0, -1.0][b % 5] for b in range(len(some))]) if heat else None
    return dict(logits=logits, tokens=tokens, uniform=torch.rand(T, generator=gen), starts=starts,
                parent=parent if tree else None, draft=y if draft is not None else None, temperature=temperature)
