"""flashd_draft_verify against a plain fp64 model.  Its results are whole numbers and have to be equal: a random number
that falls within 1e-12 of a border (sums of up to 2e5 numbers in fp64 differ by less) would not be decided, and none of the
inputs has one."""
import math

import pytest
import torch

from paper_2505_14201_amd import flashd
from tests.verify_model import random_call, verify

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def ints(*shape):
    return torch.full(shape, 77, dtype=torch.int32, device="cuda")


def call(a, max_keep, logits=None, draft=None, **kw):
    """keep, n_keep, next of the operator as lists."""
    B = len(a["starts"]) - 1
    keep, n, then = ints(B, max_keep), ints(B), ints(B)
    gpu = {k: None if a[k] is None else a[k].cuda() for k in ("tokens", "uniform", "parent", "temperature")}
    draft = draft if draft is not None or a["draft"] is None else a["draft"].cuda()
    flashd.draft_verify(a["logits"].cuda() if logits is None else logits, gpu["tokens"], gpu["uniform"],
                        torch.tensor(a["starts"], dtype=torch.int32).cuda(), keep, n, then, parent=gpu["parent"],
                        draft=draft, temperature=gpu["temperature"], **kw)
    return keep.tolist(), n.tolist(), then.tolist()


def check(a, max_keep, **kw):
    got = call(a, max_keep, **kw)
    *want, near = verify(max_keep=max_keep, **a)
    assert near > 1e-12
    assert got == tuple(want)
    return got


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("draft", [None, F32, F16, BF16])
@pytest.mark.parametrize("tree", [False, True])
def test_types_and_kinds(dtype, draft, tree):
    some = [5, 1, 0, 9, 3, 17]
    for seed, V in ((1, 1000), (2, 4097)):
        a = random_call(some, V, dtype, tree, draft, heat=seed == 2, seed=seed)
        check(a, 20)
        a["uniform"] *= 2.0 ** -10           # most are kept
        assert max(check(a, 20)[1]) > 1


@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 255, 256, 257, 4095, 4096, 4097, 8191, 50257, 131072])
@pytest.mark.parametrize("draft", [None, F32])
def test_vocabularies(V, draft):
    for tree in (False, True):
        check(random_call([4, 2, 6], V, BF16, tree, draft, seed=V), 6)


@pytest.mark.parametrize("n", [63, 64, 65, 66, 130, 300])
@pytest.mark.parametrize("draft", [None, BF16])
def test_many_tokens(n, draft):
    """More tokens than lanes of a wavefront; a wide tree whose refused tokens are many, and a deep one."""
    check(random_call([n, 3], 64, F32, True, draft, seed=n), n)
    a = random_call([n], 50, F32, True, draft, seed=n + 1)
    a["parent"] = torch.zeros(n, dtype=torch.int32)          # all of them continue the first
    a["tokens"] = (torch.arange(n) % 50).to(torch.int32)     # some twice
    a["uniform"][1:] = 0.999
    check(a, n)


@pytest.mark.parametrize("n", [200, 330])
@pytest.mark.parametrize("top", [0.0, 14.0])
def test_refused_tokens_of_many_chunks(n, top):
    """Fewer and more of them than have a place on the chip; with and without one that is most of its chunk."""
    a = random_call([n, 2], 9001, BF16, True, None, seed=n)
    a["parent"][:n] = 0
    a["tokens"][:n] = (torch.arange(n) * 27 % 9001).to(torch.int32)
    a["logits"][0, 27 * 5] += top
    a["uniform"][1:n] = 0.99999994
    _, kept, _ = check(a, 4)
    assert kept[0] == 1


def test_many_sequences():
    gen = torch.Generator().manual_seed(3)
    some = torch.randint(0, 4, (4096,), generator=gen).tolist()
    check(random_call(some, 40, F16, False, None, heat=True, seed=4), 4)


def test_strides_and_odd_addresses():
    a = random_call([5, 4], 501, BF16, True, F32, seed=5)
    wide = torch.full((9, 777), float("nan"), dtype=BF16, device="cuda")
    wide[:, 3:504] = a["logits"]
    deep = torch.full((9, 603), float("nan"), dtype=F32, device="cuda")
    deep[:, 1:502] = a["draft"]
    check(a, 5, logits=wide[:, 3:504], draft=deep[:, 1:502])


@pytest.mark.parametrize("max_keep", [1, 2, 3])
def test_the_path_ends_at_max_keep(max_keep):
    a = random_call([6, 6, 1], 100, F32, False, None, seed=6)
    a["uniform"][:] = 0.0
    _, n, _ = check(a, max_keep)
    assert n == [max_keep, max_keep, 1]


def test_rows_behind_the_last_sequence_and_numbers_that_are_none():
    a = random_call([4, 5], 200, F32, True, F32, seed=7, extra=6)
    a["logits"][9:] = float("nan")
    a["tokens"][2] = 200
    a["tokens"][5] = -1
    a["parent"][3] = 3                     # itself
    a["parent"][6] = 100
    check(a, 5)
    # starts that run past the rows, or backwards: every sequence stays inside
    keep, n, then = ints(3, 4), ints(3), ints(3)
    flashd.draft_verify(a["logits"].cuda(), a["tokens"].cuda(), a["uniform"].cuda(),
                        torch.tensor([-5, 1000000, 3, -7], dtype=torch.int32).cuda(), keep, n, then)
    assert n.tolist()[1:] == [0, 0] and 1 <= n.tolist()[0] <= 4


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("heat", [None, 0.0, 1.0, 0.3, math.inf, 1e-30, math.nan])
def test_infinities_nan_and_equal_logits(dtype, heat):
    a = random_call([3, 3, 3, 3, 3], 5000, dtype, False, None, seed=8)
    x = a["logits"]
    x[0:3, ::2] = -math.inf
    x[3:6, 1::3] = math.nan
    x[6:9] = -math.inf                     # nothing at all
    x[9:12, [17, 4500]] = math.inf         # they share everything
    x[12:15] = 0.0
    x[12:15, [4100, 4200]] = 3.0
    if heat is not None:
        a["temperature"] = torch.full((5,), heat)
    _, n, then = check(a, 3)
    assert (n[2], then[2]) == (1, -1)


def test_a_draft_that_is_the_target_is_always_kept():
    a = random_call([9, 9], 300, F32, False, F32, seed=9)
    a["draft"] = torch.softmax(a["logits"].double(), 1).float() * (1 - 2.0 ** -20)
    for s in (0, 9):
        for j in range(1, 9):
            a["tokens"][s + j] = int(torch.multinomial(a["draft"][s + j - 1], 1))
    assert call(a, 9)[1] == [9, 9]


@pytest.mark.parametrize("draft", [None, F32])
def test_the_tokens_have_the_targets_probabilities(draft):
    """Two drafts behind the first token, many times: the token that follows it (a draft kept, or the one drawn) is
    distributed as the target says.  Chi square of 11 degrees of freedom: above 45 once in 2e5 draws."""
    N, V = 4096, 12
    gen = torch.Generator().manual_seed(10)
    row = torch.randn(V, generator=gen)
    q = torch.softmax(row + torch.randn(V, generator=gen), 0)
    a = dict(logits=row.repeat(3 * N, 1), uniform=torch.rand(3 * N, generator=gen), starts=list(range(0, 3 * N + 1, 3)),
             parent=torch.tensor([-1, 0, 0], dtype=torch.int32).repeat(N), draft=None if draft is None else q.repeat(3 * N, 1),
             tokens=torch.multinomial(q, 3 * N, replacement=True, generator=gen).to(torch.int32), temperature=None)
    if draft is None:
        a["tokens"] = torch.tensor([0, 3, 7], dtype=torch.int32).repeat(N)
    keep, n, then = call(a, 2)
    first = [then[b] if n[b] == 1 else int(a["tokens"][3 * b + keep[b][1]]) for b in range(N)]
    count = torch.bincount(torch.tensor(first), minlength=V).double()
    want = torch.softmax(row.double(), 0) * N
    assert float(((count - want) ** 2 / want).sum()) < 45


def test_a_captured_call_is_replayed_with_other_numbers():
    a = random_call([5, 3, 8], 4500, BF16, True, F32, seed=11)
    other = random_call([5, 3, 8], 4500, BF16, True, F32, seed=12)
    B, T = 3, 16
    names = ("logits", "tokens", "uniform", "parent", "draft")
    g = {k: a[k].cuda() for k in names}
    starts = torch.tensor(a["starts"], dtype=torch.int32).cuda()
    keep, n, then = ints(B, 8), ints(B), ints(B)
    ws = torch.empty(flashd.verify_workspace_bytes(T, 4500), dtype=torch.uint8, device="cuda")

    def run(**kw):
        flashd.draft_verify(g["logits"], g["tokens"], g["uniform"], starts, keep, n, then, parent=g["parent"], draft=g["draft"], **kw)

    run(workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(workspace=ws)
    for x in (a, other, a, other):
        for k in names:
            g[k].copy_(x[k])
        graph.replay()
        torch.cuda.synchronize()
        got = keep.tolist(), n.tolist(), then.tolist()
        assert got == tuple(verify(max_keep=8, **x)[:3])
        run()                              # an eager call between replays, with the stream's own workspace
        assert (keep.tolist(), n.tolist(), then.tolist()) == got
    with pytest.raises(flashd.FlashdError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            run()


def test_other_streams_and_no_rows():
    a = random_call([5, 4], 3000, F16, False, None, seed=13)
    g = {k: a[k].cuda() for k in ("logits", "tokens", "uniform")}
    starts, keep, n, then = torch.tensor(a["starts"], dtype=torch.int32).cuda(), ints(2, 5), ints(2), ints(2)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    flashd.draft_verify(g["logits"], g["tokens"], g["uniform"], starts, keep, n, then, stream=side)
    side.synchronize()
    assert (keep.tolist(), n.tolist(), then.tolist()) == tuple(verify(max_keep=5, **a)[:3])
    keep, n, then = ints(2, 3), ints(2), ints(2)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    flashd.draft_verify(torch.empty(0, 30, device="cuda"), none, torch.empty(0, device="cuda"),
                        torch.zeros(3, dtype=torch.int32, device="cuda"), keep, n, then)
    assert (keep.tolist(), n.tolist(), then.tolist()) == ([[-1] * 3] * 2, [0, 0], [-1, -1])
