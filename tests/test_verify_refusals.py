"""What flashd_draft_verify refuses before anything reaches the GPU, and its plain model on calls that can be done by hand."""
import pytest
import torch

from paper_2505_14201_amd import flashd
from tests.test_abi import E_ALIGN, E_DTYPE, E_NULL, E_SHAPE, E_WS
from tests.verify_model import verify

E_OVERLAP = -12
L, D, X, PARENT, U, HEAT, START, KEEP, N, NEXT, WS = (0x100000000000 + i * 0x10000000000 for i in range(11))


def call(logits=L, ls=100, draft=D, ds=100, tokens=X, parent=PARENT, uniform=U, heat=HEAT, start=START, B=3, T=7, V=100,
         dtype=flashd.BF16, ddtype=flashd.F32, most=4, keep=KEEP, n=N, then=NEXT, ws=WS, ws_bytes=1 << 20):
    return flashd.raw().flashd_draft_verify(logits, ls, draft, ds, tokens, parent, uniform, heat, start, B, T, V, dtype, ddtype,
                                            most, keep, n, then, None, ws, ws_bytes)


def test_of_draft_verify():
    for name in ("logits", "tokens", "uniform", "start", "keep", "n", "then"):
        assert call(**{name: None}) == E_NULL
    for name in ("B", "V", "most"):
        assert call(**{name: 0}) == E_SHAPE and call(**{name: -1}) == E_SHAPE
    assert call(B=4097) == E_SHAPE and call(T=-1) == E_SHAPE and call(T=10000001) == E_SHAPE
    assert call(V=(1 << 24) + 1, ls=1 << 25, ds=1 << 25) == E_SHAPE and call(most=1 << 30) == E_SHAPE
    assert call(ls=99) == E_SHAPE and call(ds=99) == E_SHAPE and call(ls=1 << 40) == E_SHAPE
    for dtype in (-1, 3):
        assert call(dtype=dtype) == E_DTYPE and call(ddtype=dtype) == E_DTYPE
    assert call(logits=L + 1) == E_ALIGN and call(draft=D + 2) == E_ALIGN and call(ws=WS + 8) == E_ALIGN
    for name, at in (("tokens", X), ("parent", PARENT), ("uniform", U), ("heat", HEAT), ("start", START), ("keep", KEEP),
                     ("n", N), ("then", NEXT)):
        assert call(**{name: at + 2}) == E_ALIGN
    need = flashd.verify_workspace_bytes(7, 100)
    assert need > 0 and call(ws_bytes=need - 1) == E_WS
    assert flashd.verify_workspace_bytes(7, 0) == 0 and flashd.verify_workspace_bytes(-1, 100) == 0
    for out, size in (("keep", 3 * 4 * 4), ("n", 12), ("then", 12)):
        for at, length in ((L, 1400), (D, 2800), (X, 28), (PARENT, 28), (U, 28), (HEAT, 12), (START, 16), (WS, need)):
            assert call(**{out: at}) == E_OVERLAP and call(**{out: at + length - 4}) == E_OVERLAP
            assert call(**{out: at - size + 4}) == E_OVERLAP
    assert call(n=KEEP + 44) == E_OVERLAP and call(then=N + 8) == E_OVERLAP and call(ws=L + 1392) == E_OVERLAP


def test_of_its_python_form():
    t = torch.zeros
    i = lambda *s: t(*s, dtype=torch.int32)     # noqa: E731
    with pytest.raises(ValueError, match="logits"):
        flashd.draft_verify(t(4, 10), i(4), t(4), i(2), i(1, 4), i(1), i(1))
    with pytest.raises(ValueError, match="logits"):
        flashd.draft_verify(t(4), i(4), t(4), i(2), i(1, 4), i(1), i(1))


def test_the_model_by_hand():
    # p = (1/4, 1/2, 1/4); id 1 is refused by u >= 1/2, then r = (1/2, 0, 1/2)
    logits = torch.log(torch.tensor([[1.0, 2.0, 1.0]] * 3).double())
    ask = lambda u, **kw: verify(logits, torch.tensor([0, 1, 0]), torch.tensor(u), [0, 3], 3, **kw)[:3]     # noqa: E731
    tree = torch.tensor([-1, 0, 0])
    assert ask([0.6, 0.4, 0.2]) == ([[0, 1, 2]], [3], [1])
    assert ask([0.6, 0.51, 0.0]) == ([[0, -1, -1]], [1], [2])
    assert ask([0.4, 0.51, 0.0]) == ([[0, -1, -1]], [1], [0])
    assert ask([0.4, 0.51, 0.49], parent=tree) == ([[0, 2, -1]], [2], [1])
    assert ask([0.4, 0.51, 0.51], parent=tree) == ([[0, -1, -1]], [1], [2])
    # q = (0, 3/4, 1/4): id 1 is refused by u >= 2/3, then r = (1, 0, 0)
    q = torch.tensor([[0.0, 0.75, 0.25]] * 3)
    assert ask([0.9, 0.66, 0.3], draft=q) == ([[0, 1, 2]], [3], [2])
    assert ask([0.9, 0.67, 0.3], draft=q) == ([[0, -1, -1]], [1], [0])
    # the largest logit, whatever the number
    assert ask([0.9, 0.99, 0.3], temperature=torch.zeros(1)) == ([[0, 1, -1]], [2], [1])
