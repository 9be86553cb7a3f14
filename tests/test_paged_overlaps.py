"""Outputs of the paged cache's operators that lie on an input or on another output are refused, whichever two they are."""
import pytest

from paper_2505_14201_amd import flashd
from tests.test_abi import NO_GPU
from tests.test_paged_refusals import (AUX, AUX2, E_HIP, E_OVERLAP, K, KN, LENS, O, Q, REFS, START, TABLE, V, VN, append, commit, fork, reserve,
                                       tree)

WS = AUX2
NEED = flashd.tree_workspace_bytes(4, 2, 3, 64, flashd.BF16)
PAGES = 10 * 2 * 16 * 64 * 2        # bytes of a pool of the caches here

# (call, name of an argument, an address that is an output's or that an output must not touch)
CASES = [(fork, "refs", at) for at in (TABLE, LENS, AUX, O, Q)] + \
        [(fork, "table_out", at) for at in (REFS, TABLE, LENS, AUX, Q)] + [(fork, "lens_out", at) for at in (REFS, TABLE, LENS, AUX, O)] + \
        [(reserve, "refs", at) for at in (TABLE, LENS, START, O, K, V, K + PAGES - 4)] + \
        [(reserve, "report", at) for at in (TABLE, LENS, START, REFS, K, V + PAGES - 4)] + \
        [(reserve, "table", at) for at in (LENS, START, REFS, O, K + 2048, V)] + [(reserve, "lens", at) for at in (K, V)] + \
        [(reserve, "start", at) for at in (K + 16, V)] + \
        [(append, "o", at) for at in (TABLE, LENS, START, AUX, Q + 16, KN, VN, K, V)] + \
        [(append, "pos", at) for at in (O, O + 512, K, V)] + [(append, "inv", at) for at in (O, K, V)] + \
        [(append, "qw", at) for at in (O, K)] + [(append, "kw_", at) for at in (O, V)] + \
        [(append, name, at) for name in ("table", "lens", "start") for at in (O, K, V)] + \
        [(tree, "o", at) for at in (TABLE, LENS, START, AUX, Q, K, V)] + \
        [(tree, "ws", at) for at in (TABLE, LENS, START, AUX, Q, O, K, V, O - 4096)] + \
        [(commit, "out", at) for at in (TABLE, LENS, START, AUX, AUX2, K, V)] + \
        [(commit, name, at) for name in ("table", "lens", "start", "keep", "n") for at in (K, V, O)]


@pytest.mark.parametrize("call,name,at", CASES, ids=[f"{c.__name__}-{n}-{i}" for i, (c, n, _) in enumerate(CASES)])
def test_outputs_lie_apart(call, name, at):
    more = dict(ws_bytes=NEED) if name == "ws" else {}
    assert call(**{name: at}, **more) == E_OVERLAP


@pytest.mark.skipif(not NO_GPU, reason="a valid call would launch a kernel on made-up pointers")
def test_neighbours_are_taken():
    """One element behind an output's last, or before its first, is nobody's."""
    assert fork(refs=O + 3 * 4 * 4) == E_HIP and fork(lens_out=O - 12) == E_HIP
    assert reserve(report=K + PAGES) == E_HIP and reserve(refs=O + 16) == E_HIP and reserve(refs=O - 40) == E_HIP
    assert append(pos=O + 5 * 512) == E_HIP and append(qw=K - 128) == E_HIP
    assert tree(ws=WS, ws_bytes=NEED) == E_HIP and tree(ws=O + 5 * 512, ws_bytes=NEED) == E_HIP and tree(ws=Q - (NEED + 15) // 16 * 16, ws_bytes=NEED) == E_HIP
    assert commit(out=K - 12) == E_HIP and commit(keep=V + PAGES) == E_HIP
    # inputs may be one another's
    assert append(pos=START, qw=AUX, kw_=AUX) == E_HIP and append(k=KN, v=KN) == E_HIP and commit(n=LENS) == E_HIP
    # no tokens, no elements
    assert tree(T=0, o=Q) == E_HIP and append(T=0, o=K + 512, q=K, k=K, v=K) == E_HIP
