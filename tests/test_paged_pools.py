"""Where K and V may lie: pools of any strides are refused exactly where a page of one shares memory with a page of the other."""
import random

import pytest

from tests.test_abi import NO_GPU
from tests.test_paged_refusals import E_HIP, E_OVERLAP, K, append, cache, commit, reserve

PAGE = 2 * 16 * 64          # elements of a page of the caches here, of 2 bytes each


def test_values_on_the_keys_of_the_next_layer():
    """Strides that are no multiples of one another: V's pages lie between K's in its own layer, and on K's in the next."""
    for call in (append, reserve, commit):
        assert call(c=cache(v=K + 2 * 3 * PAGE, page_stride=2 * PAGE, layers=2, layer_stride=21 * PAGE)) == E_OVERLAP
        assert call(c=cache(v=K + 2 * 3 * PAGE, page_stride=7 * PAGE, layers=3, layer_stride=2 * PAGE, P=4)) == E_OVERLAP


@pytest.mark.skipif(not NO_GPU, reason="a valid call would launch a kernel on made-up pointers")
def test_every_layout_against_its_pages():
    rng = random.Random(5)
    seen = {True: 0, False: 0}
    for _ in range(4000):
        P, layers = rng.randint(1, 5), rng.randint(1, 4)
        if rng.random() < 0.5:                          # pages of a layer next to each other
            ps = rng.randint(2, 7) * (PAGE // 2)
            ls = max((P - 1) * ps + PAGE, 0) + rng.randint(0, 6) * (PAGE // 2)
        else:                                           # layers of a page
            ls = rng.randint(2, 5) * (PAGE // 2)
            ps = (layers - 1) * ls + PAGE + rng.randint(0, 6) * (PAGE // 2)
        off = rng.randint(-40, 40) * (PAGE // 2) + rng.choice([0, 0, 8, -8])
        at = [y * ls + p * ps for y in range(layers) for p in range(P)]
        shared = any(abs(off + b - a) < PAGE for a in at for b in at)
        rc = reserve(c=cache(v=K + 2 * off, P=P, layers=layers, page_stride=ps, layer_stride=ls))
        assert rc == (E_OVERLAP if shared else E_HIP), (P, layers, ps / PAGE, ls / PAGE, off / PAGE, rc)
        seen[shared] += 1
    assert min(seen.values()) > 500


@pytest.mark.parametrize("P,layers,ps,ls", [(3, 65535, 65535 * PAGE, PAGE), (200000, 2, PAGE, 200000 * PAGE), (200000, 1, PAGE, 0)])
def test_many_layers_and_pages(P, layers, ps, ls):
    """Pages of half of PAGE: V in the half that K leaves, or on the next page (or layer) of K."""
    c = dict(P=P, layers=layers, page_stride=ps, layer_stride=ls, Hkv=1)
    for call in (append, reserve, commit):
        more = dict(Hq=4, ks=64, vs=64) if call is append else {}
        assert call(c=cache(v=K + 2 * PAGE, **c), **more) == E_OVERLAP
        if NO_GPU:
            assert call(c=cache(v=K + PAGE, **c), **more) == E_HIP
