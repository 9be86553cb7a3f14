"""What the operators on a paged cache refuse, before anything reaches the GPU: through the C ABI
with made-up pointers, and through the Python functions with CPU tensors and wrong shapes."""
import pytest
import torch

from paper_2505_14201_amd import flashd
from tests.test_abi import E_ALIGN, E_DTYPE, E_GQA, E_HEADDIM, E_NULL, E_SHAPE, E_VARIANT, E_WS, NO_GPU

E_CACHE, E_OVERLAP = -11, -12
E_HIP, OK = -8, 0

# made-up, aligned addresses far apart; none is ever read on these paths
K, V, TABLE, LENS, REFS, START, Q, O, KN, VN, AUX, AUX2 = (0x100000000000 + i * 0x10000000000 for i in range(12))


def cache(**kw):
    a = dict(k=K, v=V, table=TABLE, lens=LENS, page_stride=2 * 16 * 64, layer_stride=0, layers=1, P=10, page=16,
             max_pages=4, B=3, Hkv=2, d=64, dtype=flashd.BF16, kscale=1.0, vscale=1.0)
    a.update(kw)
    return flashd.Cache(*(a[n] for n, _ in flashd.Cache._fields_))


def tree(c=None, layer=0, q=Q, qs=4 * 64, o=O, os=4 * 64, T=5, max_q=3, Hq=4, start=START, bits=AUX, words=1,
         scale=0.1, dtype=flashd.BF16, ws=None, ws_bytes=0, **kw):
    return flashd.raw().flashd_attn_fwd_tree(c or cache(**kw), layer, q, qs, o, os, T, max_q, Hq, start, bits, words,
                                             scale, dtype, None, ws, ws_bytes)


def append(c=None, layer=0, q=Q, qs=4 * 64, k=KN, ks=2 * 64, v=VN, vs=2 * 64, o=O, os=4 * 64, T=5, Hq=4, start=START,
           pos=None, inv=AUX, rot=64, qw=None, kw_=None, dtype=flashd.BF16, **kw):
    return flashd.raw().flashd_cache_append(c or cache(**kw), layer, q, qs, k, ks, v, vs, o, os, T, Hq, start, pos, inv,
                                            rot, 0, qw, kw_, 1e-6, dtype, None)


def fork(c=None, refs=REFS, parent=AUX, n=3, table_out=O, lens_out=Q, **kw):
    return flashd.raw().flashd_cache_fork(c or cache(**kw), refs, parent, n, table_out, lens_out, None)


def reserve(c=None, refs=REFS, start=START, report=O, **kw):
    return flashd.raw().flashd_cache_reserve(c or cache(**kw), refs, start, report, None)


def commit(c=None, start=START, keep=AUX, most=4, n=AUX2, out=O, **kw):
    return flashd.raw().flashd_cache_commit(c or cache(**kw), start, keep, most, n, out, None)


ALL = (tree, append, fork, reserve, commit)


@pytest.mark.parametrize("call", ALL)
def test_of_the_cache(call):
    for name in ("k", "v", "table", "lens"):
        assert call(**{name: None}) == E_NULL
    for name in ("B", "P", "layers", "Hkv", "max_pages"):
        assert call(**{name: 0}) == E_SHAPE and call(**{name: -2}) == E_SHAPE
    assert call(B=4097) == E_SHAPE
    assert call(max_pages=100000000) == E_SHAPE                       # keys of a sequence
    assert call(B=4096, max_pages=1 << 20) == E_SHAPE                 # entries of the table
    assert call(P=1000000000) == E_SHAPE                              # elements of a pool
    for dtype in (-1, 4):
        assert call(dtype=dtype) == E_DTYPE or call in (tree, append)
    assert call(d=96) == E_HEADDIM
    for page in (0, -16, 8, 17, 48, 512):
        assert call(page=page) == E_CACHE
    assert call(page_stride=2 * 16 * 64 - 8) == E_CACHE               # pages that overlap
    assert call(layers=2, layer_stride=5 * 2 * 16 * 64) == E_CACHE    # layers that overlap
    assert call(layers=2, layer_stride=-8) == E_CACHE
    assert call(page_stride=2 * 16 * 64 + 4) == E_ALIGN
    assert call(k=K + 8) == E_ALIGN and call(v=V + 4) == E_ALIGN
    assert call(table=TABLE + 2) == E_ALIGN and call(lens=LENS + 1) == E_ALIGN
    assert flashd.raw().flashd_cache_fork(None, REFS, AUX, 3, O, Q, None) == E_NULL


def test_of_the_packed_tensors():
    for call in (tree, append):
        for name in ("q", "o", "start"):
            assert call(**{name: None}) == E_NULL
        assert call(layer=1) == E_CACHE and call(layer=-1) == E_CACHE
        assert call(T=-1) == E_SHAPE and call(Hq=0) == E_SHAPE and call(T=1000000000, Hq=4) == E_SHAPE
        assert call(T=10000001) == E_SHAPE
        assert call(Hq=5, qs=5 * 64, os=5 * 64) == E_GQA
        assert call(c=cache(dtype=flashd.F16)) == E_VARIANT           # q in another type than the cache
        assert call(qs=4 * 64 - 8) == E_SHAPE and call(os=0) == E_SHAPE
        assert call(qs=4 * 64 + 4) == E_ALIGN
        assert call(q=Q + 8) == E_ALIGN and call(o=O + 2) == E_ALIGN and call(start=START + 2) == E_ALIGN
        assert call(o=K + 64) == E_OVERLAP and call(o=V) == E_OVERLAP
    assert tree(o=Q) == E_OVERLAP and tree(o=Q + 256) == E_OVERLAP
    assert append(o=Q + 256) == E_OVERLAP and append(o=KN) == E_OVERLAP and append(k=V) == E_OVERLAP
    assert append(k=None) == E_NULL and append(v=None) == E_NULL and append(inv=None) == E_NULL
    for rot in (-16, 8, 24, 80, 128):
        assert append(rot=rot) == E_SHAPE
    assert append(ks=64) == E_SHAPE and append(vs=2 * 64 + 4) == E_ALIGN and append(qw=AUX + 8) == E_ALIGN
    assert append(pos=AUX + 1) == E_ALIGN
    assert tree(max_q=0) == E_SHAPE and tree(words=0) == E_SHAPE and tree(bits=AUX + 4) == E_ALIGN
    need = flashd.tree_workspace_bytes(4, 2, 3, 64, flashd.BF16)
    assert need > 0 and tree(ws=AUX2, ws_bytes=need - 1) == E_WS and tree(ws=AUX2 + 8, ws_bytes=need) == E_ALIGN
    assert flashd.tree_workspace_bytes(5, 2, 3, 64, flashd.BF16) == 0 and flashd.tree_workspace_bytes(4, 2, 0, 64, 1) == 0
    c = cache(dtype=flashd.CACHE_FP8)
    raw = flashd.raw()
    assert raw.flashd_attn_fwd_tree(c, 0, Q, 256, O, 256, 5, 3, 4, START, None, 0, 0.1, flashd.F32, None, None, 0) == E_VARIANT


def test_of_keys_and_values_in_one_place():
    page = 2 * 16 * 64                                                 # elements; 2 bytes each
    for call in (append, reserve, commit):
        assert call(c=cache(v=K)) == E_OVERLAP and call(c=cache(v=K + 2 * page)) == E_OVERLAP        # pages on pages
        assert call(c=cache(v=K + page, page_stride=2 * page)) == E_OVERLAP                 # half a page on
        two = dict(layers=2, layer_stride=20 * page)
        assert call(c=cache(v=K + 2 * page, **two)) == E_OVERLAP and call(c=cache(v=K + 2 * 19 * page, **two)) == E_OVERLAP
        if NO_GPU:
            assert call(c=cache(v=K + 2 * 10 * page, **two)) == E_HIP                       # a layer's K, then its V
            assert call(c=cache(v=K + 2 * page, page_stride=2 * page)) == E_HIP
            # layers of a page next to each other, its K first
            assert call(c=cache(v=K + 2 * 2 * page, layers=2, layer_stride=page, page_stride=4 * page)) == E_HIP
        assert call(c=cache(v=K + 2 * page, layers=2, layer_stride=page, page_stride=4 * page)) == E_OVERLAP


def test_of_an_append_in_place():
    """q_out = q: k and v lie apart, or between the tokens of q."""
    one = dict(q=Q, o=Q, qs=512, os=512, ks=512, vs=512, v=VN)
    assert append(**{**one, "k": Q}) == E_OVERLAP and append(**{**one, "k": Q + 256}) == E_OVERLAP
    assert append(**{**one, "k": Q + 1024 - 128}) == E_OVERLAP         # into the next token
    assert append(**{**one, "k": Q + 512, "ks": 256}) == E_OVERLAP     # of another stride
    assert append(**{**one, "k": Q + 512, "v": Q + 512 - 16}) == E_OVERLAP
    if NO_GPU:
        assert append(**{**one, "k": Q + 512, "v": Q + 768}) == E_HIP


def test_of_the_bookkeeping():
    for name in ("refs", "parent", "table_out", "lens_out"):
        assert fork(**{name: None}) == E_NULL
        assert fork(**{name: O + 0x1002}) == E_ALIGN
    assert fork(n=0) == E_SHAPE and fork(n=4097) == E_SHAPE
    assert fork(table_out=TABLE + 16) == E_OVERLAP and fork(lens_out=LENS) == E_OVERLAP
    assert fork(table_out=AUX) == E_OVERLAP and fork(lens_out=O + 8) == E_OVERLAP and fork(lens_out=REFS) == E_OVERLAP
    for name in ("refs", "start", "report"):
        assert reserve(**{name: None}) == E_NULL and reserve(**{name: O + 0x1001}) == E_ALIGN
    for at in (TABLE, LENS, START, REFS):
        assert reserve(report=at) == E_OVERLAP
    assert commit(start=None) == E_NULL and commit(out=None) == E_NULL
    assert commit(most=0) == E_SHAPE and commit(keep=None) == E_SHAPE and commit(most=1 << 30) == E_SHAPE
    assert commit(keep=AUX + 2) == E_ALIGN and commit(n=AUX2 + 1) == E_ALIGN
    for at in (LENS, TABLE + 8, START, AUX + 16, AUX2):
        assert commit(out=at) == E_OVERLAP


@pytest.mark.skipif(not NO_GPU, reason="a valid call would launch a kernel on made-up pointers")
def test_valid_calls_get_as_far_as_the_device():
    for call in ALL:
        assert call() == E_HIP
    assert commit(keep=None, most=0, n=None) == E_HIP
    assert append(o=Q) == E_HIP                                        # in place
    assert append(q=Q, k=Q + 512, v=Q + 768, qs=512, ks=512, vs=512) == E_HIP
    assert tree(layers=3, layer_stride=10 * 2 * 16 * 64, layer=2) == E_HIP
    assert tree(layers=3, layer_stride=2 * 16 * 64, page_stride=3 * 2 * 16 * 64, layer=2) == E_HIP
    assert tree(v=K + 2 * 16 * 64 * 2, page_stride=2 * 2 * 16 * 64) == E_HIP       # K and V side by side


def test_python_functions_refuse_wrong_tensors():
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t)           # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)                   # noqa: E731
    kc = z(4, 2, 16, 64)
    with pytest.raises(ValueError):
        flashd.attn_fwd_tree(z(1, 4, 64), kc, kc, z(1, 4, 64), i(1, 2), i(1), i(2), 1, 0.1)
    with pytest.raises(ValueError):
        flashd.cache_append(z(1, 4, 64), z(1, 2, 64), z(1, 2, 64), z(1, 4, 64), kc, kc, i(1, 2), i(1), i(2))
    with pytest.raises(ValueError):
        flashd.cache_fork(i(1), i(4), i(1, 2), i(1), i(1, 2), i(1))
    with pytest.raises(ValueError):
        flashd.cache_reserve(kc, kc, i(4), i(1, 2), i(1), i(2), i(2))
    with pytest.raises(ValueError):
        flashd.cache_commit(kc, kc, i(1, 2), i(1), i(2), i(1))


@pytest.mark.gpu
def test_python_functions_refuse_wrong_shapes_on_the_gpu():
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")           # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")                   # noqa: E731
    good = dict(q=z(3, 4, 64), kcache=z(4, 2, 16, 64), vcache=z(4, 2, 16, 64), o=z(3, 4, 64), table=i(2, 2), lens=i(2),
                q_start=i(3), max_q=1, scale=0.1)
    flashd.attn_fwd_tree(**good)
    for name, bad in (("q", z(3, 4, 128)), ("q", z(3, 4, 64, t=torch.float64)), ("q", z(3, 64, 4).transpose(1, 2)),
                      ("o", z(2, 4, 64)), ("o", z(3, 4, 64, t=torch.float16)), ("kcache", z(4, 2, 64, 16).transpose(2, 3)),
                      ("kcache", z(5, 2, 16, 64)), ("vcache", z(4, 2, 16, 64, t=torch.float16)), ("table", i(2, 2).long()),
                      ("table", i(2, 4)[:, ::2]), ("lens", i(3)), ("q_start", i(2)), ("q_start", z(3))):
        with pytest.raises((ValueError, flashd.FlashdError)):
            flashd.attn_fwd_tree(**{**good, name: bad})
    with pytest.raises(ValueError):
        flashd.attn_fwd_tree(**good, tree=z(3, 1, t=torch.int32))
    with pytest.raises(ValueError):
        flashd.attn_fwd_tree(**good, tree=z(2, 1, t=torch.int64))
    with pytest.raises(flashd.FlashdError):
        flashd.attn_fwd_tree(**good, workspace=z(16))
    with pytest.raises(flashd.FlashdError):
        flashd.attn_fwd_tree(**{**good, "max_q": 0})
    with pytest.raises(flashd.FlashdError):
        flashd.attn_fwd_tree(**{**good, "o": good["q"]})
    flashd.attn_fwd_tree(**{**good, "q": z(0, 4, 64), "o": z(0, 4, 64)})               # no tokens: no work
    torch.cuda.synchronize()
