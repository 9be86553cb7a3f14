"""Ends of what the paged cache's operators take: values near the end of fp32, many layers and heads, sizes
that the C call's ints do not hold."""
import math

import pytest
import torch

from paper_2505_14201_amd import flashd
from tests import paged_util as pu
from tests.test_gpu_tree import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hint", (1, 12))               # 4 rows to a token: 16 and 32 rows to a tile
@pytest.mark.parametrize("exponent,rise", [(100, "by turns"), (125, "by turns"), (100, 50.0), (124, 50.0), (125, 0.0), (125, 300.0)])
@pytest.mark.parametrize("keys,d", [(900, 128), (5000, 64), (50000, 64)])
def test_fp32_values_of_any_size(keys, d, exponent, rise, hint):
    """Values of 2^exponent times N(0, 1) under scores that rise along the sequence by `rise` powers of two, or by 50 and back every 128
    keys: every output is finite in fp32 (a mean of values below 2^128) and as near to fp64 as that of values of 1."""
    c = pu.make([keys - 3], [3], 1, d, 32, "f32", seed=91, qk_std=0.02)
    j = torch.arange(keys)
    power = 50.0 * (j // 128 % 2) if rise == "by turns" else j * (rise / keys)
    c.k[c.table[0].long()[j // 32], :, j % 32, 0] = (power * math.log(2)).float().view(-1, 1)
    q = pu.queries(c, 4, "f32", seed=92)
    q[..., 0] = 1.0
    o, mass, size = pu.attention(c, q, 1.0)
    bound = pu.attention_bound(c, "f32", o, mass, size)
    c.v *= 2.0 ** exponent
    assert torch.isfinite(c.v).all()
    got = run(c, q, 1.0, max_q=hint)
    assert bool(torch.isfinite(got).all())
    worst = float(((got.double() * 2.0 ** -exponent - o).abs() / bound).max())
    assert worst <= 1.0, worst


@pytest.mark.parametrize("hint", (1, 12))
def test_fp32_weights_are_as_near_as_fp32_holds_them(hint):
    """The error of an output in units of what independent errors of the weights by a part of themselves would make of it.  In fp32: the
    argument of the exponential lies within 8 of zero, half a step of it is at most 2^-22, 0.95e-7 of a weight (rms); its product 0.5e-7,
    the exponential 1.2e-7, the sums of 64 keys 2.4e-7 as a share of sqrt(sum w^2 v^2): 2.9e-7 together, and not above 5e-7.  (An argument of
    32 to 64 alone would be off by 7.6e-7.)"""
    c = pu.make([63] * 40, [1] * 40, 1, 128, 32, "f32", seed=93)
    gen = torch.Generator().manual_seed(94)
    c.k[..., 0] = torch.randint(-256, 1, c.k.shape[:3], generator=gen) / 64.0
    q = torch.zeros(40, 4, 128)
    q[..., 0] = 1.0
    got = run(c, q, 1.0, max_q=hint).double()
    total = 0.0
    for b in range(40):
        k, v, _ = c.keys(b)
        w = torch.softmax(k[0, :, 0], 0)
        o = w @ v[0]
        total += float((((got[b, 0] - o) / ((w[:, None] * (v[0] - o)) ** 2).sum(0).sqrt()) ** 2).mean())
    assert (total / 40) ** 0.5 <= 5e-7


def test_commit_in_a_million_layers_and_heads():
    layers, heads = 65535, 17
    k, v = (torch.randint(0, 120, (layers, 1, heads, 16, 64), dtype=torch.uint8, device="cuda") for _ in "kv")
    was = [x[:, 0, :, 1].clone() for x in (k, v)]
    table, lens, starts = (pu.ints(x).cuda() for x in ([[0]], [0], [0, 2]))
    out = torch.zeros(1, dtype=torch.int32, device="cuda")
    flashd.cache_commit(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), table, lens, starts, out, keep=pu.ints([[1]]).cuda())
    torch.cuda.synchronize()
    assert out.tolist() == [1]
    assert torch.equal(k[:, 0, :, 0], was[0]) and torch.equal(v[:, 0, :, 0], was[1])


def test_sizes_that_an_int_does_not_hold_are_refused():
    """2^32 + 1 of anything is not taken for 1."""
    many = 2 ** 32 + 1
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")            # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")                    # noqa: E731
    kc, x, table, lens, starts = z(2, 1, 16, 64), z(1, 1, 64), i(1, 1), i(1), i(2)
    with pytest.raises(flashd.FlashdError) as e:
        flashd.attn_fwd_tree(x, kc, z(2, 1, 16, 64), torch.empty_like(x), table, lens, starts, 1, 0.1,
                             tree=torch.empty(1, many, dtype=torch.int64, device="cuda"))
    assert e.value.status == -2
    with pytest.raises(flashd.FlashdError) as e:
        flashd.attn_fwd_tree(x, kc, z(2, 1, 16, 64), torch.empty_like(x), table, lens, starts, many, 0.1)
    assert e.value.status == -2
    with pytest.raises(flashd.FlashdError) as e:
        flashd.cache_append(x, x.clone(), x.clone(), torch.empty_like(x), kc, z(2, 1, 16, 64), table, lens, starts,
                            inv_freq=torch.empty(2 ** 31, dtype=torch.float32, device="cuda"))
    assert e.value.status == -2
    with pytest.raises(flashd.FlashdError) as e:
        flashd.cache_commit(kc, z(2, 1, 16, 64), table, lens, starts, i(1), keep=torch.empty(1, many, dtype=torch.int32, device="cuda"))
    assert e.value.status == -2
    with pytest.raises(flashd.FlashdError) as e:
        flashd.cache_fork(i(1), torch.empty(many, dtype=torch.int32, device="cuda"), table, lens, i(1, 1), i(1))
    assert e.value.status == -2
    one = kc.view(1, 2, 1, 16, 64)
    with pytest.raises(flashd.FlashdError) as e:
        flashd.cache_reserve(one.expand(many, -1, -1, -1, -1), z(1, 2, 1, 16, 64).expand(many, -1, -1, -1, -1), i(2), table, lens, starts, i(2))
    assert e.value.status == -2
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
