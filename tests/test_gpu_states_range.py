"""Attention to 8-bit states at the end of the numbers' range: queries that hold
infinities or NaN, and scales of every size."""
import math

import pytest
import torch

from . import layers_common as R
from . import more_layers_common as M
from .test_gpu_layers import gen_of, normal, say
from .test_gpu_states import F8, states

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2210_10108_amd import layers
    layers.lib()
    return layers


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("Sq", [1, 9, 70, 300])
@pytest.mark.parametrize("D", [64, 128, 100])
def test_queries_that_are_no_numbers(L, D, Sq, dt):
    # entries: no key allowed by the mask; none by the length; a part of a tile; a whole one
    # beside a hidden one; all
    B, Sk, Hq, Hkv = 5, 192, 4, 2
    g = gen_of(1)
    q = normal(g, B, Sq, Hq, D, dt=dt)
    (k8, ks), (v8, vs) = states(g, B, Sk, Hkv, D), states(g, B, Sk, Hkv, D)
    kv_len = torch.tensor([192, 0, 130, 192, 192], dtype=torch.int32, device="cuda")
    mask = torch.ones(B, Sk, dtype=torch.bool, device="cuda")
    mask[0] = False
    mask[2] = torch.rand(Sk, generator=g, device="cuda") > 0.5
    mask[3, 64:128] = False
    say("queries that are no numbers", D, Sq, dt)
    clean = L.cross_attention_q8(q, k8, v8, ks, vs, kv_len=kv_len, kv_mask=mask, return_lse=True)
    row = Sq // 2
    for junk in (math.inf, -math.inf, math.nan):
        bad = q.clone()
        bad[:, row, 1, 0] = junk
        bad[:, row, 2, D - 1] = math.nan
        o, lse = L.cross_attention_q8(bad, k8, v8, ks, vs, kv_len=kv_len, kv_mask=mask, return_lse=True)
        # without a key: 0 and -inf, whatever the query is
        assert bool((o[:2] == 0).all()) and bool((lse[:2] == -math.inf).all()), junk
        # rows beside it: as without it
        rest = torch.ones(B, Sq, Hq, dtype=torch.bool, device="cuda")
        rest[:, row, 1:3] = False
        assert torch.equal(o[rest], clean[0][rest])
        assert torch.equal(lse.transpose(1, 2)[rest], clean[1].transpose(1, 2)[rest])
        # the row itself, with keys: no number
        assert bool(o[2:, row, 1:3].isnan().all()) and bool(lse[2:, 1:3, row].isnan().all()), junk


def check_scales(L, q, k8, v8, ks, vs, what, **masks):
    """As test_gpu_states' check, but with a bound that does not grow with the largest
    value, which may have no weight: p is rounded relative to itself (u), in float16 to
    2^-25 of the value at least (or less: the weights are below 2^8 in the row's unit,
    2^-25 in which is 2^-33 of the largest), and what a block adds is lost only beside sums
    2^50 times as large.  An exponential below 2^-126 is no 32-bit number, and a part of the
    keys is joined by one of its largest p, which p reach 2^8 times of: weights below 2^-118
    may be lost."""
    say("scales", what, tuple(q.shape), q.dtype)
    ref = R.attention_ref(q, M.widened(k8, ks), M.widened(v8, vs), **masks)
    o, lse = L.cross_attention_q8(q, k8, v8, ks, vs, return_lse=True, **masks)
    B, Sq, Hq, D = q.shape
    G = Hq // k8.shape[2]
    K, V = (M.widened(*t).repeat_interleave(G, 2) for t in ((k8, ks), (v8, vs)))
    A = torch.einsum("bihd,bjhd->bhij", q.double(), K) * D ** -0.5
    on = M.allowed(B, k8.shape[1], masks.get("kv_len"), masks.get("kv_mask"), q.device)
    A = A.masked_fill(~on[:, None, None, :], -math.inf)
    P = torch.softmax(A, 3)
    V = V * on[:, :, None, None]
    terms = torch.einsum("bhij,bjhd->bihd", P, V.abs())
    terms_lost = torch.einsum("bhij,bjhd->bihd", torch.where(P < 2.0 ** -118, P, 0.0), V.abs())
    e = 2 * ref["lse"][1].amax() + R.EF
    u, tiny = R.U[R.name_of(q.dtype)], R.TINY[R.name_of(q.dtype)]
    bound = (2 * u + 2 * e) * terms + 2.0 ** -50 * terms.amax(3, keepdim=True) + terms_lost + 2 * tiny
    if q.dtype == torch.float16:
        bound += 2.0 ** -24 * V.abs().sum(1)[:, None]
    R.check(o, ref["o"][0], bound, what + " o")
    R.check(lse, *ref["lse"], what + " lse")


@pytest.mark.parametrize("Sq", [1, 40, 300])
@pytest.mark.parametrize("D", [64, 128, 100])
def test_states_of_blocks_far_apart_quantized(L, D, Sq):
    # bfloat16 states whose blocks are of every size that the type has, in both orders and in
    # turn; weights alike, or all on the small blocks, or all on the large ones
    B, Sk, Hq, Hkv = 2, 64 * 7 + 9, 4, 2
    g = gen_of(2)
    q, k, v = (normal(g, B, S, H, D, dt="bf16") for S, H in ((Sq, Hq), (Sk, Hkv), (Sk, Hkv)))
    q[..., 0] = 16.0
    block = torch.arange(Sk, device="cuda") // 64
    for large in (1.0, 1e36):
        for small in (1e-37, 1e-30, 1e-20):
            for name, first in (("falling", block < 3), ("rising", block >= 3), ("in turn", block % 2 == 0),
                                ("one", block == 4), ("all but one", block != 4)):
                x = (v.float() * torch.where(first, large, small)[None, :, None, None]).bfloat16()
                for way in (0.0, 20.0, -20.0, 60.0, -60.0):  # scores apart by 32 |way| / sqrt(D)
                    y = k.clone()
                    y[..., 0] = torch.where(first, way, -way)[None, :, None]
                    check_scales(L, q, *L.quantize_states(y, x), f"{large} {small} {name} {way}")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("Sq", [1, 40, 300])
@pytest.mark.parametrize("seed", range(6))
def test_scales_of_every_size(L, seed, Sq, dt):
    # any positive normal scales, block by block, and scores that move the weight between them
    B, Sk, Hq, Hkv, D = 2, 64 * 24 + 5, 4, 2, (64, 128, 100)[seed % 3]
    g = gen_of(100 + seed)
    q = normal(g, B, Sq, Hq, D, dt=dt)
    q[..., 0] = 16.0
    nb = 25
    top = 6.0 if dt == "f16" else 118.0
    reach = (2.0, 30.0, 90.0, 125.0, 240.0, 60.0)[seed]
    e = torch.rand(B, nb, Hkv, generator=g, device="cuda") * reach
    vs = torch.exp2((top - e).clamp_min(-126.0))
    if seed % 2:
        vs = torch.exp2(torch.floor(torch.log2(vs)))
    x = torch.randn(2, B, Sk, Hkv, D, generator=g, device="cuda") * 100
    move = torch.randn(B, nb, Hkv, generator=g, device="cuda") * (0.0, 5.0, 30.0)[seed // 2]
    x[0, ..., 0] = move.repeat_interleave(64, 1)[:, :Sk] * 8
    k8, v8 = x.clamp(-448, 448).to(F8)
    ks = torch.full((B, nb, Hkv), 2.0 ** -6, device="cuda")
    check_scales(L, q, k8, v8, ks, vs, f"reach {reach}")
    mask = torch.rand(B, Sk, generator=g, device="cuda") > 0.3
    mask[0, 64:192] = False
    kv_len = torch.tensor([Sk, 700], dtype=torch.int32, device="cuda")
    check_scales(L, q, k8, v8, ks, vs, f"reach {reach} masked", kv_len=kv_len, kv_mask=mask)


@pytest.mark.parametrize("Sq,Sk", [(1, 40003), (7, 9000), (600, 3000)])
@pytest.mark.parametrize("D", [64, 128, 33])
def test_values_near_the_largest_number_over_many_keys(L, D, Sq, Sk):
    # their weighted sums pass float32's range, the results do not: by parts of the key axis,
    # by wavefronts and by groups of them
    g = gen_of(5)
    B, Hq, Hkv = 1, 4, 2
    q, k = normal(g, B, Sq, Hq, D, dt="bf16", std=0.1), normal(g, B, Sk, Hkv, D, dt="bf16")
    v = (1 + torch.rand(B, Sk, Hkv, D, generator=g, device="cuda")) * 1.4e38
    block = (torch.arange(Sk, device="cuda") // 64 % 5)[None, :, None, None]
    for name, x in (("all", v), ("of both signs", v * torch.sign(torch.randn(v.shape, generator=g, device="cuda"))),
                    ("one block in five", torch.where(block == 3, v, v * 1e-30)), ("four in five", torch.where(block == 3, v * 1e-60, v))):
        check_scales(L, q, *L.quantize_states(k, x.bfloat16()), name)
    # a query that is no number, its sums joined too
    bad = q.clone()
    bad[0, Sq - 1, 1, 0] = math.inf
    packed = L.quantize_states(k, v.bfloat16())
    want, got = (L.cross_attention_q8(t, *packed, return_lse=True) for t in (q, bad))
    assert bool(got[0][0, Sq - 1, 1].isnan().all()) and bool(got[1][0, 1, Sq - 1].isnan())
    rest = torch.ones(Sq, Hq, dtype=torch.bool, device="cuda")
    rest[Sq - 1, 1] = False
    assert torch.equal(got[0][0][rest], want[0][0][rest])
    none = torch.zeros(B, Sk, dtype=torch.bool, device="cuda")
    o, lse = L.cross_attention_q8(bad, *packed, kv_mask=none, return_lse=True)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())
