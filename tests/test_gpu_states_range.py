"""Attention to 8-bit states at the end of the numbers' range: queries that hold
infinities or NaN."""
import math

import pytest
import torch

from .test_gpu_layers import gen_of, normal, say
from .test_gpu_states import states

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
