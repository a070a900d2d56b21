"""8-bit states and the attention that reads them, against their definitions in 64 bits."""
import math
import sys

import pytest
import torch

from . import layers_common as R
from . import more_layers_common as M

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def L():
    from paper_2210_10108_amd import layers
    layers.lib()
    return layers


def say(*a):
    sys.stderr.write("[gpu] " + " ".join(str(x) for x in a) + "\n")
    sys.stderr.flush()


def normal(gen, *shape, dt="f16", std=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(R.DT[dt])


def gen_of(seed):
    return torch.Generator("cuda").manual_seed(seed)


def same8(a, b):
    """Equal as numbers, NaN in the same places (the sign of a zero is not looked at)."""
    a, b = a.float().double(), b.double()
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


# ---------------------------------------------------------------- quantisation
def check_quantize(L, k, v, what, kv_len=None, kv_mask=None, **out):
    say("quantize", what, tuple(k.shape), k.dtype)
    on = M.allowed(*k.shape[:2], kv_len, kv_mask, k.device)
    got = L.quantize_states(k, v, kv_len=kv_len, kv_mask=kv_mask, **out)
    for i, x in enumerate((k, v)):
        x8, scale = M.quantize_ref(x, on)
        assert got[i].dtype == F8 and got[2 + i].shape == scale.shape
        assert torch.equal(got[2 + i], scale), (what, i)
        assert same8(got[i], x8), (what, i)
    return got


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 64), (2, 63, 2, 128), (1, 64, 3, 32), (3, 65, 1, 96), (2, 300, 4, 80),
                                   (1, 130, 2, 1), (2, 100, 3, 7), (1, 200, 2, 100), (2, 128, 1, 127), (1, 1000, 16, 64),
                                   (65, 70, 2, 8)], ids=str)
def test_quantize_states(L, shape, dt):
    g = gen_of(1)
    size = torch.exp(3 * torch.randn(shape[0], shape[1], shape[2], 1, generator=g, device="cuda"))
    k, v = ((torch.randn(*shape, generator=g, device="cuda") * size).clamp(-6e4, 6e4).to(R.DT[dt]) for _ in range(2))
    check_quantize(L, k, v, "plain")
    kv_len = torch.randint(0, shape[1] + 1, shape[:1], generator=g, device="cuda", dtype=torch.int32)
    mask = torch.rand(*shape[:2], generator=g, device="cuda") > 0.3
    check_quantize(L, k, v, "masked", kv_len=kv_len, kv_mask=mask)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 33])
def test_quantize_states_masks_and_what_lies_behind_them(L, D, dt):
    B, S, H = 6, 200, 2
    g = gen_of(2)
    k, v = normal(g, B, S, H, D, dt=dt), normal(g, B, S, H, D, dt=dt)
    kv_len = torch.tensor([0, 1, 64, 200, 999, -5], dtype=torch.int32, device="cuda")
    mask = torch.rand(B, S, generator=g, device="cuda") > 0.4
    mask[3] = False
    mask[4, 64:128] = False
    seen = M.allowed(B, S, kv_len, mask, "cuda")
    want = None
    for junk in (math.nan, math.inf, -math.inf, torch.finfo(R.DT[dt]).max, 0.0):
        k2, v2 = k.clone(), v.clone()
        k2[~seen], v2[~seen] = junk, junk
        for form in (mask, mask.to(torch.uint8) * 7):
            got = check_quantize(L, k2, v2, f"junk {junk}", kv_len=kv_len, kv_mask=form)
            want = want or got
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got[:2], want[:2]))


def test_quantize_states_numbers(L):
    # every 16-bit number, a head alone: zeros, subnormal numbers, ties, infinities, NaN
    for dt in ("f16", "bf16"):
        every = torch.arange(-32768, 32768, device="cuda", dtype=torch.int32).to(torch.int16).view(R.DT[dt])
        x = every.view(1, 1024, 1, 64)
        check_quantize(L, x, x.flip(1), "every number")
        # a block for each number, beside one that fixes the scale at 1
        few = every[::17].clone()
        few = few[few.abs() <= 448.0]
        rows = torch.zeros(1, 64 * len(few), 1, 8, dtype=R.DT[dt], device="cuda")
        rows[0, ::64, 0, 0] = 448.0
        rows[0, 1::64, 0, 3] = few
        check_quantize(L, rows, -rows, "scale 1")
    top = torch.zeros(1, 64, 1, 8, dtype=torch.float16, device="cuda")
    for most, scale in ((448.0, 1.0), (448.25, 2.0), (224.0, 0.5), (65504.0, 256.0), (2.0 ** -24, 2.0 ** -32), (0.0, 1.0)):
        top[0, 5, 0, 3] = -most
        got = check_quantize(L, top, top, f"most {most}")
        assert float(got[2]) == scale


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_quantize_states_layouts(L, dt):
    g = gen_of(3)
    B, S, H, D = 3, 150, 2, 64
    kv = normal(g, B, S, 2, H, D, dt=dt)
    want = check_quantize(L, kv[:, :, 0], kv[:, :, 1], "side by side")
    odd = torch.empty(B * S * H * (D + 3) + 1, dtype=kv.dtype, device="cuda")[1:].view(B, S, H, D + 3)[..., :D]
    odd.copy_(kv[:, :, 0])
    check_quantize(L, odd, kv[:, :, 1], "odd rows")
    # into a part of a larger cache, heads first: what lies beside it stays
    cache8 = torch.full((B + 2, H, S + 70, D), 77, dtype=torch.uint8, device="cuda")
    scales = torch.full((B + 2, 6, H), 5.0, device="cuda")
    k8 = cache8.view(F8)[1:B + 1, :, :S].transpose(1, 2)
    ks = scales[1:B + 1, :3]
    got = L.quantize_states(kv[:, :, 0], kv[:, :, 1], k8=k8, k_scale=ks)
    assert got[0] is k8 and got[2] is ks
    for a, b in zip(got, want):
        assert torch.equal(a.float(), b.float())
    assert bool((cache8[[0, -1]] == 77).all()) and bool((cache8[:, :, S:] == 77).all())
    assert bool((scales[[0, -1]] == 5).all()) and bool((scales[:, 3:] == 5).all())
    # bytes on odd addresses
    w = torch.full((B * S * H * (D + 1) + 1,), 77, dtype=torch.uint8, device="cuda")[1:].view(B, S, H, D + 1)
    got = L.quantize_states(kv[:, :, 0], kv[:, :, 1], k8=w.view(F8)[..., :D])
    assert torch.equal(got[0].float(), want[0].float()) and bool((w[..., D] == 77).all())
    for B, S in ((0, 5), (2, 0)):
        k = torch.empty(B, S, 2, 64, dtype=R.DT[dt], device="cuda")
        got = L.quantize_states(k, k)
        assert got[0].shape == k.shape and got[2].shape == (B, -(-S // 64), 2)


# ---------------------------------------------------------------- attention
def states(gen, B, Sk, Hkv, D, spread=1.0):
    """8-bit states whose scales differ from block to block; values of every e4m3 size."""
    x = torch.randn(B, Sk, Hkv, D, generator=gen, device="cuda")
    nb = -(-Sk // M.BLOCK)
    s = torch.exp(torch.randn(B, nb, Hkv, generator=gen, device="cuda") * spread)
    return (x * 100).clamp(-448, 448).to(F8), s / 100


def check_attention(L, q, k8, v8, ks, vs, what, **masks):
    say("attention", what, tuple(q.shape), tuple(k8.shape), q.dtype)
    ref = R.attention_ref(q, M.widened(k8, ks), M.widened(v8, vs), **masks)
    o, lse = L.cross_attention_q8(q, k8, v8, ks, vs, return_lse=True, **masks)
    R.check(o, *ref["o"], what + " o")
    empty = torch.isinf(ref["lse"][0])
    assert torch.equal(empty, torch.isinf(lse) & (lse < 0)), what + " empty rows"
    assert bool((o.transpose(1, 2)[empty] == 0).all())
    R.check(lse[~empty], ref["lse"][0][~empty], ref["lse"][1][~empty], what + " lse")
    assert torch.equal(L.cross_attention_q8(q, k8, v8, ks, vs, **masks), o)
    return o, lse


SHAPES = [  # B, Sq, Sk, Hq, Hkv, D
    (1, 1, 1, 1, 1, 64), (1, 1, 300, 8, 8, 64), (2, 1, 65, 8, 2, 128), (3, 2, 63, 4, 4, 32), (1, 7, 64, 4, 1, 96),
    (2, 33, 129, 6, 2, 80), (1, 128, 1, 2, 2, 128), (2, 130, 77, 4, 2, 64), (1, 5, 1000, 8, 1, 128),
    (1, 300, 513, 3, 3, 128), (4, 1, 700, 32, 8, 128), (1, 64, 2000, 2, 1, 64), (1, 1, 5000, 4, 2, 128),
    (2, 40, 333, 4, 2, 112), (1, 1, 4097, 8, 1, 16), (64, 1, 300, 16, 8, 64), (3, 600, 700, 16, 16, 128)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention_q8(L, shape, dt):
    B, Sq, Sk, Hq, Hkv, D = shape
    g = gen_of(5)
    q = normal(g, B, Sq, Hq, D, dt=dt)
    (k8, ks), (v8, vs) = states(g, B, Sk, Hkv, D), states(g, B, Sk, Hkv, D)
    check_attention(L, q, k8, v8, ks, vs, "plain")
    kv_len = torch.randint(0, Sk + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    q_len = torch.randint(0, Sq + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    mask = torch.rand(B, Sk, generator=g, device="cuda") > 0.3
    check_attention(L, q, k8, v8, ks, vs, "masked", q_len=q_len, kv_len=kv_len, kv_mask=mask)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("shape", [(5, 700, 400, 16, 8, 64), (40, 300, 200, 6, 2, 128), (70, 300, 150, 3, 3, 64),
                                   (130, 1, 500, 12, 6, 128), (70, 150, 100, 4, 4, 33)], ids=str)
def test_attention_q8_longest_entries_first(L, shape, dt):
    # more workgroups than compute units, entries of every length: equal ones, empty ones, over 64
    B, Sq, Sk, Hq, Hkv, D = shape
    g = gen_of(15)
    q = normal(g, B, Sq, Hq, D, dt=dt)
    (k8, ks), (v8, vs) = states(g, B, Sk, Hkv, D), states(g, B, Sk, Hkv, D)
    kv_len = torch.randint(0, Sk + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    kv_len[B // 2:B // 2 + 3] = kv_len[0]
    kv_len[-1], kv_len[-2] = 0, Sk + 9
    q_len = torch.randint(0, Sq + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    check_attention(L, q, k8, v8, ks, vs, "kv lengths", kv_len=kv_len)
    check_attention(L, q, k8, v8, ks, vs, "both lengths", q_len=q_len, kv_len=kv_len,
                    kv_mask=torch.rand(B, Sk, generator=g, device="cuda") > 0.1)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D", [1, 7, 33, 72, 100, 127])
def test_attention_q8_odd_head_widths(L, D, dt):
    g = gen_of(6)
    for Sq in (1, 37):
        q = normal(g, 2, Sq, 4, D, dt=dt)
        (k8, ks), (v8, vs) = states(g, 2, 191, 2, D), states(g, 2, 191, 2, D)
        check_attention(L, q, k8, v8, ks, vs, f"D={D}")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("Sq", [1, 45, 200])
@pytest.mark.parametrize("D", [64, 128, 100])
def test_attention_q8_masks_and_what_lies_behind_them(L, dt, Sq, D):
    # NaN codes, and scales that are no numbers, wherever nothing may be read
    B, Sk, Hq, Hkv = 8, 200, 4, 2
    g = gen_of(7)
    q = normal(g, B, Sq, Hq, D, dt=dt)
    (k8, ks), (v8, vs) = states(g, B, Sk, Hkv, D), states(g, B, Sk, Hkv, D)
    kv_len = torch.tensor([0, 1, 64, 200, 999, -5, 130, 130], dtype=torch.int32, device="cuda")
    q_len = torch.tensor([Sq, Sq, 0, Sq, max(Sq - 3, 1), Sq, 1, 99], dtype=torch.int32, device="cuda")
    mask = torch.rand(B, Sk, generator=g, device="cuda") > 0.4
    mask[1] = True
    mask[3] = False
    mask[4, :64] = False   # the first block
    mask[6, 64:128] = False  # one between others
    mask[7] = False
    mask[7, 129] = True
    seen = M.allowed(B, Sk, kv_len, mask, "cuda")
    want = check_attention(L, q, k8, v8, ks, vs, "clean", q_len=q_len, kv_len=kv_len, kv_mask=mask)
    k8.view(torch.uint8)[~seen], v8.view(torch.uint8)[~seen] = 0x7F, 0xFF
    block = torch.nn.functional.pad(seen, (0, 4 * 64 - Sk)).view(B, 4, 64).any(2)
    q[torch.arange(Sq, device="cuda") >= q_len[:, None]] = math.nan
    for junk in (math.nan, math.inf, 0.0, -1.0):
        ks[~block], vs[~block] = junk, junk
        for form in (mask, mask.to(torch.uint8) * 255):
            got = L.cross_attention_q8(q, k8, v8, ks, vs, q_len=q_len, kv_len=kv_len, kv_mask=form, return_lse=True)
            assert all(torch.equal(a, b) for a, b in zip(got, want)), junk


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("Sq", [1, 50, 300])
def test_attention_q8_scales_of_every_size(L, Sq, dt):
    # powers of two and others, far apart, rising and falling, the weight where the scale is small
    B, Sk, H, D = 1, 64 * 9 + 5, 2, 64
    g = gen_of(8)
    q = normal(g, B, Sq, H, D, dt=dt)
    x = torch.randn(B, Sk, H, D, generator=g, device="cuda")
    k8, v8 = (x * 100).clamp(-448, 448).to(F8), (x.flip(1) * 100).clamp(-448, 448).to(F8)
    even = torch.full((B, 10, H), 2.0 ** -7, device="cuda")
    steps = torch.arange(10, device="cuda")[None, :, None].expand(B, -1, H)
    for name, ks, vs in (("equal", even, even), ("rising", even, torch.exp2(steps - 12.0)), ("falling", even, torch.exp2(-2.0 * steps - 8)),
                         ("odd", even * 1.37, even * (1 + 0.1 * steps)), ("up and down", even, torch.exp2((steps % 2) * 5.0 - 12)),
                         ("keys", torch.exp2(steps - 12.0), even), ("keys falling", torch.exp2(-steps - 5.0), even),
                         ("one block takes everything", torch.where(steps == 4, 0.5, 2.0 ** -10), torch.where(steps == 4, 2.0 ** -9, 2.0 ** -7))):
        check_attention(L, q, k8, v8, ks.contiguous(), vs.contiguous(), name)
    if dt == "bf16":
        check_attention(L, q, k8, v8, even, torch.exp2((steps % 3) * 30.0 - 40), "far apart")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("Sq", [1, 70])
def test_attention_q8_layouts(L, Sq, dt):
    g = gen_of(9)
    B, Sk, Hq, Hkv, D = 3, 150, 4, 2, 64
    q = normal(g, B, Sq, Hq, D, dt=dt)
    (k8, ks), (v8, vs) = states(g, B, Sk, Hkv, D), states(g, B, Sk, Hkv, D)
    want = check_attention(L, q, k8, v8, ks, vs, "contiguous")
    # a part of a larger cache, heads first; scales of more blocks; queries within wider rows
    big = torch.full((2, B + 1, Hkv, Sk + 40, D), 0x7F, dtype=torch.uint8, device="cuda")
    big[0, :B, :, :Sk], big[1, :B, :, :Sk] = (x.view(torch.uint8).transpose(1, 2) for x in (k8, v8))
    big = big.view(F8)
    k2, v2 = (big[i, :B, :, :Sk].transpose(1, 2) for i in (0, 1))
    s2 = torch.full((2, B, 7, Hkv), math.nan, device="cuda")
    s2[0, :, :3], s2[1, :, :3] = ks, vs
    q2 = torch.full((B, Sq, 3, Hq, D + 8), math.nan, dtype=q.dtype, device="cuda")
    q2[:, :, 1, :, :D] = q
    out = torch.zeros(B, Sq, 3, Hq, D + 8, dtype=q.dtype, device="cuda")[:, :, 1, :, :D]
    got = L.cross_attention_q8(q2[:, :, 1, :, :D], k2, v2, s2[0, :, :3], s2[1, :, :3], o=out, return_lse=True)
    assert got[0] is out and all(torch.equal(a, b) for a, b in zip(got, want))
    # bytes on odd addresses
    odd = torch.full((B * Sk * Hkv * (D + 3) + 1,), 0x7F, dtype=torch.uint8, device="cuda")[1:].view(B, Sk, Hkv, D + 3)
    odd[..., :D] = k8.view(torch.uint8)
    check_attention(L, q, odd.view(F8)[..., :D], v8, ks, vs, "odd rows")
    # one view's states for every batch entry
    one = [t[:1].expand(B, *t.shape[1:]) for t in (k8, v8, ks, vs)]
    check_attention(L, q, *one, "broadcast")
    for Sq2, Sk2, B2 in ((5, 0, 2), (0, 5, 2), (5, 5, 0)):
        o, lse = L.cross_attention_q8(q.new_empty(B2, Sq2, Hq, D), *(torch.empty(B2, Sk2, Hkv, D, device="cuda").to(F8) for _ in range(2)),
                                      *(torch.empty(B2, -(-Sk2 // 64), Hkv, device="cuda") for _ in range(2)), return_lse=True)
        assert bool((o == 0).all()) and bool((lse == -math.inf).all())


def test_attention_q8_offsets_beyond_32_bits(L):
    # rows 2^31 bytes and more apart
    g = gen_of(10)
    Sk, step = 3, (1 << 31) + 64
    big = torch.zeros((Sk - 1) * step + 128, dtype=torch.uint8, device="cuda").view(F8)
    k8 = big.as_strided((1, Sk, 1, 64), (big.numel(), step, 64, 1))
    v8 = big[64:].as_strided((1, Sk, 1, 64), (big.numel(), step, 64, 1))
    (a, ks), (b, vs) = states(g, 1, Sk, 1, 64), states(g, 1, Sk, 1, 64)
    k8.view(torch.uint8).copy_(a.view(torch.uint8))
    v8.view(torch.uint8).copy_(b.view(torch.uint8))
    for Sq in (1, 40):
        check_attention(L, normal(g, 1, Sq, 1, 64), k8, v8, ks, vs, "far rows")
    del k8, v8, big
    torch.cuda.empty_cache()


def test_attention_q8_long_states_for_one_token(L):
    g = gen_of(11)
    (k8, ks), (v8, vs) = states(g, 1, 40003, 2, 128), states(g, 1, 40003, 2, 128)
    check_attention(L, normal(g, 1, 1, 8, 128), k8, v8, ks, vs, "long")


def test_attention_of_quantized_states(L):
    # both together: as attention to what the 8-bit states stand for; and near the
    # 16-bit states, as e4m3 holds them: a score is off by 2^-4 of sum |q k|, at most, and
    # a value by 2^-4 of its own
    g = gen_of(12)
    B, Sq, Sk, D = 2, 60, 500, 64
    q, k, v = normal(g, B, Sq, 4, D), normal(g, B, Sk, 2, D, std=0.3), normal(g, B, Sk, 2, D)
    lens = torch.tensor([500, 77], dtype=torch.int32, device="cuda")
    packed = L.quantize_states(k, v, kv_len=lens)
    o, _ = check_attention(L, q, *packed, "quantized", kv_len=lens)
    full = L.cross_attention(q, k, v, kv_len=lens)
    off = 2.0 ** -4 * 0.125 * float((q.abs().double().amax((1, 2)) [:, None, None, :] * k.abs().double()).sum(3).amax())
    assert float((o - full).abs().max()) <= (math.exp(2 * off) - 1 + 2.0 ** -4) * float(v.abs().max())
    assert float((o.double() - full.double()).norm() / full.double().norm()) < 2.0 ** -3


def test_states_refusals(L):
    from paper_2210_10108_amd import pnerf
    g = gen_of(13)
    q, k = normal(g, 2, 5, 4, 64), normal(g, 2, 70, 2, 64)
    k8, v8, ks, vs = L.quantize_states(k, k)
    for kind, fn in [(TypeError, lambda: L.quantize_states(k, k.bfloat16())), (TypeError, lambda: L.quantize_states(k8, v8)),
                     (ValueError, lambda: L.quantize_states(k, k[:, :3])), (ValueError, lambda: L.quantize_states(k[0], k[0])),
                     (TypeError, lambda: L.quantize_states(k, k, k8=k)), (ValueError, lambda: L.quantize_states(k, k, k_scale=ks[:, :1])),
                     (TypeError, lambda: L.cross_attention_q8(q, k, v8, ks, vs)), (TypeError, lambda: L.cross_attention_q8(q, k8, v8, ks.half(), vs)),
                     (ValueError, lambda: L.cross_attention_q8(q, k8, v8, ks[:, :1], vs)), (ValueError, lambda: L.cross_attention_q8(q, k8, v8[:, :1], ks, vs)),
                     (ValueError, lambda: L.cross_attention_q8(q[0], k8, v8, ks, vs)), (TypeError, lambda: L.cross_attention_q8(k8, k8, v8, ks, vs))]:
        with pytest.raises(kind):
            fn()
    wide = normal(g, 1, 3, 1, 129)
    for status, fn in [(pnerf.ERR_NOT_SUPPORTED, lambda: L.quantize_states(k.float(), k.float())),
                       (pnerf.ERR_NOT_SUPPORTED, lambda: L.quantize_states(wide, wide)),
                       (pnerf.ERR_INVALID_ARG, lambda: L.quantize_states(k, k, k8=k8[:1].expand(2, -1, -1, -1))),
                       (pnerf.ERR_NOT_SUPPORTED, lambda: L.cross_attention_q8(q.float(), k8, v8, ks, vs)),
                       (pnerf.ERR_INVALID_ARG, lambda: L.cross_attention_q8(q[:, :, :3], k8, v8, ks, vs)),
                       (pnerf.ERR_INVALID_ARG, lambda: L.cross_attention_q8(q, k8, v8, ks, vs, scale=0.0))]:
        with pytest.raises(pnerf.PnerfError) as e:
            fn()
        assert e.value.status == status
