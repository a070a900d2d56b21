"""The layer operators' slower forms where their work is split: attention element
by element over parts of the keys and rows, linear layers over copies of
strided operands; and that a call's work is on the stream that it names."""
import sys

import pytest
import torch

from . import layers_common as R
from . import test_gpu_layers as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2210_10108_amd import layers
    layers.lib()
    return layers


# ---------------------------------------------------------------- attention
def off_by_one(t):
    """t's values in rows on odd addresses."""
    B, S, H, D = t.shape
    w = torch.full((B * S * H * (D + 3) + 1,), float("nan"), dtype=t.dtype, device=t.device)
    w = w[1:].view(B, S, H, D + 3)
    w[..., :D] = t
    return w[..., :D]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("B,Sq,Sk,Hq,Hkv,D", [
    (1, 1, 5001, 4, 2, 100), (1, 40, 5001, 4, 1, 33), (2, 700, 1003, 4, 2, 100), (1, 700, 5001, 2, 1, 100),
    (1, 1, 9000, 3, 3, 33), (1, 1000, 130, 8, 2, 128), (1, 700, 1003, 4, 1, 128), (1, 3, 5001, 16, 2, 128),
    (3, 520, 700, 4, 2, 64)])
def test_attention_element_by_element_in_parts(L, B, Sq, Sk, Hq, Hkv, D, masked, dt):
    g = T.gen_of(100)
    q, do = T.normal(g, B, Sq, Hq, D, dt=dt), T.normal(g, B, Sq, Hq, D, dt=dt)
    k, v = T.normal(g, B, Sk, Hkv, D, dt=dt), T.normal(g, B, Sk, Hkv, D, dt=dt)
    if D % 8 == 0:
        q, do, k, v = (off_by_one(t) for t in (q, do, k, v))
    masks = {}
    if masked:
        # the first entry ends within a part, so that its last ones are empty
        masks = dict(kv_len=torch.tensor([Sk * 2 // 5] + [Sk - 3 - i for i in range(B - 1)], dtype=torch.int32, device="cuda"),
                     q_len=torch.tensor([Sq - Sq // 3] + [Sq] * (B - 1), dtype=torch.int32, device="cuda"),
                     kv_mask=torch.rand(B, Sk, generator=g, device="cuda") > 0.2)
        masks["kv_mask"][:, 64:300] = False
    T.check_attention(L, q, k, v, do, f"parts D={D} masked={masked}", **masks)


# ---------------------------------------------------------------- linear
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("pad,off", [(3, 1), (8, 4), (5, 0), (0, 1)])
@pytest.mark.parametrize("M,K,N", [(300, 2100, 1001), (7, 2048, 1032), (600, 512, 520)])
def test_linear_copies_of_strided_operands(L, M, K, N, pad, off, dt):
    g = T.gen_of(101)

    def wide(rows, cols, std=1.0):
        flat = torch.full((rows * (cols + pad) + off,), float("nan"), dtype=R.DT[dt], device="cuda")
        t = flat[off:].view(rows, cols + pad)[:, :cols]
        t.copy_(T.normal(g, rows, cols, dt=dt, std=std))
        return t
    x, w, dy, res = wide(M, K), wide(K, N, K ** -0.5), wide(M, N), wide(M, N)
    b = T.normal(g, N, dt=dt)
    T.check_linear(L, x, w, b, res, "gelu", dy, f"pad {pad} off {off}")
    T.check_linear(L, x, w, None, None, "none", dy, f"pad {pad} off {off}, product alone")


# ---------------------------------------------------------------- streams
def test_results_are_there_on_the_stream_that_was_named(L):
    # the current stream is held by long work; on the other one the results are
    # complete before that work is.  (Work sent to the current stream instead would
    # still be queued when the copies to the host are made.)
    run, _ = T._calls(L, T.gen_of(102))
    want = [t.cpu() for t in run()]
    host = [torch.empty_like(t, pin_memory=True) for t in want]
    busy, small = torch.zeros(1 << 27, device="cuda"), torch.zeros(64, device="cuda")
    torch.cuda.synchronize()

    def hold():
        for _ in range(400):
            busy.add_(1.0)
        e = torch.cuda.Event()
        e.record()
        return e
    for _ in range(8):  # a stream whose queue is not the current one's
        other = torch.cuda.Stream()
        with torch.cuda.stream(other):
            small.add_(1.0)
        torch.cuda.synchronize()
        held = hold()
        with torch.cuda.stream(other):
            small.add_(1.0)
        other.synchronize()
        apart = not held.query()
        torch.cuda.synchronize()
        if apart:
            break
    else:
        pytest.skip("no stream here runs beside the current one")
    for named in (True, False):
        for h in host:
            h.zero_()
        held = hold()
        if named:
            got = run(stream=other)
        else:
            with torch.cuda.stream(other):
                got = run()
        with torch.cuda.stream(other):
            for h, t in zip(host, got):
                h.copy_(t, non_blocking=True)
        other.synchronize()
        assert not held.query(), "the held stream came first"
        assert all(torch.equal(h, w) for h, w in zip(host, want)), named
        torch.cuda.synchronize()
    sys.stderr.write("[gpu] streams: results beside held work\n")
