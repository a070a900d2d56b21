"""The operators of test_gpu_more_layers on a stream that is named: their work is there
and nowhere else.  The current stream has other work in front of it all the while, and
results are read on the named one before that is done: a launch that went to the current
stream has not run then.  (Each pass has inputs of its own, so that what an earlier one
left in the memory is wrong.)"""
import pytest
import torch

from .test_gpu_layers import gen_of
from .test_gpu_more_layers import calls

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2210_10108_amd import layers
    layers.lib()
    return layers


def hold_up(busy):
    """Some 200 ms of work for the current stream; an event after it."""
    for _ in range(400):
        busy.add_(1.0)  # 2 GB each
    done = torch.cuda.Event()
    done.record()
    return done


def beside(busy):
    """A stream whose work does not wait for the current one's: streams share a few
    hardware queues, and two of one queue follow each other."""
    for _ in range(16):
        s = torch.cuda.Stream()
        done, ran = hold_up(busy), torch.cuda.Event()
        ran.record(s)
        ran.synchronize()
        if not done.query():
            torch.cuda.synchronize()
            return s
    pytest.fail("no stream runs beside the current one")


def test_work_is_on_the_named_stream(L):
    runs = [calls(L, gen_of(21 + i))[0] for i in range(3)]
    last = calls(L, gen_of(31))[0]
    wants = [[t.cpu() for t in run()] for run in runs]
    busy = torch.zeros(1 << 28, device="cuda")
    other = beside(busy)
    for _ in range(3):
        last(), last(stream=other)
    torch.cuda.synchronize()
    for run, want in zip(runs, wants):
        done = hold_up(busy)
        got = run(stream=other)
        with torch.cuda.stream(other):
            host = [t.cpu() for t in got]
        assert not done.query(), "the current stream was to be behind"
        assert all(torch.equal(a, b) for a, b in zip(want, host))
        torch.cuda.synchronize()
        last(), last(stream=other)
        torch.cuda.synchronize()
