"""The sampler's binding without a GPU: what it hands to the library, and its refusals.

The library's call is replaced by one that notes its arguments; tensors are the
host's, and no kernel runs.
"""

import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_2608_13076_amd import sampling

ROWS, V = 4, 10


class Recorder:
    """Takes the place of the library: a call's parameters, as it reads them."""

    def __init__(self):
        self.calls = []

    def spade_sample(self, *args):
        p = args[6]._obj
        at = ["temperature", "top_k", "top_p", "min_p"]
        self.calls.append(SimpleNamespace(per=args[5], all={n: getattr(p, n) for n in at},
                                          given={n: a for n, a in zip(at, args[7:11])}))
        return 0


@pytest.fixture
def sampler(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(sampling, "load_library", lambda: SimpleNamespace(
        spade_sample_workspace_bytes=lambda rows, vocab: 256, spade_sample=Recorder().spade_sample))
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    s = sampling.Sampler(ROWS, V, device="cpu")
    s._index = -1  # (what a host tensor's get_device gives)
    s.lib = Recorder()
    return s


def draw(s, **kw):
    return s.draw(torch.zeros(ROWS, V), torch.zeros(ROWS), **kw)


def test_numbers_and_tensors(sampler):
    t = torch.full((2,), 0.5)
    draw(sampler, temperature=0.25, top_k=3, top_p=0.5, min_p=0.125)
    draw(sampler, top_p=t)
    draw(sampler)
    a, b, c = sampler.lib.calls
    assert a.all == dict(temperature=0.25, top_k=3, top_p=0.5, min_p=0.125) and a.per == ROWS
    assert set(a.given.values()) == {None}
    assert b.given == dict(temperature=None, top_k=None, top_p=t.data_ptr(), min_p=None) and b.per == 2
    assert c.all == dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)


@pytest.mark.parametrize("name,dtype", [("temperature", torch.float32), ("top_k", torch.int32), ("top_p", torch.float32),
                                        ("min_p", torch.float32)])
def test_no_requests_are_refused(sampler, name, dtype):
    """A tensor of no requests has no address: the library would take the number of an
    earlier call."""
    with pytest.raises(ValueError):
        draw(sampler, **{name: torch.empty(0, dtype=dtype)})
    # nor does it hide that another parameter has other requests
    with pytest.raises(ValueError):
        draw(sampler, temperature=torch.empty(0), min_p=torch.zeros(2))
    with pytest.raises(ValueError):
        draw(sampler, temperature=torch.ones(2), min_p=torch.empty(0))
    assert not sampler.lib.calls


@pytest.mark.parametrize("k", [V, V + 1, 2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 3, 2 ** 63 - 1, 10 ** 30, -1, -2 ** 31 - 7,
                               3 - 2 ** 32])
def test_a_top_k_beyond_32_bits_is_no_limit(sampler, k):
    draw(sampler, top_k=k)
    got = sampler.lib.calls[0].all["top_k"]
    assert got <= 0 or got >= V
