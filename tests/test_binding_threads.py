"""One sampler and one cache in two threads, without a GPU.

A call's kernels share the object's workspace, so the launches of two calls must not
mix, also on one stream, and a call must have its own parameters.  The library's calls
are replaced by ones that wait inside for a second thread, which may not come in.
"""

import contextlib
import threading
from types import SimpleNamespace

import pytest
import torch

from paper_2608_13076_amd import sampling, tree


@pytest.fixture
def host(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    return monkeypatch


class Inside:
    """The library's call: notes what it is given when it comes in and when it leaves."""

    def __init__(self, read):
        self.read, self.here, self.most, self.seen = read, 0, 0, []
        self.count, self.second = threading.Lock(), threading.Event()

    def __call__(self, *args):
        with self.count:
            self.here += 1
            self.most = max(self.most, self.here)
            if self.here == 2:
                self.second.set()
        before = self.read(args)
        self.second.wait(0.3)  # (long enough for the other thread, if it can come in)
        self.seen.append((before, self.read(args)))
        with self.count:
            self.here -= 1
        return 0


def in_two_threads(f):
    errors = []

    def run(i):
        try:
            f(i)
        except Exception as e:  # noqa: BLE001 (shown below)
            errors.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(30)
    assert not errors and not any(t.is_alive() for t in threads), errors


def test_a_sampler_in_two_threads(host):
    call = Inside(lambda args: (args[6]._obj.temperature, args[6]._obj.top_k))
    host.setattr(sampling, "load_library", lambda: SimpleNamespace(
        spade_sample_workspace_bytes=lambda rows, vocab: 256, spade_sample=call))
    s = sampling.Sampler(4, 10, device="cpu")
    s._index = -1  # (what a host tensor's get_device gives)
    in_two_threads(lambda i: s.draw(torch.zeros(4, 10), torch.zeros(4), temperature=0.5 + i, top_k=1 + i))
    assert sorted(call.seen) == [((0.5, 1), (0.5, 1)), ((1.5, 2), (1.5, 2))]
    assert call.most == 1


def test_a_cache_in_two_threads(host):
    call = Inside(lambda args: args[1])
    host.setattr(tree, "load_library", lambda: SimpleNamespace(
        spade_tree_bytes=lambda s: 256, spade_tree_workspace_bytes=lambda s, r: 256, spade_tree_attend=call))
    c = tree.TreeCache(2, 1, 2, 1, 64, 100, max_rows=4, device="cpu")
    c._index = -1
    in_two_threads(lambda i: c.attend(i, torch.zeros(1, 2, 2, 64)))
    assert sorted(call.seen) == [(0, 0), (1, 1)]
    assert call.most == 1
