import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu on the GPU box)")


@pytest.fixture(scope="session")
def rng():
    import numpy as np
    return np.random.default_rng(20080343)


def _runs_beside_the_default_stream(torch, stream):
    """Whether work of the default stream ends while the stream sleeps.  (A delay of the host can only make it look as if it did not.)"""
    one, end = torch.zeros(1, device="cuda"), torch.cuda.Event()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(10_000_000)   # some four milliseconds
        end.record()
    one.add_(1.0)
    torch.cuda.current_stream().synchronize()
    beside = not end.query()
    torch.cuda.synchronize()
    return beside


class _StreamPool:
    """torch hands out its pooled streams in turn, and the runtime puts them on four hardware queues, one of which the default stream has too:
    work of a stream there waits for the default stream's and the other way round."""

    def __init__(self):
        import torch
        self.torch = torch
        self.beside = []   # of the pool's streams, in the order in which they are handed out
        self.place = {}
        while True:
            stream = torch.cuda.Stream()
            if stream.cuda_stream in self.place:
                break
            self.place[stream.cuda_stream] = len(self.beside)
            self.beside.append(_runs_beside_the_default_stream(torch, stream))

    def go_to_one_beside_the_default_stream(self):
        for _ in self.beside:
            if self.beside[(self.place[self.torch.cuda.Stream().cuda_stream] + 1) % len(self.beside)]:
                return


_pool = []


@pytest.fixture(autouse=True)
def next_stream_runs_beside_the_default_one(request):
    """The first stream that a GPU test takes has another hardware queue than the default stream, however many the tests before took."""
    if request.node.get_closest_marker("gpu"):
        if not _pool:
            _pool.append(_StreamPool())
        _pool[0].go_to_one_beside_the_default_stream()
