"""The streams that GPU tests get (conftest.py)."""
import pytest

from conftest import _runs_beside_the_default_stream
from util import torch_mod

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("more", [0, 1, 2, 3, 4, 5])
def test_the_first_stream_runs_beside_the_default_one_however_many_were_taken(more):
    torch = torch_mod()
    stream = torch.cuda.Stream()
    assert any(_runs_beside_the_default_stream(torch, stream) for _ in range(3))
    for _ in range(more):
        torch.cuda.Stream()
