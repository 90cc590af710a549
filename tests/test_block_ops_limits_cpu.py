"""What the operators of a trained block refuse before they reach the library.  No GPU."""
import pytest
import torch

from paper_2501_02379_b200 import binding as B
from paper_2501_02379_b200 import build as builder


@pytest.fixture(scope="module", autouse=True)
def _built():
    builder.build()


def test_packed_matrices_that_are_not_on_a_gpu_are_refused():
    host = B.Packed(torch.zeros(B._packed_bytes(4, 64), dtype=torch.uint8), 4, 64, torch.float32)
    for call in (lambda: B.act_unpack(host), lambda: B.act_unpack(host, out=torch.zeros(4, 64)), lambda: B.act_unpack(host.data), lambda: B.act_unpack(None)):
        with pytest.raises(ValueError):
            call()
