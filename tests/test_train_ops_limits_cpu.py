"""Refusals of the operators around the step that a machine without a GPU, or with one, can only see through stand-ins."""
import pytest
import torch

from paper_2501_02379_b200 import binding as B
from paper_2501_02379_b200 import build as builder


@pytest.fixture(scope="module", autouse=True)
def _built():
    builder.build()


class Elsewhere:
    """What the binding asks of a scale, on a device of our choice."""

    dtype, is_cuda = torch.float32, True

    def __init__(self, index, entries=1):
        self.index, self.entries = index, entries

    def get_device(self):
        return self.index

    def numel(self):
        return self.entries

    def data_ptr(self):
        return 0x1000


def test_a_scale_on_another_device_is_refused():
    assert B._scalar_ptr(Elsewhere(0), 0) == 0x1000 and B._scalar_ptr(Elsewhere(3), 3) == 0x1000 and B._scalar_ptr(None, 0) is None
    for scale, index in ((Elsewhere(1), 0), (Elsewhere(0), 1), (Elsewhere(0, 2), 0)):
        with pytest.raises(ValueError):
            B._scalar_ptr(scale, index)


def test_steps_refuse_a_scale_on_another_device():
    class State:
        handle = None

    class Tensor(Elsewhere):
        pass

    with pytest.raises(ValueError):
        B.TgradState.step_scaled(State(), Tensor(0), Tensor(0), Elsewhere(1), stream=0)
    with pytest.raises(ValueError):
        B.step_batched([State()], [Tensor(0)], [Tensor(0)], stream=0, scale=Elsewhere(1))
