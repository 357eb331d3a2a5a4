"""Options of us_adamw that are numbers of float64 but none of float32 (1 invalid argument, 5 no device: everything else was in order)."""
import pytest
import torch

from tests.test_optimizer_refusals import adamw, tensor

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="valid calls with fake addresses")


def test_learning_rates_beyond_float32():
    assert adamw(tensor(), lr=3e38) == 5 and adamw(tensor(), lr=1e39) == 1 and adamw(tensor(), lr=1e300) == 1
