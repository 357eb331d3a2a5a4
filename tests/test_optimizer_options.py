"""Options of us_adamw: learning rates that are numbers of float64 but none of float32, and the rounding of states (1 invalid argument, 5 no device: everything else was in order)."""
import pytest
import torch

from paper_2303_11257_b200 import optim
from tests.test_optimizer_refusals import EIGHT, adamw, tensor

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="valid calls with fake addresses")


def test_learning_rates_beyond_float32():
    assert adamw(tensor(), lr=3e38) == 5 and adamw(tensor(), lr=1e39) == 1 and adamw(tensor(), lr=1e300) == 1


def test_rounding_of_states():
    def with_rounding(kind, **kw):
        t = tensor(**kw)
        t.rounding = kind
        return adamw(t)
    assert with_rounding(0) == 5 and with_rounding(0, **EIGHT) == 5 and with_rounding(1, **EIGHT) == 5
    assert with_rounding(1) == 2                                   # states in 32 bits are not rounded
    assert with_rounding(2, **EIGHT) == 1 and with_rounding(-1) == 1
    p = [torch.zeros(4)]
    for kw in (dict(rounding="random"), dict(states="8bit", rounding="up")):
        with pytest.raises(ValueError, match="rounding"):
            optim.AdamW(p, p, **kw)
