"""Rates that fp32 does not hold are refused before anything is launched (no GPU: see test_operator_refusals.py)."""
import pytest

from paper_2203_05705_b200 import ard
from test_operator_refusals import CTX, STEP, TENSOR


@pytest.mark.parametrize("number", [3.5e38, 1e39, 1e300])
@pytest.mark.parametrize("key", ["lr", "eps", "weight_decay"])
def test_numbers_beyond_fp32(key, number):
    """lr and weight_decay of infinity made parameters NaN."""
    step, tensor = ({**d, key: number} if key in d else d for d in (STEP, TENSOR))
    with pytest.raises(ard.ArdError) as e:
        ard.ard_adamw_step(CTX, ard.adamw_tensors([tensor]), 1, *step.values(), stream=0)
    assert e.value.status == ard.ARD_ERR_INVALID_ARG
