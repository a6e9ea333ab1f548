"""Pointers that lie inside an element are refused before anything is launched (no GPU: see test_operator_refusals.py)."""
import pytest

from paper_2203_05705_b200 import ard
from test_operator_refusals import CTX, GLR_BWD, GLR_FWD, LN_BWD, LN_FWD, P, STEP, TENSOR

BF_ONLY = {"X", "Y", "dY", "dX", "Zf", "Zg", "Zo", "dZf", "dZg", "dZo"}
LN_F = {**LN_FWD, "weight": P[8], "bias": P[9], "mean": P[10], "rstd": P[11]}
LN_B = {**LN_BWD, "weight": P[8], "dweight": P[9], "dbias": P[10]}
GLR_F = {**GLR_FWD, "Zo": P[8], "lens": P[9], "h0": P[10], "hT": P[11], "S": P[12]}
GLR_B = {**GLR_BWD, "lens": P[8], "dhT": P[9], "dh0": P[10]}
POINTERS = [(name, good, k) for name, good in (("ard_layer_norm_fwd", LN_F), ("ard_layer_norm_bwd", LN_B), ("ard_glr_forward", GLR_F), ("ard_glr_backward", GLR_B))
            for k, v in good.items() if v in P]


@pytest.mark.parametrize("dtype", [ard.ARD_F32, ard.ARD_BF16])
@pytest.mark.parametrize("name,good,key", POINTERS)
def test_layer_norm_and_recurrence(name, good, key, dtype):
    for off in (1, 2, 3):
        if off == 2 and dtype == ard.ARD_BF16 and key in BF_ONLY:
            continue    # a whole element
        with pytest.raises(ard.ArdError) as e:
            getattr(ard, name)(CTX, *{**good, "dtype": dtype, key: good[key] + off}.values(), stream=0)
        assert e.value.status == ard.ARD_ERR_ALIGNMENT


def test_optimiser():
    def step(bits, table, **more):
        with pytest.raises(ard.ArdError) as e:
            ard.ard_adamw_step(CTX, table, 2, *{**STEP, "bits": bits}.values(), stream=0, **more)
        return e.value.status

    def norm(table, out):
        with pytest.raises(ard.ArdError) as e:
            ard.ard_grad_norm(CTX, table, 2, 1.0, out, stream=0)
        return e.value.status

    good = ard.adamw_tensors([TENSOR, TENSOR])
    for bits, key, off in [(b, k, o) for b in (8, 32) for k, o in (("p", 2), ("g", 2), ("g", 1), ("w", 1))] + [(32, "m", 1), (32, "v", 2), (8, "m_scale", 2), (8, "v_scale", 1)]:
        bad = ard.adamw_tensors([TENSOR, {**TENSOR, key: TENSOR[key] + off}])
        assert step(bits, bad) == ard.ARD_ERR_ALIGNMENT, (bits, key, off)
        if key == "g":
            assert norm(bad, P[8]) == ard.ARD_ERR_ALIGNMENT
    assert step(8, ard.adamw_tensors([TENSOR, {**TENSOR, "g_dtype": ard.ARD_BF16, "g": TENSOR["g"] + 1}])) == ard.ARD_ERR_ALIGNMENT
    for more in (dict(step_counter=P[9] + 4), dict(lr_factor=P[9] + 2), dict(grad_factor=P[9] + 1)):
        assert step(8, good, **more) == ard.ARD_ERR_ALIGNMENT
    assert norm(good, P[9] + 2) == ard.ARD_ERR_ALIGNMENT
