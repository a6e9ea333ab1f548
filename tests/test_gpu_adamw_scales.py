"""States in 8 bits of tensors whose scales lie on a 16-byte grid (brought by bulk copies) and off it (fetched by lanes), in turn in one table: a warp's tiles
of either kind follow one another in the same places of shared memory."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx
from paper_2203_05705_b200 import ard

pytestmark = pytest.mark.gpu


def _table(offs, n, seed):
    rng = np.random.default_rng(seed)
    rows = []
    for off in offs:
        f = lambda scale, k=n: torch.from_numpy((rng.standard_normal(k) * scale).astype(np.float32)).cuda()  # noqa: E731
        blocks = n // 128
        code = lambda: torch.from_numpy(rng.integers(0, 120, n).astype(np.uint8)).cuda()  # noqa: E731
        scale = lambda: (f(1e-5, blocks + 4).abs() + 1e-7)[off:off + blocks]  # noqa: E731
        rows.append(dict(rows=1, cols=n, p=f(0.1), g=f(1e-2), m=code(), v=code(), m_scale=scale(), v_scale=scale(), weight_decay=0.1))
    return rows


@pytest.mark.parametrize("per_tensor", [1, 2, 3])
def test_scales_on_and_off_the_grid_in_one_table(per_tensor):
    """The same bits as one tensor after the other."""
    ctx = Ctx(0)
    try:
        # a CTA's warps take neighbouring tiles and go on by 2368 of them: tensors a little shorter than that, so that a warp meets both kinds
        n = 512 * 2368 * per_tensor // 2 + 512 * 5
        offs = [0, 1, 0, 3, 2, 0, 1, 0]
        together, alone = _table(offs, n, 7), _table(offs, n, 7)
        for k in range(1, 4):
            ard.ard_adamw_step(ctx.h, ard.adamw_tensors(together), len(offs), 1e-3, 0.9, 0.999, 1e-8, 8, 5, k)
            for i in range(len(offs)):
                # the number of a tensor in its table is part of its random words' counter: empty ones before it
                table = ard.adamw_tensors([{"rows": 0, "cols": 1, "g": None, "g_dtype": 0}] * i + [alone[i]])
                ard.ard_adamw_step(ctx.h, table, i + 1, 1e-3, 0.9, 0.999, 1e-8, 8, 5, k)
        torch.cuda.synchronize()
        assert ard.ard_last_device_status(ctx.h) == 0
        for i, (a, b) in enumerate(zip(together, alone)):
            for key in ("p", "m", "v", "m_scale", "v_scale"):
                assert torch.equal(a[key], b[key]), (i, key)
            assert bool(torch.isfinite(a["p"]).all())
    finally:
        ctx.close()
