"""What the entry points of include/mtgr_block.h take and refuse at the ends of their documented ranges, on the CPU: a
call that gets past one check is told apart by the next check's refusal, so that nothing is launched."""
import math

import pytest

from paper_2505_18654_amd import hstu
from tests.test_block_cpu import FAKE, INVALID, NULL, UNSUPPORTED, drop, loss_bwd, loss_fwd, loss_problem, status_of


@pytest.mark.parametrize("cols", [1 << 22, (1 << 22) + 8, 1 << 30])
def test_dropout_takes_dense_rows_of_any_width(cols):
    # (rng is checked after the matrices)
    wide = dict(cols=cols, ld_x=cols, ld_out=cols, ld_residual=cols, residual=FAKE, rng=None)
    for rows in (1, 2):
        assert status_of(drop, rows=rows, **wide) == NULL
        assert "rng" in hstu.mtgr_last_error_message()
    for gap in ("ld_x", "ld_out", "ld_residual"):            # rows with gaps keep the limit of the other operators
        assert status_of(drop, **{**wide, gap: cols + 8}) == UNSUPPORTED


@pytest.mark.parametrize("scale", [2.37e38, -2.37e38, 3.4e38])
def test_loss_scale_is_a_number_in_units_of_log_2(scale):
    """The logits are formed as scale log2(e) x.w: beyond 2.358e38 that factor is infinite."""
    for call in (loss_fwd, loss_bwd):
        assert status_of(call, loss_problem(scale=scale)) == INVALID
        assert status_of(call, loss_problem(scale=math.copysign(2.35e38, scale)), x=None) == NULL
