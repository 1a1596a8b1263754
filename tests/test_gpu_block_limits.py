"""The operators of include/mtgr_block.h at the ends of their documented ranges, against 64-bit definitions."""
import pytest
import torch

from paper_2505_18654_amd import ops
from tests.block_ref import keep_mask, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("rows, cols", [(1, 1 << 22), (3, (1 << 22) + 8)])
def test_dropout_of_dense_rows_of_any_width(rows, cols):
    print(f"[limits] dropout {rows} x {cols}", flush=True)
    x, r = normal((rows, cols), 1), normal((rows, cols), 2)
    rng = torch.tensor([31, 4], dtype=torch.int64, device="cuda")
    got = ops.dropout(x, 0.5, rng, 6, residual=r)
    # (p = 0.5 doubles exactly: one rounding, that of the sum)
    keep = keep_mask((rows, cols), 0.5, 31, 4, 6).cuda()
    assert torch.equal(got, (torch.where(keep, 2 * x.float(), 0.0) + r.float()).bfloat16())
