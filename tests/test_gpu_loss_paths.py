"""The softmax loss on each of its kernels, against its 64-bit definition: the sizes of tests/block_shapes.py, whose
kernels tests/test_block_plans_cpu.py asserts.  Bounds: tests/block_ref.py."""
import pytest
import torch

from paper_2505_18654_amd import ops
from tests import block_shapes as S
from tests.block_ref import normal
from tests.test_gpu_softmax_loss import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def make(N, V, d, labels, bias=True, seed=1, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    t = torch.full((N,), -1)
    t[torch.randperm(N, generator=g)[:labels]] = torch.randint(0, V, (labels,), generator=g)
    return (normal((N, d), seed), normal((V, d), seed + 1, spread * d ** -0.5), t.cuda(),
            (0.7 * torch.randn(V, generator=g)).cuda() if bias else None, (torch.randn(N, generator=g) / labels).cuda())


@pytest.mark.parametrize("N, V, d, labels", S.LOSS)
def test_loss_and_gradients(N, V, d, labels):
    print(f"[loss] N={N} V={V} d={d} labels={labels}", flush=True)
    x, w, t, b, dloss = make(N, V, d, labels)
    first = check(x, w, t, b, dloss)
    ws = ops.softmax_loss_workspace(N, V, d, backward=True)
    ws.fill_(255)                                        # NaN where a kernel reads what no kernel wrote
    again = ops.softmax_loss_bwd(dloss, x, w, t, first[1], bias=b, scale=0.9, workspace=ws)
    assert all(torch.equal(p, q) for p, q in zip(first[2:], again))
