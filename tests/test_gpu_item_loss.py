"""The embedding table's item loss: what its gradient adds up to for items that a batch holds several times."""
import pytest
import torch

from paper_2505_18654_amd import ops
from paper_2505_18654_amd.embedding import DynamicEmbedding
from tests.block_ref import normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def batch_of(ids, dim=32, rows=512, dtype=torch.bfloat16):
    table = DynamicEmbedding(row_capacity=rows, dim=dim, dtype=dtype)
    _, batch = table.lookup(ids.cuda(), now=1)
    table.values.copy_((0.3 * torch.randn(rows, dim, generator=torch.Generator().manual_seed(2))).to(dtype))
    return table, batch


def test_positions_add_up_to_the_items_gradient_exactly():
    """grad_out of an item's positions sums to the item's gradient as softmax_loss_bwd rounds it, with no rounding of
    its own, whatever the number of positions (3, 5, 7, ... do not divide a bf16 number)."""
    g = torch.Generator().manual_seed(1)
    ids = torch.cat([torch.full((k,), 100 + k) for k in range(1, 24)])[torch.randperm(276, generator=g)]
    table, batch = batch_of(ids)
    x, labels = normal((60, 32), 3), torch.randint(-40, 276, (60,), generator=g).cuda()
    dloss = torch.full((60,), 1.0 / 60, device="cuda")
    _, saved = table.item_loss(x, batch, labels, scale=0.7)
    dx, grad_out = table.item_loss_bwd(dloss, saved)
    w, targets, lse, bias = saved[1:5]
    want_dx, dw, _ = ops.softmax_loss_bwd(dloss, x, w, targets, lse, bias=bias, scale=0.7)
    item = batch.inverse[:276].long()
    total = torch.zeros(w.shape, dtype=torch.float64, device="cuda").index_add_(0, item, grad_out.double())
    n = int(batch.num_unique)
    assert n == 23 and dw[:n].any()
    assert torch.equal(total[:n], dw[:n].double()) and torch.equal(dx, want_dx)
    again = table.item_loss_bwd(dloss, saved)[1]
    assert torch.equal(again, grad_out)


def test_a_hot_item_and_an_empty_batch():
    """More positions of one item than the tables of first positions; no positions at all."""
    ids = torch.where(torch.arange(5000) % 3 == 0, torch.arange(5000) % 700, torch.full((5000,), 9))
    table, batch = batch_of(ids, rows=1024)
    x, labels = normal((50, 32), 3), torch.arange(50, device="cuda") * 99
    _, saved = table.item_loss(x, batch, labels)
    _, grad_out = table.item_loss_bwd(torch.full((50,), 0.02, device="cuda"), saved)
    first = torch.tensor([int((ids == v).nonzero()[0]) for v in ids.unique()], device="cuda")
    held = grad_out.any(1).nonzero().squeeze(1)
    assert len(held) > 200 and torch.isin(held, first).all()
    table, batch = batch_of(torch.empty(0, dtype=torch.int64))
    loss, saved = table.item_loss(x, batch, labels)
    dx, grad_out = table.item_loss_bwd(torch.ones(50, device="cuda"), saved)
    assert not loss.any() and not dx.any() and grad_out.shape == (0, 32)


def test_captured_and_replayed():
    """lookup's batch held, x and labels changed between replays; the eager program runs in between."""
    ids = torch.randint(0, 90, (700,), generator=torch.Generator().manual_seed(4))
    table, batch = batch_of(ids)
    x, labels = normal((80, 32), 3), torch.randint(-100, 700, (80,), generator=torch.Generator().manual_seed(5)).cuda()
    dloss = torch.full((80,), 1.0 / 80, device="cuda")

    def step():
        loss, saved = table.item_loss(x, batch, labels, scale=0.7)
        return loss, *table.item_loss_bwd(dloss, saved)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for k in range(4):
        x.copy_(normal((80, 32), 30 + k))
        labels.copy_(torch.randint(-100, 700, (80,), generator=torch.Generator().manual_seed(50 + k)))
        graph.replay()
        torch.cuda.synchronize()
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), k
