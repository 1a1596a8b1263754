"""The softmax loss on each of its kernels, against its 64-bit definition: the sizes of tests/block_shapes.py, whose
kernels tests/test_block_plans_cpu.py asserts.  Bounds: tests/block_ref.py.

Statistics carried over class tiles are kept relative to the first tile's maximum of a lane (ref), up to a sum of 2^100,
106 with what a lane adds on top: beside the bounds of block_ref, the difference z - ref and the two of the joins (up
to 106 in units of log 2) are rounded, 106 ln 2 U each, and the logarithm of a sum of up to 2^106 by 2 U of its 106:
CARRY = (3 + 2) 106 ln 2 U."""
import math

import pytest
import torch

from paper_2505_18654_amd import ops
from tests import block_shapes as S
from tests.block_ref import U, half_step, normal, softmax_loss, within
from tests.test_gpu_softmax_loss import check

pytestmark = pytest.mark.gpu
CARRY = 5 * 106 * math.log(2) * U


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


def statistics(x, w, t, b, scale):
    """loss and lse of rows that all have a label, and their bounds, in 64 bits and some thousand rows at a time."""
    parts = [softmax_loss(x[i:i + 4000], w, t[i:i + 4000], b, scale) for i in range(0, x.shape[0], 4000)]
    return [{k: torch.cat([p[j][k] for p in parts]) for k in ("loss", "lse")} for j in (0, 1)]


def check_statistics(name, x, w, t, b, scale=0.9):
    loss, lse = ops.softmax_loss_fwd(x, w, t, bias=b, scale=scale)
    torch.cuda.synchronize()
    want, e = statistics(x, w, t, b, scale)
    within(f"{name}: lse", lse, want["lse"], e["lse"] + CARRY)
    within(f"{name}: loss", loss, want["loss"], e["loss"] + CARRY)
    return loss, lse


def steps_of(shape):
    """Which of an item's class tiles each class lies in (0: the first one)."""
    c = torch.arange(shape[1], device="cuda")
    run = S.CARRIED_RUN[shape]
    if shape == S.CARRIED_REGISTERS:
        return c // 64 % run
    blocks = -(-shape[1] // 256)
    return c // 256 // -(-blocks // run)


@pytest.mark.parametrize("shape", S.CARRIED_RUN)
def test_first_tiles_out_or_far_below_the_later_ones(shape):
    N, V, d = shape
    print(f"[loss] carried statistics of {shape}", flush=True)
    x, w, t, b, _ = make(N, V, d, N)
    step = steps_of(shape)
    assert int(step.max()) == S.CARRIED_RUN[shape] - 1
    live = (step > 0).nonzero().squeeze(1)
    t_live = live[t % len(live)]
    # the first tile of every item out; all but the last one out
    check_statistics("first out", x, w, t_live, b.masked_fill(step == 0, float("-inf")))
    last = (step == int(step.max())).nonzero().squeeze(1)
    check_statistics("last live", x, w, last[t % len(last)], b.masked_fill(step < int(step.max()), float("-inf")))
    # from the first tile's maximum: below a sum of 2^100 (kept), above it (the reference moves), past the float range
    for nats in (40.0, 66.0, 68.0, 71.0, 90.0, 300.0, 20000.0):
        check_statistics(f"first {nats} below", x, w, t_live, b - nats * (step == 0))
    # every tile above the one before it, and below
    for nats in (30.0, 60.0, 80.0):
        check_statistics(f"rising {nats}", x, w, t_live, b + nats * step)
        check_statistics(f"falling {nats}", x, w, t, b - nats * step)


@pytest.mark.parametrize("shape", S.CARRIED_RUN)
def test_large_logits_over_carried_tiles(shape):
    """Logits of hundreds: each lane's maximum of its first tile is far from the later ones, up and down."""
    N, V, d = shape
    x, w, t, b, _ = make(N, V, d, N, spread=60.0)
    check_statistics("large", x, w, t, b, scale=3.0)
    best = torch.cat([(x[i:i + 4000].float() @ w.float().t()).argmax(1) for i in range(0, N, 4000)])
    check_statistics("confident", x, w, best, None, scale=3.0)
    check_statistics("negative scale", x, w, t, b, scale=-0.5)


@pytest.mark.parametrize("shape", S.CARRIED_RUN)
def test_no_class_left_and_lowest_numbers(shape):
    N, V, d = shape
    x, w, t, b, dloss = make(N, V, d, N)
    none = torch.full_like(b, float("-inf"))
    loss, lse = ops.softmax_loss_fwd(x, w, t, bias=none)
    assert not loss.any() and bool((lse == float("-inf")).all())
    assert not any(v.any() for v in ops.softmax_loss_bwd(dloss, x, w, t, lse, bias=none))
    out = torch.arange(V, device="cuda") % 3 == 1
    t = torch.where(out[t], t - 1, t)
    for lowest in (torch.finfo(torch.float32).min, torch.finfo(torch.bfloat16).min):
        got, want = (ops.softmax_loss_fwd(x, w, t, bias=b.masked_fill(out, v)) for v in (lowest, float("-inf")))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    one = none.clone()
    one[V - 1] = 0.25                                    # a single class left, in the last tile: no loss
    check_statistics("one left", x, w, torch.full_like(t, V - 1), one)


@pytest.mark.parametrize("shape", S.CARRIED_RUN)
def test_one_infinite_gradient_stays_in_its_row(shape):
    N, V, d = shape
    x, w, t, b, dloss = make(N, V, d, N, bias=False)
    _, lse = ops.softmax_loss_fwd(x, w, t)
    want = ops.softmax_loss_bwd(dloss, x, w, t, lse)[0]
    bad = dloss.clone()
    bad[777] = float("inf")
    got = ops.softmax_loss_bwd(bad, x, w, t, lse)[0]
    rest = torch.arange(N, device="cuda") != 777
    # (the largest finite gradient is the same with and without row 777, whose own is not the largest)
    assert float(dloss[777].abs()) < float(dloss.abs().max())
    assert not torch.isfinite(got[777]).all() and torch.equal(got[rest], want[rest])


@pytest.mark.parametrize("shape", S.CARRIED_RUN)
def test_few_labels_of_many_rows(shape):
    """The grids are laid out for all rows; unlabelled rows hold NaN; 0, 1, 255, 256 and 257 labels."""
    N, V, d = shape
    for labels in (0, 1, 255, 256, 257):
        print(f"[loss] {shape}: {labels} labels", flush=True)
        x, w, t, b, dloss = make(N, V, d, max(labels, 1), seed=labels)
        if labels == 0:
            t.fill_(-1)
        x[t < 0] = float("nan")
        loss, lse = ops.softmax_loss_fwd(x, w, t, bias=b, scale=0.9)
        dx, dw, db = ops.softmax_loss_bwd(dloss, x, w, t, lse, bias=b, scale=0.9)
        on = t >= 0
        assert not loss[~on].any() and not lse[~on].any() and not dx[~on].any()
        if labels == 0:
            assert not dw.any() and not db.any()
            continue
        want, e = softmax_loss(x[on], w, t[on], b, 0.9, dloss[on])
        for name, got in (("loss", loss[on]), ("lse", lse[on]), ("dx", dx[on]), ("dw", dw), ("dbias", db)):
            within(name, got, want[name], e[name] + (half_step(got) if name in ("dx", "dw") else 0))
