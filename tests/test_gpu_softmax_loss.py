"""Softmax loss over a class set against its 64-bit definition, with the bounds that tests/block_ref.py derives."""
import pytest
import torch

from paper_2505_18654_amd import hstu, ops
from tests.block_ref import half_step, normal, softmax_loss, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def make(N, V, d, share=1.0, bias=False, seed=1, wide=0, bits=64, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x, w = normal((N, d), seed, wide=d + wide if wide else None), normal((V, d), seed + 1, spread * d ** -0.5,
                                                                       wide=d + wide if wide else None)
    t = torch.randint(0, V, (N,), generator=g)
    t[torch.rand(N, generator=g) >= share] = -1
    if N > 4 and 0 < share < 1:
        t[1], t[3] = V, -100                                 # both outside: no label either
    b = (torch.randn(V, generator=g) * 0.7).cuda() if bias else None
    dloss = (torch.randn(N, generator=g) / max(N, 1)).cuda()
    return x, w, t.to(torch.int64 if bits == 64 else torch.int32).cuda(), b, dloss


def check(x, w, t, b, dloss, scale=0.9):
    loss, lse = ops.softmax_loss_fwd(x, w, t, bias=b, scale=scale)
    dx, dw, db = ops.softmax_loss_bwd(dloss, x, w, t, lse, bias=b, scale=scale)
    torch.cuda.synchronize()
    want, e = softmax_loss(x, w, t, b, scale, dloss)
    within("lse", lse, want["lse"], e["lse"])
    within("loss", loss, want["loss"], e["loss"])
    within("dx", dx, want["dx"], half_step(dx) + e["dx"])
    within("dw", dw, want["dw"], half_step(dw) + e["dw"])
    if b is not None:
        within("dbias", db, want["dbias"], e["dbias"])
    off = (t < 0) | (t >= w.shape[0])
    assert not loss[off].any() and not lse[off].any() and not dx[off].any()
    return loss, lse, dx, dw, db


@pytest.mark.parametrize("N, V, d, share, bias, bits", [
    (1, 1, 32, 1.0, False, 64), (1, 2, 32, 1.0, True, 32), (1, 1000, 128, 1.0, False, 64), (3, 255, 64, 1.0, True, 64),
    (16, 256, 96, 1.0, False, 64), (17, 257, 544, 1.0, True, 32), (255, 33, 64, 0.5, True, 64), (256, 4099, 64, 1.0, False, 64),
    (257, 700, 160, 0.3, True, 32), (1000, 5003, 256, 0.6, True, 64), (5000, 301, 32, 0.2, True, 64),
    (2100, 1999, 1056, 0.9, False, 64), (40, 20011, 128, 1.0, True, 64), (300, 64, 2048, 0.5, True, 32),
    (2500, 20000, 256, 0.9, True, 64), (3001, 16001, 224, 0.7, False, 32), (5000, 9999, 160, 0.6, True, 64),
    (4000, 12345, 96, 1.0, True, 64), (9000, 7001, 32, 0.95, True, 64), (300, 70001, 256, 1.0, True, 64),
    (8001, 9999, 128, 0.9, False, 64), (7000, 30011, 288, 1.0, True, 64),
])
def test_loss_and_gradients(N, V, d, share, bias, bits):
    print(f"[loss] N={N} V={V} d={d} share={share} bias={bias} int{bits}", flush=True)
    check(*make(N, V, d, share, bias, bits=bits))


def test_strided_and_neighbouring_columns():
    x, w, t, b, dloss = make(300, 513, 96, 0.5, True, wide=40)
    dx, dw = (torch.full((n, 136), 7.0, dtype=torch.bfloat16, device="cuda") for n in (300, 513))
    _, lse = ops.softmax_loss_fwd(x, w, t, bias=b)
    ops.softmax_loss_bwd(dloss, x, w, t, lse, bias=b, grads=(dx[:, :96], dw[:, :96], None))
    torch.cuda.synchronize()
    want, e = softmax_loss(x, w, t, b, 1.0, dloss)
    within("dx", dx[:, :96], want["dx"], half_step(dx[:, :96]) + e["dx"])
    within("dw", dw[:, :96], want["dw"], half_step(dw[:, :96]) + e["dw"])
    assert bool((dx[:, 96:] == 7).all()) and bool((dw[:, 96:] == 7).all())


@pytest.mark.parametrize("share", [0.0, 1e-9])
def test_no_label_at_all(share):
    x, w, t, b, dloss = make(600, 300, 64, share, True)
    x.fill_(float("nan"))
    loss, lse = ops.softmax_loss_fwd(x, w, t, bias=b)
    dx, dw, db = ops.softmax_loss_bwd(dloss, x, w, t, lse, bias=b)
    for v in (loss, lse, dx, dw, db):
        assert not v.any()


def test_rows_without_a_label_may_hold_anything():
    x, w, t, b, dloss = make(700, 400, 64, 0.4, True)
    a = check(x, w, t, b, dloss)
    off = (t < 0) | (t >= 400)
    x, dloss = x.clone(), dloss.clone()
    x[off] = float("nan")
    dloss[off] = float("inf")
    loss, lse = ops.softmax_loss_fwd(x, w, t, bias=b, scale=0.9)
    again = (loss, lse, *ops.softmax_loss_bwd(dloss, x, w, t, lse, bias=b, scale=0.9))
    assert all(torch.equal(p, q) for p, q in zip(a, again))


def test_classes_taken_out():
    """bias -inf: the same as without those classes; a label among them: loss +inf; no class left: 0 and no gradient."""
    x, w, t, b, dloss = make(300, 600, 64, 1.0, True)
    out = torch.rand(600, generator=torch.Generator().manual_seed(9)).cuda() < 0.5
    out[256:512] = True                                      # a whole tile of classes
    left = (~out).nonzero().squeeze(1)
    t = left[t % len(left)]
    b = torch.where(out, torch.full_like(b, float("-inf")), b)
    loss, lse, dx, dw, db = check(x, w, t, b, dloss)
    assert not dw[out].any() and not db[out].any()
    small = torch.searchsorted(left, t)
    l2, _ = ops.softmax_loss_fwd(x, w[left].contiguous(), small, bias=b[left].contiguous(), scale=0.9)
    assert float((loss - l2).abs().max()) < 1e-5
    t2 = t.clone()
    t2[5] = int(out.nonzero()[0])
    l3, _ = ops.softmax_loss_fwd(x, w, t2, bias=b, scale=0.9)
    keep = torch.arange(300, device="cuda") != 5
    assert l3[5] == float("inf") and torch.equal(l3[keep], loss[keep])
    none = torch.full_like(b, float("-inf"))
    l4, s4 = ops.softmax_loss_fwd(x, w, t, bias=none)
    assert not l4.any() and bool((s4 == float("-inf")).all())
    assert not any(v.any() for v in ops.softmax_loss_bwd(dloss, x, w, t, s4, bias=none))


def test_lowest_numbers_take_classes_out():
    """A bias below -2.36e38 is -inf in units of log 2; one that a mask of 16-bit logits would use is a number."""
    x, w, t, b, dloss = make(300, 600, 64, 1.0, True)
    out = torch.arange(600, device="cuda") % 3 == 1
    t = torch.where(out[t], t - 1, t)
    for lowest in (torch.finfo(torch.float32).min, torch.finfo(torch.bfloat16).min):
        got, want = (ops.softmax_loss_fwd(x, w, t, bias=b.masked_fill(out, v)) for v in (lowest, float("-inf")))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    half = torch.full_like(b, -65504.0)                      # all classes: the softmax of what is left of them
    check(x, w, t, half, dloss)


def test_one_infinite_gradient_stays_in_its_row():
    x, w, t, b, dloss = make(300, 200, 64, 1.0, False)
    _, lse = ops.softmax_loss_fwd(x, w, t)
    want, _, _ = ops.softmax_loss_bwd(dloss, x, w, t, lse)
    bad = dloss.clone()
    bad[7] = float("inf")
    got, _, _ = ops.softmax_loss_bwd(bad, x, w, t, lse)
    rest = torch.arange(300, device="cuda") != 7
    assert not torch.isfinite(got[7]).all()
    # (both are within a bf16 rounding of each product's operand; dz is kept relative to the largest gradient)
    assert torch.isfinite(got[rest]).all()
    assert float((got[rest].double() - want[rest].double()).norm() / want[rest].double().norm()) < 2.0 ** -7


def test_large_logits():
    """Logits of a thousand and more: the maximum is taken out first; confident rows have losses near 0."""
    x, w, t, b, dloss = make(200, 500, 128, 1.0, False, spread=60.0)
    check(x, w, t, b, dloss, scale=3.0)
    z = x.float() @ w.float().t()
    check(x, w, z.argmax(1), b, dloss, scale=3.0)
    check(x, w, t, b, dloss, scale=-0.5)
    check(x, w, t, b, dloss, scale=0.0)


def test_same_label_everywhere_and_repeats_bit_for_bit():
    x, w, t, b, dloss = make(3000, 900, 96, 0.7, True)
    t = torch.where(t >= 0, torch.full_like(t, 13), t)
    a = check(x, w, t, b, dloss)
    c = check(x, w, t, b, dloss)
    assert all(torch.equal(p, q) for p, q in zip(a, c))


def test_pieces():
    """Long batches, whose workspace bounds force several pieces of classes, forward and backward: few rows have a
    label, so that the 64-bit reference stays small."""
    x, w, t, b, dloss = make(240000, 18000, 32, 0.004, True, seed=31)
    check(x, w, t, b, dloss)


def test_more_classes_than_a_piece_may_have():
    """2^22 classes are the most of a piece of the backward, whatever the rows."""
    x, w, t, b, dloss = make(3, (1 << 22) + 5000, 32, 1.0, True, seed=33)
    t[0], t[1] = w.shape[0] - 1, 1 << 22
    check(x, w, t, b, dloss)


def test_offsets_past_32_bits():
    """2.2e9 elements of x, then of w: labels among the last rows (and the first ones), then among the last classes."""
    n, d = 1_100_003, 2048
    few, w, t, b, dloss = make(40, 300, d, 1.0, True, seed=35)
    x = torch.full((n, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    at = torch.cat([torch.arange(4), torch.arange(n - 36, n)]).cuda()
    x[at] = few
    labels, g = torch.full((n,), -1, device="cuda"), torch.ones(n, device="cuda")
    labels[at], g[at] = t, dloss
    loss, lse = ops.softmax_loss_fwd(x, w, labels, bias=b, scale=0.9)
    dx, dw, db = ops.softmax_loss_bwd(g, x, w, labels, lse, bias=b, scale=0.9)
    want, e = softmax_loss(few, w, t, b, 0.9, dloss)
    for name, got in (("loss", loss[at]), ("lse", lse[at]), ("dx", dx[at]), ("dw", dw), ("dbias", db)):
        within(name, got, want[name], e[name] + (half_step(got) if name in ("dx", "dw") else 0))
    assert not dx[4:n - 36].any() and not loss[4:n - 36].any()
    del x, dx, labels, g
    w = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    w[-600:] = normal((600, d), 36, 2.0 * d ** -0.5)
    b = torch.full((n,), float("-inf"), device="cuda")
    b[-600:] = 0.5
    t = n - 1 - t
    loss, lse, dx, dw, db = check(few, w[-600:], t - (n - 600), b[-600:], dloss)
    loss2, lse2 = ops.softmax_loss_fwd(few, w, t, bias=b, scale=0.9)
    dx2, dw2, db2 = ops.softmax_loss_bwd(dloss, few, w, t, lse2, bias=b, scale=0.9)
    want, e = softmax_loss(few, w[-600:], t - (n - 600), b[-600:], 0.9, dloss)
    for name, got in (("loss", loss2), ("lse", lse2), ("dx", dx2), ("dw", dw2[-600:]), ("dbias", db2[-600:])):
        within(name, got, want[name], e[name] + (half_step(got) if name in ("dx", "dw") else 0))
    assert not dw2[:-600].any() and not db2[:-600].any()


def test_gradients_against_differences():
    """The 64-bit definition's gradients against differences of its losses."""
    x, w, t, b, dloss = make(9, 23, 32, 0.8, True)
    want, _ = softmax_loss(x, w, t, b, 0.7, dloss)
    for i, name in enumerate(("dx", "dw", "dbias")):
        base = [x.double(), w.double(), b.double()]
        v = torch.randn(base[i].shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64).cuda()
        f = []
        for s in (1e-5, -1e-5):
            a = [u + s * v if j == i else u for j, u in enumerate(base)]
            f.append(float((softmax_loss(a[0], a[1], t, a[2], 0.7)[0]["loss"] * dloss.double()).sum()))
        diff = (f[0] - f[1]) / 2e-5
        assert abs(diff - float((want[name] * v).sum())) <= 1e-7 * (1 + abs(diff)), name


def test_own_workspace_of_any_contents():
    x, w, t, b, dloss = make(500, 700, 64, 0.5, True)
    a = check(x, w, t, b, dloss)
    ws, wb = (ops.softmax_loss_workspace(500, 700, 64, backward=k) for k in (False, True))
    ws.fill_(255)
    wb.fill_(255)
    loss, lse = ops.softmax_loss_fwd(x, w, t, bias=b, scale=0.9, workspace=ws)
    again = (loss, lse, *ops.softmax_loss_bwd(dloss, x, w, t, lse, bias=b, scale=0.9, workspace=wb))
    assert all(torch.equal(p, q) for p, q in zip(a, again))
    with pytest.raises(hstu.MtgrError):
        ops.softmax_loss_fwd(x, w, t, bias=b, workspace=ws[:1024])


def test_captured_and_replayed_with_other_labels():
    """A captured step follows the labels of each replay, whose number the host never sees."""
    x, w, t, b, dloss = make(900, 800, 64, 0.5, True)
    out = {}

    def step():
        out["loss"], out["lse"] = ops.softmax_loss_fwd(x, w, t, bias=b)
        out["dx"], out["dw"], out["db"] = ops.softmax_loss_bwd(dloss, x, w, t, out["lse"], bias=b)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    held = dict(out)
    for k, share in enumerate((0.9, 0.0, 0.1, 1.0)):
        t.copy_(make(900, 800, 64, share, seed=50 + k)[2])
        graph.replay()
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        for n, v in out.items():
            assert torch.equal(v, held[n]), (n, k)


def test_no_rows():
    w = normal((5, 32), 1)
    x, t = torch.empty(0, 32, dtype=torch.bfloat16, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    b = torch.zeros(5, device="cuda")
    loss, lse = ops.softmax_loss_fwd(x, w, t, bias=b)
    assert loss.shape == lse.shape == (0,)
    dx, dw, db = ops.softmax_loss_bwd(loss, x, w, t, lse, bias=b, grads=(x, torch.ones_like(w), torch.ones_like(b)))
    assert not dw.any() and not db.any()


def test_refusals():
    x, w, t, b, dloss = make(6, 9, 32, 1.0, True)
    for bad in (lambda: ops.softmax_loss_fwd(x, w[:, :16], t), lambda: ops.softmax_loss_fwd(x, w, t.float()),
                lambda: ops.softmax_loss_fwd(x, w, t[:5]), lambda: ops.softmax_loss_fwd(x, w, t, bias=b[:8]),
                lambda: ops.softmax_loss_fwd(x, w, t, bias=b.double()), lambda: ops.softmax_loss_fwd(x.float(), w, t),
                lambda: ops.softmax_loss_fwd(x, w, t.cpu()), lambda: ops.softmax_loss_fwd(x, w.t().contiguous().t(), t),
                lambda: ops.softmax_loss_bwd(dloss.double(), x, w, t, dloss), lambda: ops.softmax_loss_bwd(dloss, x, w, t, dloss[:3])):
        with pytest.raises(ValueError):
            bad()
