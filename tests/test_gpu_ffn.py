"""The gated feed-forward block against its 64-bit definition, element by element (bounds: tests/block_ref.py).  The
forward's h is checked against exact pre-activations, y against the product of the kernel's own h (what the backward
gets), and serving, whose h is not returned, with h's bound carried through the product."""
import pytest
import torch

from paper_2505_18654_amd import hstu, ops
from tests.block_ref import U, ffn_back, ffn_h, ffn_pre, half_step, normal, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def weights(d, f, seed=1, wide=0):
    return (normal((d, 2 * f), seed, d ** -0.5, 2 * f + wide if wide else None),
            normal((f, d), seed + 1, f ** -0.5, d + wide if wide else None))


def check_forward(T, d, f, residual=False, wide=0):
    print(f"[ffn] forward T={T} d={d} f={f} residual={residual} wide={wide}", flush=True)
    x = normal((T, d), 3, wide=d + wide if wide else None)
    w_in, w_out = weights(d, f, 1, wide)
    r = normal((T, d), 4, wide=d + wide if wide else None) if residual else None
    y, pre, h = ops.gated_ffn_fwd(x, w_in, w_out, residual=r, save=True)
    s = ops.gated_ffn_fwd(x, w_in, w_out, residual=r)
    torch.cuda.synchronize()
    want_pre, e_pre = ffn_pre(x, w_in)
    within("pre", pre, want_pre, half_step(pre) + e_pre)
    want_h, e_h = ffn_h(want_pre, e_pre)
    within("h", h, want_h, half_step(h) + e_h)
    W = w_out.double()

    def product(hh, e):
        v = hh @ W
        b = (f + 5) * U * (hh.abs() @ W.abs()) + (e @ W.abs() if e is not None else 0)
        if r is not None:
            v = v + r.double()
            b = b + 2 * U * (r.double().abs() + v.abs())
        return v, b

    want, b = product(h.double(), None)
    within("y", y, want, half_step(y) + b)
    want, b = product(want_h, e_h + half_step(want_h) + half_step(e_h))
    within("serving", s, want, half_step(s) + b)


# one token up to a few tiles; tokens around the 16-, 64- and 256-row edges; d and f that end inside a k step or tile
@pytest.mark.parametrize("T, d, f", [
    (1, 32, 32), (1, 512, 1408), (2, 96, 160), (5, 1024, 2816), (15, 64, 96), (16, 256, 704), (17, 256, 704),
    (31, 544, 416), (64, 128, 352), (65, 768, 2048), (255, 160, 288), (256, 64, 128), (257, 96, 1120), (700, 512, 1408),
    (2049, 256, 672), (9000, 128, 352), (20011, 64, 704), (33, 96, 2816), (127, 1024, 2848),
])
def test_forward(T, d, f):
    check_forward(T, d, f, residual=T % 2 == 1)


def test_forward_strided():
    check_forward(130, 96, 160, residual=True, wide=40)
    check_forward(3, 96, 160, residual=True, wide=24)


@pytest.mark.parametrize("T, d, f", [(1, 32, 32), (3, 544, 96), (64, 128, 352), (257, 256, 704), (1000, 96, 160),
                                     (5003, 512, 1408), (30011, 64, 704)])
def test_backward(T, d, f):
    print(f"[ffn] backward T={T} d={d} f={f}", flush=True)
    x, dy = normal((T, d), 5), normal((T, d), 6, 0.1)
    w_in, w_out = weights(d, f)
    _, pre, h = ops.gated_ffn_fwd(x, w_in, w_out, save=True)
    dx, dw_in, dw_out = ops.gated_ffn_bwd(dy, x, pre, h, w_in, w_out)
    torch.cuda.synchronize()
    for name, got, (want, b) in zip(("dx", "dw_in", "dw_out"), (dx, dw_in, dw_out),
                                    ffn_back(dy, x, pre, h, w_in, w_out).values()):
        within(name, got, want, half_step(got) + b)


def test_backward_strided():
    T, d, f = 300, 96, 160
    x, dy = normal((T, d), 5, wide=d + 40), normal((T, d), 6, wide=d + 8)
    w_in, w_out = weights(d, f, wide=16)
    _, pre, h = ops.gated_ffn_fwd(x, w_in, w_out, save=True)
    both = torch.cat([pre, h, torch.full((T, 8), 5.0, dtype=torch.bfloat16, device="cuda")], 1)
    pre, h = both[:, :2 * f], both[:, 2 * f:3 * f]               # column views of one buffer
    room = [torch.full((n, m), 7.0, dtype=torch.bfloat16, device="cuda") for n, m in ((T, d + 40), (d, 2 * f + 16), (f, d + 16))]
    grads = room[0][:, :d], room[1][:, :2 * f], room[2][:, :d]
    ops.gated_ffn_bwd(dy, x, pre, h, w_in, w_out, grads=grads)
    torch.cuda.synchronize()
    for name, got, (want, b) in zip(("dx", "dw_in", "dw_out"), grads, ffn_back(dy, x, pre, h, w_in, w_out).values()):
        within(name, got, want, half_step(got) + b)
    assert all(bool((t[:, g.shape[1]:] == 7).all()) for t, g in zip(room, grads))
    with pytest.raises(ValueError, match="row stride"):
        ops.gated_ffn_bwd(dy, x, pre, h, w_in, w_out, grads=(grads[0].contiguous(), grads[1], grads[2]))


def test_offsets_past_32_bits():
    """pre and its gradient hold 2.2e9 elements; the gradient of y is zero but for the last rows, so that the weights'
    gradients follow from them alone (zeros add no rounding)."""
    T, d, f, n = 1_000_003, 32, 1120, 400
    x, dy = normal((T, d), 41), torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    dy[-n:] = normal((n, d), 42, 0.1)
    w_in, w_out = weights(d, f)
    y, pre, h = ops.gated_ffn_fwd(x, w_in, w_out, save=True)
    s = ops.gated_ffn_fwd(x, w_in, w_out)
    dx, dw_in, dw_out = ops.gated_ffn_bwd(dy, x, pre, h, w_in, w_out)
    torch.cuda.synchronize()
    W = w_out.double()
    for rows in (slice(0, n), slice(T - n, T)):
        want_pre, e_pre = ffn_pre(x[rows], w_in)
        want_h, e_h = ffn_h(want_pre, e_pre)
        within("pre", pre[rows], want_pre, half_step(pre[rows]) + e_pre)
        within("h", h[rows], want_h, half_step(h[rows]) + e_h)
        within("y", y[rows], h[rows].double() @ W, half_step(y[rows]) + (f + 5) * U * (h[rows].double().abs() @ W.abs()))
        assert torch.equal(s[rows], y[rows])                 # (the same kernels, and h rounded alike)
    assert not dx[:-n].any()
    for name, got, (want, b) in zip(("dx", "dw_in", "dw_out"), (dx[-n:], dw_in, dw_out),
                                    ffn_back(dy[-n:], x[-n:], pre[-n:], h[-n:], w_in, w_out).values()):
        within(name, got, want, half_step(got) + b)


def test_gradients_against_differences():
    """(y(w + e v) - y(w - e v)) . dy / 2e of the 64-bit definition, whose gradients ffn_back states."""
    T, d, f = 7, 32, 64
    x, dy = normal((T, d), 8), normal((T, d), 9)
    w_in, w_out = weights(d, f, 10)
    pre, _ = ffn_pre(x, w_in)
    h, _ = ffn_h(pre, torch.zeros_like(pre))
    back = ffn_back(dy, x, pre, h, w_in, w_out)

    def y(x, w_in, w_out):
        p = x @ w_in
        return (p[:, :f] * torch.sigmoid(p[:, :f]) * p[:, f:]) @ w_out

    base = [t.double() for t in (x, w_in, w_out)]
    for i, name in enumerate(("dx", "dw_in", "dw_out")):
        v = torch.randn(base[i].shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64).cuda()
        up, down = ([t + s * 1e-5 * v if j == i else t for j, t in enumerate(base)] for s in (1, -1))
        diff = float(((y(*up) - y(*down)) * dy.double()).sum() / 2e-5)
        assert abs(diff - float((back[name][0] * v).sum())) <= 1e-6 * (1 + abs(diff)), name


def test_rows_do_not_depend_on_their_neighbours():
    """NaN in one token's row stays in that row, in the forward pass and in dx."""
    T, d, f = 300, 64, 96
    x, w = normal((T, d), 11), weights(d, f)
    y, pre, h = ops.gated_ffn_fwd(x, *w, save=True)
    s = ops.gated_ffn_fwd(x, *w)
    bad = x.clone()
    bad[123] = float("nan")
    y2, pre2, h2 = ops.gated_ffn_fwd(bad, *w, save=True)
    s2 = ops.gated_ffn_fwd(bad, *w)
    rest = torch.arange(T, device="cuda") != 123
    for a, b in ((y, y2), (pre, pre2), (h, h2), (s, s2)):
        assert torch.equal(a[rest], b[rest]) and bool(b[123].isnan().all())


def test_no_tokens():
    w_in, w_out = weights(64, 96)
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    y, pre, h = ops.gated_ffn_fwd(x, w_in, w_out, save=True)
    assert y.shape == (0, 64) and pre.shape == (0, 192) and h.shape == (0, 96)
    grads = x, torch.ones_like(w_in), torch.ones_like(w_out)
    ops.gated_ffn_bwd(x, x, pre, h, w_in, w_out, grads=grads)
    assert not grads[1].any() and not grads[2].any()


def test_residual_in_place_and_own_workspace():
    for T in (3, 200, 3000):
        x, r, w = normal((T, 96), 12), normal((T, 96), 13), weights(96, 160)
        want = ops.gated_ffn_fwd(x, *w, residual=r)
        ws = ops.gated_ffn_workspace(T, 96, 160)
        ws.fill_(255)                                    # NaN where a kernel read what it had not written
        out = r.clone()
        ops.gated_ffn_fwd(x, *w, residual=out, out=out, workspace=ws)
        assert torch.equal(out, want)
        _, pre, h = ops.gated_ffn_fwd(x, *w, save=True)
        a = ops.gated_ffn_bwd(r, x, pre, h, *w)
        ws = ops.gated_ffn_workspace(T, 96, 160, backward=True)
        ws.fill_(255)
        b = ops.gated_ffn_bwd(r, x, pre, h, *w, workspace=ws)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        with pytest.raises(hstu.MtgrError):
            ops.gated_ffn_bwd(r, x, pre, h, *w, workspace=ws[:256])


@pytest.mark.parametrize("T", [1, 40, 600])
def test_captured_and_replayed(T):
    d, f = 128, 352
    x, dy, w = normal((T, d), 14), normal((T, d), 15), weights(d, f)
    out = {}

    def step():
        out["s"] = ops.gated_ffn_fwd(x, *w, residual=x)
        y, pre, h = ops.gated_ffn_fwd(x, *w, save=True)
        out["y"] = y
        out["dx"], out["dw_in"], out["dw_out"] = ops.gated_ffn_bwd(dy, x, pre, h, *w)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    held = dict(out)
    for k in range(3):
        x.copy_(normal((T, d), 20 + k))
        graph.replay()
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        for n, v in out.items():
            assert torch.equal(v, held[n]), (n, k)


def test_refusals():
    x, (w_in, w_out) = normal((4, 64), 1), weights(64, 96)
    for bad in (lambda: ops.gated_ffn_fwd(x, w_in[:, :-32], w_out), lambda: ops.gated_ffn_fwd(x, w_in, w_out.t()),
                lambda: ops.gated_ffn_fwd(x.float(), w_in, w_out), lambda: ops.gated_ffn_fwd(x, w_in, w_out, residual=x[:2]),
                lambda: ops.gated_ffn_fwd(x.t().contiguous().t(), w_in, w_out), lambda: ops.gated_ffn_fwd(x.cpu(), w_in, w_out),
                lambda: ops.gated_ffn_fwd(x[:1].expand(4, 64), w_in, w_out)):
        with pytest.raises(ValueError):
            bad()
