"""The block's operators together, as a training step uses them: Group-LN, gated feed-forward block, dropout on the
residual branch, softmax loss, and the gradients back through all of them; and the embedding table's item loss.

Reference: the same step in 64 bits on the GPU, gradients by torch.autograd, the dropout mask from its plain
definition.  Bar: max |got - want| / rms(want) <= 2e-2 for tensors of bf16 chains (the bar of the encoder layer's tests:
each stage rounds once, 2^-9 relative, and a dozen independent roundings of that size stay below it)."""
import pytest
import torch

from paper_2505_18654_amd import ops
from paper_2505_18654_amd.embedding import DynamicEmbedding
from paper_2505_18654_amd.layer import FfnParams, ffn_bwd, ffn_fwd
from tests.block_ref import keep_mask, normal

pytestmark = pytest.mark.gpu
BAR = 2e-2


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def close(name, got, want, bar=BAR):
    want = want.double()
    rms = float(want.square().mean().sqrt())
    err = float((got.double() - want).abs().max())
    # (a value far above the rms is stored with half a step of its own size)
    slack = float(want.abs().max()) * 2.0 ** -8
    print(f"[block step] {name}: {err / max(rms, 1e-30):.2e} of the rms", flush=True)
    assert err <= bar * rms + slack, (name, err, rms)


def params(d, f, G=4):
    g = torch.Generator().manual_seed(3)
    return FfnParams((1 + 0.1 * torch.randn(G, d, generator=g)).cuda(), (0.1 * torch.randn(G, d, generator=g)).cuda(),
                     normal((d, 2 * f), 4, d ** -0.5), normal((f, d), 5, f ** -0.5))


def jagged(T):
    lens = [T // 3, 0, T - T // 3]
    off = [0, lens[0], lens[0], T]
    seg = [i % 4 for i in range(T)]
    return ops.Jagged.from_host(off, seg, [0] * T)


def reference(x, jag, P, w, t, bias, dloss, p, mask, scale):
    leaves = [v.double().clone().requires_grad_() for v in (x, P.gamma, P.beta, P.w_in, P.w_out, w, bias)]
    X, ga, be, wi, wo, W, b = leaves
    seg = jag.seg.long()
    zc = X - X.mean(1, keepdim=True)
    xt = ga[seg] * zc * (zc.square().mean(1, keepdim=True) + 1e-5).rsqrt() + be[seg]
    f = wo.shape[0]
    pre = xt @ wi
    y = (torch.nn.functional.silu(pre[:, :f]) * pre[:, f:]) @ wo
    out = X + torch.where(mask, y / (1 - p), torch.zeros_like(y))
    z = scale * (out @ W.t()) + b
    on = t >= 0
    loss = torch.zeros(len(t), dtype=torch.float64, device="cuda")
    loss[on] = torch.logsumexp(z[on], 1) - z[on].gather(1, t[on, None]).squeeze(1)
    (loss * dloss.double()).sum().backward()
    return out.detach(), loss.detach(), [v.grad for v in leaves]


@pytest.mark.parametrize("T, d, f, V, p", [(5, 32, 64, 7, 0.3), (333, 64, 96, 300, 0.0), (1500, 128, 352, 1001, 0.25)])
def test_training_step(T, d, f, V, p):
    jag, P = jagged(T), params(d, f)
    x, w = normal((T, d), 1), normal((V, d), 2, 2.0 * d ** -0.5)
    g = torch.Generator().manual_seed(9)
    t = torch.randint(0, V, (T,), generator=g)
    t[::3] = -1
    t = t.cuda()
    bias = (0.5 * torch.randn(V, generator=g)).cuda()
    dloss = torch.full((T,), 1.0 / T, device="cuda")
    rng = torch.tensor([1234, 5], dtype=torch.int64, device="cuda")
    out, ctx = ffn_fwd(x, jag, P, rng, p, site=2)
    loss, lse = ops.softmax_loss_fwd(out, w, t, bias=bias, scale=0.8)
    dout, dw, db = ops.softmax_loss_bwd(dloss, out, w, t, lse, bias=bias, scale=0.8)
    grads = ffn_bwd(dout, ctx, jag, P, rng, p, site=2)
    served, none = ffn_fwd(x, jag, P, rng, p, site=2, save=False)
    torch.cuda.synchronize()
    assert none is None
    mask = keep_mask((T, d), p, 1234, 5, 2).cuda()
    r_out, r_loss, (dx, dga, dbe, dwi, dwo, dW, dB) = reference(x, jag, P, w, t, bias, dloss, p, mask, 0.8)
    close("out", out, r_out)
    close("served", served, r_out)
    close("loss", loss, r_loss)
    for n, got, want in (("dw", dw, dW), ("dbias", db, dB), ("dx", grads["x"], dx), ("dw_in", grads["w_in"], dwi),
                         ("dw_out", grads["w_out"], dwo), ("dgamma", grads["gamma"], dga), ("dbeta", grads["beta"], dbe)):
        close(n, got, want)


def test_block_on_strided_rows():
    T, d, f = 200, 64, 96
    jag, P = jagged(T), params(d, f)
    x, dx_out = normal((T, d), 1), normal((T, d), 2)
    wide = torch.zeros(T, d + 32, dtype=torch.bfloat16, device="cuda")
    wide[:, :d] = x
    rng = torch.tensor([1, 2], dtype=torch.int64, device="cuda")
    a, ca = ffn_fwd(x, jag, P, rng, 0.1)
    b, cb = ffn_fwd(wide[:, :d], jag, P, rng, 0.1)
    assert torch.equal(a, b)
    ga, gb = ffn_bwd(dx_out, ca, jag, P, rng, 0.1), ffn_bwd(dx_out, cb, jag, P, rng, 0.1)
    for n in ("w_in", "w_out", "gamma", "beta"):
        assert torch.equal(ga[n], gb[n]), n
    close("dx in two passes", gb["x"], ga["x"])


def test_captured_training_steps_follow_the_eager_ones():
    T, d, f, V, p = 600, 64, 96, 500, 0.2
    jag, P = jagged(T), params(d, f)
    x, w, t = normal((T, d), 1), normal((V, d), 2, 0.2), torch.randint(-3, V, (T,), generator=torch.Generator().manual_seed(1)).cuda()
    dloss = torch.full((T,), 1.0 / T, device="cuda")
    rng = torch.tensor([7, 0], dtype=torch.int64, device="cuda")

    def step():
        out, ctx = ffn_fwd(x, jag, P, rng, p)
        loss, lse = ops.softmax_loss_fwd(out, w, t)
        dout, dw, _ = ops.softmax_loss_bwd(dloss, out, w, t, lse)
        g = ffn_bwd(dout, ctx, jag, P, rng, p)
        rng[1] += 1
        return [out, loss, dw] + [g[n] for n in sorted(g)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for k in range(3):
        rng[1] = 10 + k
        graph.replay()
        torch.cuda.synchronize()
        assert int(rng[1]) == 11 + k
        rng[1] = 10 + k
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), k


def test_two_streams_at_once():
    """Two steps on two streams, each with its own workspaces, give what each gives alone."""
    sets = []
    for k in range(2):
        x, w = normal((700, 64), 10 + k), normal((900, 64), 20 + k, 0.3)
        t = torch.randint(0, 900, (700,), generator=torch.Generator().manual_seed(k)).cuda()
        sets.append((x, w, t, torch.full((700,), 0.01, device="cuda"), normal((64, 192), 30 + k, 0.1), normal((96, 64), 40 + k, 0.1)))

    def run(s):
        x, w, t, dl, wi, wo = s
        y, pre, h = ops.gated_ffn_fwd(x, wi, wo, save=True)
        loss, lse = ops.softmax_loss_fwd(y, w, t)
        dy, dw, _ = ops.softmax_loss_bwd(dl, y, w, t, lse)
        return [loss, dw, *ops.gated_ffn_bwd(dy, x, pre, h, wi, wo)]

    want = [run(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for s, st in zip(sets, streams):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            got.append([run(s) for _ in range(3)][-1])
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_item_loss_of_the_embedding_table():
    table = DynamicEmbedding(row_capacity=256, dim=32)
    g = torch.Generator().manual_seed(5)
    ids = torch.randint(0, 60, (150,), generator=g)
    _, batch = table.lookup(ids.cuda(), now=1)
    table.values.copy_((0.3 * torch.randn(256, 32, generator=g)).bfloat16())
    before = table.values.clone()
    x = normal((40, 32), 6)
    labels = torch.randint(0, 150, (40,), generator=g)
    labels[::4], labels[1] = -1, 150
    dloss = torch.full((40,), 0.05, device="cuda")
    loss, saved = table.item_loss(x, batch, labels.cuda(), scale=0.7)
    dx, grad_out = table.item_loss_bwd(dloss, saved)
    table.sgd(batch, grad_out, lr=1.0)
    torch.cuda.synchronize()
    uniq, inv, n = torch.unique(ids, return_inverse=True, return_counts=True)
    rows = table.lookup(uniq.cuda(), now=2, insert=False, gather=False)[1]
    at = rows.rows.long()[rows.inverse.long()[:len(uniq)]]              # value row of each distinct ID
    W = before[at].double().requires_grad_()
    X = x.double().requires_grad_()
    z = 0.7 * (X @ W.t()) - torch.log(n.double() / 150).cuda()
    on = (labels >= 0) & (labels < 150)
    want = torch.zeros(40, dtype=torch.float64, device="cuda")
    zt = z[on.cuda()].gather(1, inv[labels[on]].cuda()[:, None]).squeeze(1)
    want[on.cuda()] = torch.logsumexp(z[on.cuda()], 1) - zt
    (want * 0.05).sum().backward()
    close("item loss", loss, want.detach())
    close("item dx", dx, X.grad)
    new = table.values[at].double()
    step = before[at].double() - new
    # (the update is rounded into values of up to 1.2: half a step of 2^-9 of them)
    assert float((step - W.grad).abs().max()) <= BAR * float(W.grad.abs().max()) + 2.0 ** -8 * float(new.abs().max())
    none, _ = table.item_loss(x, batch, torch.full((40,), -1, device="cuda"))
    assert not none.any()
