"""The operators of include/mtgr_block.h at the ends of their documented ranges, against 64-bit definitions."""
import pytest
import torch

from paper_2505_18654_amd import ops
from paper_2505_18654_amd.layer import FfnParams, ffn_bwd, ffn_fwd
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


@pytest.mark.parametrize("N, V, d", [(300, 500, 64), (3001, 16001, 224), (7000, 30011, 288)])
@pytest.mark.parametrize("a, b", [(80, 60), (-80, -60)])
def test_loss_gradients_when_scale_times_dloss_leaves_the_float_range(N, V, d, a, b):
    """x and w times 2^(-a/2), scale times 2^a, dloss times 2^b: the logits stay, and every step of the gradients but
    the product scale x dloss (2^140 or 2^-140) is a normal number, so that the gradients are the first ones times
    2^(a/2 + b), bit for bit."""
    print(f"[limits] loss {N} x {V} x {d}, scale 2^{a}, dloss 2^{b}", flush=True)
    g = torch.Generator().manual_seed(3)
    x, w = normal((N, d), 1), normal((V, d), 2, 2.0 * d ** -0.5)
    t = torch.randint(-1, V, (N,), generator=g).cuda()
    dloss = torch.rand(N, generator=g).cuda() + 0.5

    def step(x, w, scale, dloss):
        loss, lse = ops.softmax_loss_fwd(x, w, t, scale=scale)
        return loss, lse, *ops.softmax_loss_bwd(dloss, x, w, t, lse, scale=scale)[:2]

    base = step(x, w, 0.75, dloss)
    half = 2.0 ** (-a // 2)
    got = step(x * half, w * half, 0.75 * 2.0 ** a, dloss * 2.0 ** b)
    assert torch.equal(got[0], base[0]) and torch.equal(got[1], base[1])
    for name, p, q in zip(("dx", "dw"), got[2:], base[2:]):
        # (values whose scaled form is no normal bf16 number are left out)
        q = q.double() * 2.0 ** (a // 2 + b)
        on = (q == 0) | ((q.abs() > 2.0 ** -120) & (q.abs() < 2.0 ** 126))
        assert on.float().mean() > 0.9, name
        assert torch.equal(p.double()[on], q[on]), name


@pytest.mark.parametrize("p", [0.0, 0.4])
def test_layers_feed_forward_block_without_tokens(p):
    """A batch without a token: empty outputs, gradients of zero for every parameter."""
    d, f = 64, 96
    P = FfnParams(torch.ones(4, d, device="cuda"), torch.zeros(4, d, device="cuda"), normal((d, 2 * f), 1), normal((f, d), 2))
    jag = ops.Jagged.from_host([0, 0, 0], [], [])
    x = torch.empty(0, d, dtype=torch.bfloat16, device="cuda")
    rng = torch.zeros(2, dtype=torch.int64, device="cuda")
    out, ctx = ffn_fwd(x, jag, P, rng, p)
    g = ffn_bwd(out, ctx, jag, P, rng, p)
    torch.cuda.synchronize()
    assert out.shape == g["x"].shape == (0, d)
    assert not any(g[n].any() for n in ("w_in", "w_out", "gamma", "beta"))
