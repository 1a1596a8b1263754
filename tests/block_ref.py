"""Plain 64-bit definitions of the feed-forward block, dropout and the softmax loss, on the CPU or the GPU, and the
helpers of their tests.  U: half a step of fp32; a product of K terms in fp32 is off by at most K U of the sum of
its terms' absolute values."""
import numpy as np
import torch

U = 2.0 ** -24
M32 = 0xFFFFFFFF


def half_step(x):
    """Largest error of storing x in bf16: half the spacing of bf16 numbers around |x| (2^(e - 9) for |x| in
    [2^(e - 1), 2^e))."""
    a = x.double().abs()
    _, e = torch.frexp(a)
    return torch.where(a > 0, torch.ldexp(torch.ones_like(a), (e - 9).to(torch.int32)), torch.zeros_like(a))


def normal(shape, seed, scale=1.0, wide=None):
    """Seeded bf16 matrix on the GPU; wide: as the first columns of a wider one."""
    g = torch.Generator().manual_seed(seed)
    full = (torch.randn((shape[0], wide or shape[1]), generator=g) * scale).bfloat16().cuda()
    return full[:, :shape[1]]


def within(name, got, want, bound):
    got, want = got.double(), want.double()
    assert torch.isfinite(got).all(), name
    ratio = float(((got - want).abs() / (bound + 1e-37)).max()) if got.numel() else 0.0
    print(f"[block] {name}: max error / bound = {ratio:.3f}", flush=True)
    assert ratio <= 1.0, (name, ratio)


# ------------------------------------------------------------------ gated feed-forward block

def silu(z):
    return z * torch.sigmoid(z)


def ffn_pre(x, w_in):
    """pre = x W_in in 64 bits, and the bound of its fp32 sums."""
    x, w = x.double(), w_in.double()
    return x @ w, (x.shape[1] + 4) * U * (x.abs() @ w.abs())


def ffn_h(pre, err):
    """h of exact pre-activations that are off by err, and h's bound before its rounding: |silu'| < 1.1, the
    hardware's exp2 and reciprocal within a few U of |z| + 1."""
    f = pre.shape[1] // 2
    g, u, eg, eu = pre[:, :f], pre[:, f:], err[:, :f], err[:, f:]
    h = silu(g) * u
    return h, 1.1 * eg * u.abs() + silu(g).abs() * eu + 1.1 * eg * eu + 16 * U * (g.abs() + 1) * h.abs()


def ffn_back(dy, x, pre, h, w_in, w_out):
    """dict of (gradient, bound) of the backward pass on the same bf16 inputs."""
    dy, x, pre, h, w_in, w_out = (t.double() for t in (dy, x, pre, h, w_in, w_out))
    f = h.shape[1]
    g, u = pre[:, :f], pre[:, f:]
    dh = dy @ w_out.t().contiguous()
    e_dh = (dy.shape[1] + 4) * U * (dy.abs() @ w_out.abs().t().contiguous())
    s = torch.sigmoid(g)
    sp = s * (1 + g * (1 - s))
    dpre = torch.cat([dh * u * sp, dh * g * s], 1)
    e = torch.cat([e_dh * (u * sp).abs() + 16 * U * (g.abs() + 1) * (dh * u).abs() * s * (1 + (g * (1 - s)).abs()),
                   e_dh * (g * s).abs() + 16 * U * (g.abs() + 1) * (dh * g * s).abs()], 1)
    e = e + half_step(dpre) + half_step(e)               # (the rounding of a value that is off by e)
    T = x.shape[0]
    dx = dpre @ w_in.t().contiguous()
    dw_in, dw_out = x.t().contiguous() @ dpre, h.t().contiguous() @ dy
    return {"dx": (dx, e @ w_in.abs().t().contiguous() + (2 * f + 4) * U * (dpre.abs() @ w_in.abs().t().contiguous())),
            "dw_in": (dw_in, x.abs().t().contiguous() @ e + (T + 70) * U * (x.abs().t().contiguous() @ dpre.abs())),
            "dw_out": (dw_out, (T + 70) * U * (h.abs().t().contiguous() @ dy.abs()))}


# ------------------------------------------------------------------ dropout

def philox_words(seed, step, site, n):
    """The first n words of Philox4x32 with 7 rounds, counters (i low, i high, site, step)."""
    q = np.arange((n + 3) // 4, dtype=np.uint64)
    m, s32 = np.uint64(M32), np.uint64(32)
    c = [q & m, q >> s32, np.full_like(q, site), np.full_like(q, step & M32)]
    k = [seed & M32, (seed >> 32) & M32]
    for _ in range(7):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s32) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> s32) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return np.stack(c, 1).reshape(-1)[:n]


def keep_mask(shape, p, seed, step, site):
    n = shape[0] * shape[1]
    return torch.from_numpy((philox_words(seed, step, site, n) >= np.uint64(int(p * 2.0 ** 32))).reshape(shape))


# ------------------------------------------------------------------ softmax loss

def softmax_loss(x, w, targets, bias=None, scale=1.0, dloss=None):
    """(values, bounds) of loss, lse and, with dloss, dx, dw, dbias: 64 bits, rows without a label 0.

    z is off by dz = |scale| (d + 6) U |x||w| + 4 U |z| (fp32 sums, then one fma in units of log 2); the sums of
    exponentials by (terms added one after another) U and the exponentials by 4 U and the difference's own rounding;
    the loss is a difference of two such numbers."""
    N, d = x.shape
    V = w.shape[0]
    on = (targets >= 0) & (targets < V)
    t = targets[on].long()
    X, W = x[on].double(), w.double()
    b = torch.zeros(V, dtype=torch.float64, device=x.device) if bias is None else bias.double()
    z = scale * (X @ W.t().contiguous()) + b
    zf = torch.where(torch.isfinite(z), z.abs(), torch.zeros_like(z))
    e_z = abs(scale) * (d + 6) * U * (X.abs() @ W.abs().t().contiguous()) + 4 * U * zf
    empty = torch.isinf(b).all()
    lse = torch.logsumexp(z, 1)
    seen = torch.isfinite(z)
    worst = torch.where(seen, e_z + 4 * U * (z - lse[:, None]).abs().nan_to_num(0, 0, 0), torch.zeros_like(e_z))
    p = torch.where(seen, (z - lse[:, None]).exp(), torch.zeros_like(z))
    terms = 16 + 2 + 8 * (V / 4096 + 10) + 20
    e_lse = (p * worst).sum(1) + (terms + 8) * U + 4 * U * lse.abs().nan_to_num(0, 0, 0)
    zt = z.gather(1, t[:, None]).squeeze(1)
    e_zt = e_z.gather(1, t[:, None]).squeeze(1)
    loss = lse - zt
    if empty:
        loss, e_lse, e_zt = torch.zeros_like(loss), torch.zeros_like(e_lse), torch.zeros_like(e_zt)

    def whole(v):
        out = torch.zeros((N,) + v.shape[1:], dtype=torch.float64, device=x.device)
        out[on] = v
        return out

    vals = {"loss": whole(loss), "lse": whole(lse)}
    errs = {"loss": whole(e_lse + e_zt + 4 * U * (lse.abs() + zt.abs()).nan_to_num(0, 0, 0)), "lse": whole(e_lse)}
    if dloss is None:
        return vals, errs
    g = dloss[on].double()
    q = p.clone()
    q[torch.arange(len(t), device=x.device), t] -= 1.0
    dz = q * g[:, None]
    # (the backward takes lse as the forward rounded it: off by e_lse + U |lse|)
    e_p = p * (worst + (e_lse + 4 * U * lse.abs().nan_to_num(0, 0, 0))[:, None] + 8 * U)
    e_dz = (e_p + 2 * U * q.abs()) * g.abs()[:, None]
    if empty:
        dz, e_dz = torch.zeros_like(dz), torch.zeros_like(e_dz)
    # The operand is dz / G, G = max |g|, rounded to bf16 and multiplied by G after the sums: off by half a step of
    # dz / G times G (up to twice half a step of dz itself, whose binade is another), and U of dz for the division.
    top = g.abs().max() if len(t) and bool((g != 0).any()) else 1.0
    e16 = e_dz + top * (half_step(dz / top) + half_step(e_dz / top)) + 2 * U * dz.abs()
    s = abs(scale)
    vals.update(dx=whole(scale * (dz @ W)), dw=scale * (dz.t().contiguous() @ X), dbias=dz.sum(0))
    errs.update(dx=whole(s * (e16 @ W.abs() + (V + 82) * U * (dz.abs() @ W.abs()))),
                dw=s * (e16.t().contiguous() @ X.abs() + (len(t) + 82) * U * (dz.abs().t().contiguous() @ X.abs())),
                dbias=e_dz.sum(0) + (len(t) + 24) * U * dz.abs().sum(0))
    return vals, errs
