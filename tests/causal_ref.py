"""Plain 64-bit definitions of rotary positions and causal attention, with elementwise bounds of what the kernels may be off
by, derived from their roundings.  U: half a step of fp32, B16: half a step of bf16 (relative); a sum of K products in fp32
is off by at most K U of the sum of their absolute values."""
import math

import torch

from tests.block_ref import U, half_step

B16 = 2.0 ** -8


def heads(shape, seed, scale=1.0, wide=0, dtype=torch.bfloat16, device="cuda"):
    """Seeded [T, heads, dh]; wide: as the first heads of a row with so many more."""
    g = torch.Generator().manual_seed(seed)
    T, H, dh = shape
    return (torch.randn((T, H + wide, dh), generator=g) * scale).to(dtype).to(device)[:, :H]


def offsets_of(lengths, device="cuda"):
    o = torch.zeros(len(lengths) + 1, dtype=torch.int32)
    o[1:] = torch.cumsum(torch.tensor(lengths, dtype=torch.int64), 0)
    return o.to(device)


def rotate(x, freqs, positions, amplitude=1.0, layout="half"):
    """x [T, heads, dh] rotated, and the bound of the kernel before its final rounding: sine and cosine off by 6 U (the
    argument's 3 roundings times pi / 4, the series' last one, the amplitude's), their arguments by 4 roundings of 64 bits of
    p f on either side, and 3 U for products and sum."""
    r = 2 * len(freqs)
    x = x.double()
    angle = positions.double()[:, None] * freqs.double()
    c, s = (amplitude * angle.cos())[:, None], (amplitude * angle.sin())[:, None]
    off = (abs(amplitude) * (9 * U + 8 * 2.0 ** -53 * angle.abs()))[:, None]
    if layout == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
    u, v, e = a * c - b * s, a * s + b * c, (a.abs() + b.abs()) * off
    want, bound = x.clone(), torch.zeros_like(x)
    if layout == "half":
        want[..., :r // 2], want[..., r // 2:r] = u, v
        bound[..., :r // 2] = bound[..., r // 2:r] = e
    else:
        want[..., 0:r:2], want[..., 1:r:2] = u, v
        bound[..., 0:r:2] = bound[..., 1:r:2] = e
    return want, bound


def scores(q, k, scale):
    """z = scale q k^T in 64 bits and how far the kernel's exponents z - m may be off: dh products and the scaling in fp32, and the
    roundings of z, m and their difference."""
    z = (q @ k.t().contiguous()) * scale
    size = (q.abs() @ k.abs().t().contiguous()) * scale
    return z, (q.shape[1] + 4) * U * size + 6 * U * (z.abs().amax() + 1)


def attend(q, k, v, scale, hidden):
    """(out, lse, bound of out, bound of lse) of one head; hidden [n, m] bool."""
    q, k, v = q.double(), k.double(), v.double()
    z, dz = scores(q, k, scale)
    z = z.masked_fill(hidden, -math.inf)
    d = dz.masked_fill(hidden, 0.0).amax(1, keepdim=True)
    n = k.shape[0]
    lse = torch.logsumexp(z, 1, keepdim=True)
    p = (z - lse).exp()
    # probabilities rounded to bf16; sums and rescalings in fp32; the total divides
    rel = B16 + 3 * d + (3 * n + 40) * U
    out = p @ v
    return out, lse[:, 0], (p @ v.abs()) * rel, (2 * d + (n + 16) * U + 4 * U * lse.abs())[:, 0]


def causal(q, k, v, lengths, scale):
    """Outputs and log-sums of packed sequences with their bounds: (out, lse [H, T], bound of out, bound of lse)."""
    T, H, dh = q.shape
    group = H // k.shape[1]
    out, eo = torch.zeros(T, H, dh, dtype=torch.float64, device=q.device), torch.zeros(T, H, dh, dtype=torch.float64, device=q.device)
    lse, el = torch.zeros(H, T, dtype=torch.float64, device=q.device), torch.zeros(H, T, dtype=torch.float64, device=q.device)
    a = 0
    for n in lengths:
        r = slice(a, a + n)
        hidden = torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1)
        for h in range(H if n else 0):
            j = h // group
            out[r, h], lse[h, r], eo[r, h], el[h, r] = attend(q[r, h], k[r, j], v[r, j], scale, hidden)
        a += n
    return out, lse, eo, el


SUMMED = 128       # a sequence's first rows, whose delta is summed from P dP


def causal_back(dout, q, k, v, out, lse, lengths, scale, exact_out=False):
    """{name: (gradient, bound)} for given out and lse; exact_out: their 64-bit values, against a kernel that has them
    rounded.  delta is the sum of dO O, in the first rows that of P dP."""
    T, H, dh = q.shape
    group = H // k.shape[1]
    want = {x: torch.zeros(t.shape, dtype=torch.float64, device=q.device) for x, t in (("dq", q), ("dk", k), ("dv", v))}
    off = {x: torch.zeros_like(t) for x, t in want.items()}
    a = 0
    for n in lengths:
        r = slice(a, a + n)
        a += n
        if n == 0:
            continue
        hidden = torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1)
        for h in range(H):
            j = h // group
            Q, K, V, G, O = (t.double() for t in (q[r, h], k[r, j], v[r, j], dout[r, h], out[r, h]))
            L = lse[h, r].double()[:, None]
            z, dz = scores(Q, K, scale)
            p = (z - L).exp().masked_fill(hidden, 0.0)
            dp, size = G @ V.t().contiguous(), G.abs() @ V.abs().t().contiguous()
            delta, dsize = (G * O).sum(1, keepdim=True), (G * O).abs().sum(1, keepdim=True)
            ep = dz + 8 * U * (L.abs() + 1)                                   # of p, relative; the lse's own rounding
            # The kernel's sum of P (dP - delta'), delta' from the rounded out, is off by that of P's and dP's errors and by its
            # own additions; what the sum of its P is off 1 by multiplies what delta' lacks.
            first = torch.arange(n, device=q.device)[:, None] < SUMMED
            soft = torch.softmax(z.masked_fill(hidden, -math.inf), 1)
            summed = (soft * dp).sum(1, keepdim=True)
            lacks, near = (summed - delta).abs() + (G.abs() * half_step(O)).sum(1, keepdim=True), soft * (dp - summed).abs()
            es = (soft * (dh + 4) * U * (size + dsize) + (2 * ep + (n + 8) * U) * near).sum(1, keepdim=True)
            es = es + (4 * ep.amax(1, keepdim=True) + (n + 16) * U) * lacks          # (the lse's error too)
            delta = torch.where(first, summed, delta)
            ds = p * (dp - delta)
            ed = (dh + 4) * U * (size + dsize) + 2 * U * (dp.abs() + delta.abs()) + torch.where(first, es, 0.0)
            if exact_out:
                # (delta is formed from the rounded out)
                ed = ed + torch.where(first, 0.0, (G.abs() * half_step(O)).sum(1, keepdim=True))
                ep = ep + 4 * U * L.abs()
            e = p * (2 * ep * (dp - delta).abs() + ed) + B16 * ds.abs()       # dS is rounded to bf16
            sums = (H * n + 40) * U
            want["dq"][r, h] = scale * (ds @ K)
            off["dq"][r, h] = scale * ((e + sums * ds.abs()) @ K.abs())
            want["dk"][r, j] += scale * (ds.t().contiguous() @ Q)
            off["dk"][r, j] += scale * ((e + sums * ds.abs()).t().contiguous() @ Q.abs())
            want["dv"][r, j] += p.t().contiguous() @ G
            off["dv"][r, j] += (p * (B16 + 2 * ep + sums)).t().contiguous() @ G.abs()
    return {x: (want[x], off[x]) for x in want}
