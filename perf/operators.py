"""The operators that follow the attention layer, and the work they are measured on.

  ffn      the gated feed-forward block: "infer" (serving, with the residual), "fwd" (training: also
           what the backward needs) and "bwd" (gradients of the input and both weights)
  dropout  dropout from a counter-based generator, added to the residual branch or alone
  loss     softmax cross entropy of token rows against a set of item rows: "eval" (losses) or
           "train" (losses and gradients)

Values are those of a trained block: normalised activations ~ N(0, 1), weights ~ N(0, 1 / fan-in),
item labels after a Zipf law, the class bias minus the log of their frequency (the correction of a
class set drawn by popularity).  Only part of the token rows have a label.
"""
import math

import numpy as np
import torch

own = False

M32 = 0xFFFFFFFF


def listed():
    return [
        # serving, one token of one user: the latency of two weight reads
        dict(name="ffn_token", kind="ffn", how="infer", T=1, d=512, f=1408),
        # serving, the candidates of one request
        dict(name="ffn_request", kind="ffn", how="infer", T=312, d=768, f=2048),
        # forward pass of a training batch of the small model (128 users)
        dict(name="ffn_fwd", kind="ffn", how="fwd", T=75132, d=512, f=1408),
        # backward pass of a development-size batch (32 users)
        dict(name="ffn_bwd_small", kind="ffn", how="bwd", T=6418, d=256, f=704),
        # backward pass of a training batch of the large model (64 users)
        dict(name="ffn_bwd", kind="ffn", how="bwd", T=69563, d=1024, f=2816),
        # the smallest batch, fp32: launches and host time
        dict(name="dropout_tiny", kind="dropout", rows=96, cols=32, dtype="fp32", p=0.5, residual=False),
        # the residual branch of a training batch of the large model
        dict(name="dropout_large", kind="dropout", rows=69563, cols=1024, dtype="bf16", p=0.1, residual=True),
        # loss of a single row: one read of the item rows
        dict(name="loss_one", kind="loss", how="eval", N=1, n=1, V=30011, d=128, bias=False),
        # evaluation losses of a few users' sequences
        dict(name="loss_eval", kind="loss", how="eval", N=3000, n=2900, V=20011, d=256, bias=True),
        # training step of a development-size batch against its own de-duplicated items
        dict(name="loss_train_small", kind="loss", how="train", N=6418, n=2007, V=5003, d=128, bias=True),
        # training step of a few labelled rows against a whole catalogue
        dict(name="loss_train_items", kind="loss", how="train", N=2048, n=1900, V=400003, d=256, bias=False),
        # training step of a large batch: a third of the tokens have a label
        dict(name="loss_train_large", kind="loss", how="train", N=69563, n=24000, V=50021, d=512, bias=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["ffn", "ffn", "ffn", "dropout", "loss", "loss"])
    if kind == "dropout":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        step = 8 if dtype == "bf16" else 4
        cols = step * _log(rng, 4, 2048 // step)
        rows = _log(rng, 1, min(80000, 69563 * 1024 // (cols * (1 if dtype == "bf16" else 2))))
        return dict(kind=kind, rows=rows, cols=cols, dtype=dtype, p=rng.choice([0.0, 0.1, 0.2, 0.35, 0.5, 0.9]),
                    residual=rng.random() < 0.5)
    if kind == "ffn":
        how = rng.choice(["infer", "infer", "fwd", "bwd"])
        d, f = 32 * _log(rng, 2, 32), 32 * _log(rng, 3, 88)
        T = _log(rng, 1, min(80000, 69563 * 1024 * 2816 // (d * f)))
        return dict(kind=kind, how=how, T=T, d=d, f=f)
    how = rng.choice(["eval", "train"])
    d, V = 32 * _log(rng, 1, 32), _log(rng, 2, 400000)
    n = _log(rng, 1, min(40000, 24000 * 50021 * 512 // (d * V)))
    N = min(80000, int(n * rng.choice([1.0, 1.0, 1.4, 3.0])) + rng.randrange(3))
    return dict(kind=kind, how=how, N=N, n=n, V=V, d=d, bias=rng.random() < 0.5)


def work(case):
    if case["kind"] == "dropout":
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": case["rows"] * case["cols"] * size * (3 if case["residual"] else 2), "flops": 0}
    if case["kind"] == "ffn":
        T, d, f = case["T"], case["d"], case["f"]
        weights = 3 * d * f
        if case["how"] == "bwd":
            return {"bytes": 2 * (3 * T * d + 3 * T * f + 2 * weights), "flops": 12 * T * d * f}
        more = T * d if case["how"] == "infer" else 3 * T * f
        return {"bytes": 2 * (2 * T * d + weights + more), "flops": 6 * T * d * f}
    n, N, V, d = case["n"], case["N"], case["V"], case["d"]
    nbytes = 2 * (n * d + V * d) + 16 * N + (4 * V if case["bias"] else 0)
    if case["how"] == "eval":
        return {"bytes": nbytes, "flops": 2 * n * V * d}
    return {"bytes": nbytes + 4 * N + 2 * (N * d + V * d) + (4 * V if case["bias"] else 0), "flops": 6 * n * V * d}


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 + seed)


def _normal(g, *shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def prepare(case, seed):
    g = _gen(seed)
    if case["kind"] == "dropout":
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        shape = (case["rows"], case["cols"])
        return dict(case=case, x=_normal(g, *shape, dtype=dt), p=case["p"], site=3,
                    residual=_normal(g, *shape, dtype=dt) if case["residual"] else None,
                    rng=torch.tensor([0x5DEECE66D0 + 7919 * seed, 40 + seed], dtype=torch.int64, device="cuda"))
    if case["kind"] == "ffn":
        T, d, f = case["T"], case["d"], case["f"]
        s = dict(case=case, x=_normal(g, T, d), w_in=_normal(g, d, 2 * f, scale=d ** -0.5),
                 w_out=_normal(g, f, d, scale=f ** -0.5))
        if case["how"] == "infer":
            s["residual"] = _normal(g, T, d)
        if case["how"] == "bwd":                    # what the forward pass left
            s["dy"] = _normal(g, T, d, scale=0.1)
            pre = s["x"].float() @ s["w_in"].float()
            s["h"] = (pre[:, :f] * torch.sigmoid(pre[:, :f]) * pre[:, f:]).bfloat16()
            s["pre"] = pre.bfloat16()
        return s
    N, n, V, d = case["N"], case["n"], case["V"], case["d"]
    r = np.random.default_rng([seed, 5])
    targets = np.full(N, -1, np.int64)
    targets[r.permutation(N)[:n]] = np.minimum((V + 1.0) ** r.random(n) - 1.0, V - 1).astype(np.int64)
    s = dict(case=case, x=_normal(g, N, d), w=_normal(g, V, d, scale=2.0 * d ** -0.5), scale=0.8,
             targets=torch.from_numpy(targets).cuda(), bias=None)
    if case["bias"]:
        s["bias"] = 0.5 * torch.log(torch.arange(1, V + 1, device="cuda", dtype=torch.float32))
    if case["how"] == "train":
        s["dloss"] = torch.full((N,), 1.0 / n, device="cuda")
    return s


# ------------------------------------------------------------------ one pass

def _philox(seed, c):
    """Philox4x32 with 7 rounds: four 32-bit words per counter, as int64."""
    k0, k1 = seed & M32, (seed >> 32) & M32
    for i in range(7):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((p1 >> 32) & M32) ^ c[1] ^ k0, p1 & M32, ((p0 >> 32) & M32) ^ c[3] ^ k1, p0 & M32]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return c


def _dropout(s):
    x = s["x"]
    quad = torch.arange(x.numel() // 4, device="cuda")
    seed, step = s["rng"][0], s["rng"][1]
    site = torch.full_like(quad, s["site"])
    words = torch.stack(_philox(seed, [quad & M32, quad >> 32, site, (step & M32).expand_as(quad)]), 1)
    keep = (words >= int(s["p"] * 2.0 ** 32)).view(x.shape)
    out = torch.where(keep, x.float() * (1.0 / (1.0 - s["p"])), 0.0)
    return {"out": (out if s["residual"] is None else out + s["residual"].float()).to(x.dtype)}


def _ffn(s):
    f = s["case"]["f"]
    x, w_in, w_out = s["x"].float(), s["w_in"].float(), s["w_out"].float()
    if s["case"]["how"] == "bwd":
        dy, gate, up = s["dy"].float(), s["pre"][:, :f].float(), s["pre"][:, f:].float()
        dh = dy @ w_out.t()
        sg = torch.sigmoid(gate)
        dpre = torch.cat([dh * up * sg * (1 + gate * (1 - sg)), dh * gate * sg], 1)
        return {"dx": (dpre @ w_in.t()).bfloat16(), "dw_in": (x.t() @ dpre).bfloat16(),
                "dw_out": (s["h"].float().t() @ dy).bfloat16()}
    pre = x @ w_in
    h = pre[:, :f] * torch.sigmoid(pre[:, :f]) * pre[:, f:]
    y = h @ w_out
    if s["case"]["how"] == "infer":
        return {"y": (y + s["residual"].float()).bfloat16()}
    return {"y": y.bfloat16(), "pre": pre.bfloat16(), "h": h.bfloat16()}


def _loss(s):
    t = s["targets"]
    rows = (t >= 0).nonzero().squeeze(1)
    x, w, t = s["x"][rows].float(), s["w"].float(), t[rows]
    z = (x @ w.t()) * s["scale"]
    if s["bias"] is not None:
        z = z + s["bias"]
    top = z.max(1, keepdim=True).values
    lse = (z - top).exp().sum(1).log() + top.squeeze(1)
    N = s["case"]["N"]
    out = {"loss": torch.zeros(N, device="cuda").index_copy(0, rows, lse - z.gather(1, t[:, None]).squeeze(1)),
           "lse": torch.zeros(N, device="cuda").index_copy(0, rows, lse)}
    if s["case"]["how"] == "eval":
        return out
    dz = (z - lse[:, None]).exp()
    dz[torch.arange(len(t), device="cuda"), t] -= 1.0
    dz = dz * s["dloss"][rows][:, None]
    dx = (dz @ w) * s["scale"]
    out["dx"] = torch.zeros(s["x"].shape, device="cuda").index_copy(0, rows, dx).bfloat16()
    out["dw"] = ((dz.t() @ x) * s["scale"]).bfloat16()
    if s["bias"] is not None:
        out["dbias"] = dz.sum(0)
    return out


def run(state):
    case = state["case"]
    if not own:
        return {"dropout": _dropout, "ffn": _ffn, "loss": _loss}[case["kind"]](state)
    from paper_2505_18654_amd import ops
    s = state
    if case["kind"] == "dropout":
        return {"out": ops.dropout(s["x"], s["p"], s["rng"], s["site"], residual=s["residual"])}
    if case["kind"] == "ffn":
        if case["how"] == "infer":
            return {"y": ops.gated_ffn_fwd(s["x"], s["w_in"], s["w_out"], residual=s["residual"])}
        if case["how"] == "fwd":
            y, pre, h = ops.gated_ffn_fwd(s["x"], s["w_in"], s["w_out"], save=True)
            return {"y": y, "pre": pre, "h": h}
        dx, dw_in, dw_out = ops.gated_ffn_bwd(s["dy"], s["x"], s["pre"], s["h"], s["w_in"], s["w_out"])
        return {"dx": dx, "dw_in": dw_in, "dw_out": dw_out}
    loss, lse = ops.softmax_loss_fwd(s["x"], s["w"], s["targets"], bias=s["bias"], scale=s["scale"])
    out = {"loss": loss, "lse": lse}
    if case["how"] == "train":
        dx, dw, dbias = ops.softmax_loss_bwd(s["dloss"], s["x"], s["w"], s["targets"], lse, bias=s["bias"],
                                             scale=s["scale"])
        out.update(dx=dx, dw=dw)
        if dbias is not None:
            out["dbias"] = dbias
    return out


# ------------------------------------------------------------------ in 64 bits

def _exact_dropout(case, s):
    seed, step = (int(v) for v in s["rng"].cpu())
    x = s["x"].double().cpu().numpy().reshape(-1)
    q = np.arange(x.size // 4, dtype=np.uint64)
    c = [q & np.uint64(M32), q >> np.uint64(32), np.full_like(q, s["site"]), np.full_like(q, step & M32)]
    key = [seed & M32, (seed >> 32) & M32]
    for _ in range(7):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(key[0]), b & np.uint64(M32),
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(key[1]), a & np.uint64(M32)]
        key = [(key[0] + 0x9E3779B9) & M32, (key[1] + 0xBB67AE85) & M32]
    kept = np.stack(c, 1).reshape(-1) >= np.uint64(math.floor(s["p"] * 2.0 ** 32))
    out = np.where(kept, x / (1.0 - s["p"]), 0.0)
    if s["residual"] is not None:
        out += s["residual"].double().cpu().numpy().reshape(-1)
    return {"out": out.reshape(s["x"].shape)}


def _exact_ffn(case, s):
    f = case["f"]
    x, w_in, w_out = s["x"].double(), s["w_in"].double(), s["w_out"].double()
    if case["how"] == "bwd":
        dy, a, b = s["dy"].double(), s["pre"][:, :f].double(), s["pre"][:, f:].double()
        dh = torch.matmul(dy, w_out.t().contiguous())
        e = torch.exp(-a)
        da = dh * b * (1 / (1 + e) + a * e / (1 + e) ** 2)
        db = dh * a / (1 + e)
        dx = torch.matmul(da, w_in[:, :f].t().contiguous()) + torch.matmul(db, w_in[:, f:].t().contiguous())
        xt = x.t().contiguous()
        return {"dx": dx, "dw_in": torch.cat([torch.matmul(xt, da), torch.matmul(xt, db)], 1),
                "dw_out": torch.matmul(s["h"].double().t().contiguous(), dy)}
    a, b = torch.matmul(x, w_in[:, :f].contiguous()), torch.matmul(x, w_in[:, f:].contiguous())
    h = a / (1 + torch.exp(-a)) * b
    y = torch.matmul(h, w_out)
    if case["how"] == "infer":
        return {"y": y + s["residual"].double()}
    return {"y": y, "pre": torch.cat([a, b], 1), "h": h}


def _exact_loss(case, s):
    N, V, d = case["N"], case["V"], case["d"]
    on = s["targets"] >= 0
    x, w, t = s["x"][on].double(), s["w"].double(), s["targets"][on]
    z = s["scale"] * torch.matmul(x, w.t().contiguous())
    if s["bias"] is not None:
        z += s["bias"].double()
    lse = torch.logsumexp(z, 1)
    zt = s["scale"] * (x * w[t]).sum(1)
    if s["bias"] is not None:
        zt += s["bias"].double()[t]
    loss, whole = torch.zeros(N, dtype=torch.float64, device="cuda"), torch.zeros(N, dtype=torch.float64, device="cuda")
    loss[on], whole[on] = lse - zt, lse
    out = {"loss": loss, "lse": whole}
    if case["how"] == "eval":
        return out
    g = s["dloss"][on].double()
    p = z.sub_(lse[:, None]).exp_().mul_(g[:, None])          # g softmax; the label's part is subtracted below
    dx = torch.zeros(N, d, dtype=torch.float64, device="cuda")
    dx[on] = s["scale"] * (torch.matmul(p, w) - g[:, None] * w[t])
    dw = torch.matmul(p.t().contiguous(), x).index_add_(0, t, -g[:, None] * x)
    out.update(dx=dx, dw=s["scale"] * dw)
    if s["bias"] is not None:
        out["dbias"] = p.sum(0).index_add_(0, t, -g)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"dropout": _exact_dropout, "ffn": _exact_ffn, "loss": _exact_loss}[case["kind"]](case, s)
