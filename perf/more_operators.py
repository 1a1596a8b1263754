"""Softmax attention over a user's own past, for next-item training and for generating items one by one, and the
work it is measured on.

  rope    rotary positions of packed heads, forward ("fwd") or the gradient's way back ("bwd")
  attn    causal softmax attention of packed sequences with grouped heads: outputs and log-sums ("fwd"), or the
          gradients of q, k and v from what the forward left ("bwd")
  append  new tokens' keys (rotated on the way) and values into a paged cache, their queries rotated too
  decode  one token of each sequence against its paged cache

Queries and keys are normalised projections ~ N(0, 1), so that scores q.k / sqrt(head_dim) have a deviation of about
one.  Lengths follow a lognormal law with a long tail, the longest given; a sequence of one token is among them.  Pages
of a cache lie in random order, the last one of a sequence partly filled.
"""
import math

import numpy as np
import torch

own = False


def listed():
    return [
        # serving: queries and keys of one request's tokens, whole heads
        dict(name="rope_request", kind="rope", how="fwd", T=312, heads=8, row=10, dh=128, rot=128, layout="half",
             dtype="bf16", scaling="none"),
        # training batch of the large model: the gradients' rotation back, half of each head
        dict(name="rope_train", kind="rope", how="bwd", T=69563, heads=10, row=12, dh=128, rot=64, layout="interleaved",
             dtype="bf16", scaling="linear"),
        # the prompt of one request
        dict(name="attn_request", kind="attn", how="fwd", B=1, longest=700, heads=6, kv=2, dh=128),
        # a few whole histories, one of them very long
        dict(name="attn_histories", kind="attn", how="fwd", B=4, longest=16001, heads=16, kv=2, dh=128),
        # training step of a development-size batch
        dict(name="attn_train_small", kind="attn", how="bwd", B=32, longest=320, heads=4, kv=4, dh=64),
        # training step of a large batch
        dict(name="attn_train", kind="attn", how="bwd", B=64, longest=3200, heads=8, kv=2, dh=128),
        # one step of generation for some sessions: a token each
        dict(name="append_step", kind="append", B=64, new=1, longest=2000, heads=8, kv=2, dh=128, page=32,
             rot=128, layout="half", scaling="parts"),
        # prompts of a batch of sessions, onto what their caches hold
        dict(name="append_prompts", kind="append", B=24, new=2800, longest=3000, heads=8, kv=2, dh=128, page=64,
             rot=128, layout="half", scaling="none"),
        # the first tokens of one session: latency
        dict(name="decode_first", kind="decode", B=1, longest=411, heads=8, kv=2, dh=128, page=32),
        # one session with a very long history: little work to spread over the chip
        dict(name="decode_long", kind="decode", B=1, longest=100003, heads=6, kv=2, dh=128, page=64),
        # a serving batch of ordinary histories
        dict(name="decode_batch", kind="decode", B=128, longest=3000, heads=8, kv=4, dh=64, page=16),
        # a full serving batch of long histories: gigabytes of cache
        dict(name="decode_large", kind="decode", B=24, longest=131072, heads=32, kv=8, dh=128, page=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "attn", "attn", "attn", "append", "decode", "decode"])
    dh, kv = rng.choice([32, 64, 64, 128, 128, 128]), rng.choice([1, 2, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 8])
    if kind == "rope":
        rot = rng.choice([r for r in (16, 32, 48, 64, 96, 128) if r <= dh])
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        row = heads + rng.choice([0, 2, kv])
        T = _log(rng, 1, min(80000, 69563 * 10 * 128 // (heads * dh * (1 if dtype == "bf16" else 2))))
        return dict(kind=kind, how=rng.choice(["fwd", "bwd"]), T=T, heads=heads, row=row, dh=dh, rot=rot,
                    layout=rng.choice(["half", "interleaved"]), dtype=dtype,
                    scaling=rng.choice(["none", "linear", "base", "parts"]))
    if kind == "attn":
        how = rng.choice(["fwd", "bwd"])
        most = (3.9e11 if how == "fwd" else 6e10) / (heads * dh)        # pairs of queries and keys, at most
        # (sequences of one token alone have gradients of zero, which say nothing: the long ones are longer)
        longest = _log(rng, 1 if how == "fwd" else 8, min(16001, int(math.sqrt(2 * most))))
        B = _log(rng, 1, max(1, min(256, int(most / (longest * (longest + 1) / 2)))))
        return dict(kind=kind, how=how, B=B, longest=longest, heads=heads, kv=kv, dh=dh)
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "append":
        new = rng.choice([1, 1, _log(rng, 2, 4000)])
        B = _log(rng, 1, max(1, min(256, 24 * 2800 * 2 * 128 // (new * heads * dh))))
        return dict(kind=kind, B=B, new=new, longest=_log(rng, 1, 4000), heads=heads, kv=kv, dh=dh, page=page,
                    rot=rng.choice([r for r in (16, 32, 64, 128) if r <= dh]), layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "base", "parts"]))
    longest = _log(rng, 1, 131072)
    B = _log(rng, 1, max(1, min(512, 24 * 131072 * 8 * 128 // (2 * longest * kv * dh))))
    return dict(kind=kind, B=B, longest=longest, heads=heads, kv=kv, dh=dh, page=page)


def _lengths(B, longest, more=0):
    """B lengths of at most `longest`, that one among them and, from three on, a one."""
    r = np.random.default_rng([B, longest, more])
    n = np.clip(np.rint(longest / 4 * r.lognormal(0.0, 0.9, B)), 1, longest).astype(np.int64)
    n[r.integers(B)] = longest
    if B > 2:
        n[np.argmin(n)] = 1
    return n


def _pasts(case):
    return _lengths(case["B"], case["longest"])


def _news(case):
    return np.ones(case["B"], np.int64) if case["new"] == 1 else _lengths(case["B"], case["new"], 1)


def work(case):
    kind, dh, H = case["kind"], case["dh"], case["heads"]
    if kind == "rope":
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": case["T"] * (2 * H * dh * size + 4) + 4 * case["rot"], "flops": 3 * case["T"] * H * case["rot"]}
    kv = case["kv"]
    if kind == "append":
        N = int(_news(case).sum())
        return {"bytes": 2 * 2 * N * dh * (H + 2 * kv) + 12 * case["B"], "flops": 3 * N * (H + kv) * case["rot"]}
    n = _lengths(case["B"], case["longest"])
    if kind == "decode":
        T, B = int(n.sum()), case["B"]
        pages = int(((n + case["page"] - 1) // case["page"]).sum())
        return {"bytes": 4 * T * kv * dh + B * (4 * H * dh + 4 * H + 4) + 4 * pages, "flops": 4 * T * H * dh}
    T, pairs = int(n.sum()), int((n * (n + 1) // 2).sum())
    if case["how"] == "fwd":
        return {"bytes": 4 * T * dh * (H + kv) + 4 * T * H, "flops": 4 * pairs * H * dh}
    return {"bytes": 2 * T * dh * (4 * H + 4 * kv) + 4 * T * H, "flops": 10 * pairs * H * dh}


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(7000003 + seed)


def _normal(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _frequencies(rot, scaling):
    """Angles per position of the rot / 2 pairs, in radians, and the factor on cosine and sine.  The scalings stretch a
    model trained on 1,024 positions to eight times as many."""
    base, factor, trained = 10000.0, 8.0, 1024
    if scaling == "base":
        base *= factor ** (rot / (rot - 2.0))
    f = base ** (-np.arange(0, rot, 2) / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":                 # few turns over the trained positions: stretched; many: left alone
        keep = np.clip((trained * f / (2 * math.pi) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        f = f * (keep + (1 - keep) / factor)
    return torch.from_numpy(f).cuda(), 0.1 * math.log(factor) + 1.0 if scaling == "parts" else 1.0


def _offsets(n):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).cuda()


def _cache(g, case, n):
    """A paged cache that has room for n tokens of each sequence: keys, values and the page table."""
    pages = -(-n // case["page"])
    total = int(pages.sum()) + 5
    order = torch.randperm(total, generator=g, device="cuda").int()
    table = torch.full((case["B"], int(pages.max())), -1, dtype=torch.int32, device="cuda")
    used = torch.arange(table.shape[1], device="cuda")[None, :] < torch.from_numpy(pages).cuda()[:, None]
    table[used] = order[: int(pages.sum())]
    shape = (total, case["kv"], case["page"], case["dh"])
    return dict(keys=_normal(g, *shape), values=_normal(g, *shape), table=table)


def prepare(case, seed):
    g, kind, dh, H = _gen(seed), case["kind"], case["dh"], case["heads"]
    s = dict(case=case)
    if kind in ("rope", "append"):
        s["freqs"], s["amplitude"] = _frequencies(case["rot"], case["scaling"])
    if kind == "rope":
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        T = case["T"]
        s["x"] = _normal(g, T, case["row"], dh, dtype=dt)[:, :H]         # columns of a wider projection
        n = _lengths(max(1, T // 1087), min(T, 3200))
        at = np.arange(T) % int(n.max()) + 40 + seed % 7                 # behind what a cache may hold
        s["positions"] = torch.from_numpy(at.astype(np.int32)).cuda()
        return s
    kv = case["kv"]
    if kind == "append":
        past, new = _pasts(case), _news(case)
        s.update(_cache(g, case, past + new))
        rows = _normal(g, int(new.sum()), H + 2 * kv, dh)                # one fused projection
        s["q"], s["k"], s["v"] = rows[:, :H], rows[:, H:H + kv], rows[:, H + kv:]
        s["past"], s["offsets"] = torch.from_numpy(past.astype(np.int32)).cuda(), _offsets(new)
        return s
    n = _lengths(case["B"], case["longest"])
    if kind == "decode":
        s.update(_cache(g, case, n))
        s["q"], s["lens"] = _normal(g, case["B"], H, dh), torch.from_numpy(n.astype(np.int32)).cuda()
        s["longest"] = case["longest"]
        return s
    rows = _normal(g, int(n.sum()), H + 2 * kv, dh)
    s["q"], s["k"], s["v"] = rows[:, :H], rows[:, H:H + kv], rows[:, H + kv:]
    s["lengths"], s["offsets"] = n, _offsets(n)
    if case["how"] == "bwd":
        s["dout"] = _normal(g, int(n.sum()), H, dh)
        s["out"], s["lse"] = _attn(s).values()                           # what the forward pass left
    return s


# ------------------------------------------------------------------ one pass

def _rotated(x, freqs, positions, amplitude, layout):
    """x [T, heads, dh] in 32 bits, its first 2 len(freqs) features rotated."""
    r = 2 * len(freqs)
    angle = positions.double()[:, None, None] * freqs
    c, s = (angle.cos() * amplitude).float(), (angle.sin() * amplitude).float()
    if layout == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * c - b * s, a * s + b * c, x[..., r:]], -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2), x[..., r:]], -1)


def _rope(s):
    case = s["case"]
    at = s["positions"] if case["how"] == "fwd" else -s["positions"]
    return {"out": _rotated(s["x"].float(), s["freqs"], at, s["amplitude"], case["layout"]).to(s["x"].dtype)}


def _append(s):
    case, dev = s["case"], s["q"].device
    t = torch.arange(s["q"].shape[0], device=dev)
    b = torch.searchsorted(s["offsets"], t, right=True, out_int32=True) - 1
    at = s["past"][b].long() + t - s["offsets"][b]
    page, row = s["table"][b, at // case["page"]].long(), at % case["page"]
    q, k = (_rotated(s[x].float(), s["freqs"], at, s["amplitude"], case["layout"]).bfloat16() for x in "qk")
    s["keys"][page, :, row] = k
    s["values"][page, :, row] = s["v"]
    return {"q": q, "keys": s["keys"], "values": s["values"]}


def _decode(s):
    case, q = s["case"], s["q"].float()
    B, H, dh = q.shape
    kv, table = case["kv"], s["table"].clamp(min=0).long()
    k, v = (s[x][table].transpose(1, 2).reshape(B, kv, -1, dh).float() for x in ("keys", "values"))
    z = torch.matmul(k, q.view(B, kv, H // kv, dh).transpose(2, 3).contiguous()).transpose(2, 3) * dh ** -0.5
    out_of = torch.arange(z.shape[3], device=q.device) >= s["lens"][:, None]
    z = z.masked_fill(out_of[:, None, None, :], -math.inf)
    top = z.max(-1, keepdim=True).values
    p = (z - top).exp()
    total = p.sum(-1, keepdim=True)
    return {"out": (torch.matmul(p, v) / total).view(B, H, dh).bfloat16(), "lse": (total.log() + top).view(B, H)}


def _heads_first(x, a, b, kv):
    """Rows a to b of x [T, heads, dh] as [kv, heads / kv * rows, dh] in 32 bits, a key head's queries one after another."""
    return x[a:b].float().transpose(0, 1).reshape(kv, -1, x.shape[2])


def _probabilities(q, k, n, scale):
    """Scores of a sequence's queries and keys: exp(z - top) [kv, heads / kv, n, n], its row sums and top."""
    z = torch.matmul(q, k.transpose(1, 2).contiguous()).view(k.shape[0], -1, n, n) * scale
    z.masked_fill_(torch.ones(n, n, dtype=torch.bool, device=z.device).triu_(1), -math.inf)
    top = z.max(-1, keepdim=True).values
    p = z.sub_(top).exp_()
    return p, p.sum(-1, keepdim=True), top


def _attn(s):
    case = s["case"]
    kv, dh, T, H = case["kv"], case["dh"], s["q"].shape[0], case["heads"]
    out = torch.empty(T, H, dh, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(H, T, device="cuda")
    a = 0
    for n in s["lengths"].tolist():                                      # a sequence's scores fit the memory, a batch's need not
        q, k, v = (_heads_first(s[x], a, a + n, kv) for x in "qkv")
        p, total, top = _probabilities(q, k, n, dh ** -0.5)
        o = torch.matmul(p.view(kv, -1, n), v).view(H, n, dh) / total.view(H, n, 1)
        out[a:a + n] = o.transpose(0, 1)
        lse[:, a:a + n] = (total.log() + top).view(H, n)
        a += n
    return {"out": out, "lse": lse}


def _attn_bwd(s):
    case = s["case"]
    kv, dh, H = case["kv"], case["dh"], case["heads"]
    grads = {"d" + x: torch.empty(s[x].shape, dtype=torch.bfloat16, device="cuda") for x in "qkv"}
    a = 0
    for n in s["lengths"].tolist():
        q, k, v, g = (_heads_first(s[x], a, a + n, kv) for x in ("q", "k", "v", "dout"))
        p, total, _ = _probabilities(q, k, n, dh ** -0.5)
        p = p.div_(total).view(kv, -1, n)
        dz = torch.matmul(g, v.transpose(1, 2).contiguous())
        dz = dz.sub_((dz * p).sum(-1, keepdim=True)).mul_(p).mul_(dh ** -0.5)
        grads["dq"][a:a + n] = torch.matmul(dz, k).view(H, n, dh).transpose(0, 1)
        grads["dk"][a:a + n] = torch.matmul(dz.transpose(1, 2).contiguous(), q).transpose(0, 1)
        grads["dv"][a:a + n] = torch.matmul(p.transpose(1, 2).contiguous(), g).transpose(0, 1)
        a += n
    return grads


def run(state):
    case, s = state["case"], state
    kind = case["kind"]
    if not own:
        if kind == "attn":
            return _attn(s) if case["how"] == "fwd" else _attn_bwd(s)
        return {"rope": _rope, "append": _append, "decode": _decode}[kind](s)
    from paper_2505_18654_amd import ops
    if kind == "rope":
        rotary = ops.Rotary(s["freqs"], case["layout"], s["amplitude"])
        return {"out": ops.rope(s["x"], rotary, positions=s["positions"], inverse=case["how"] == "bwd")}
    if kind == "attn":
        if case["how"] == "fwd":
            out, lse = ops.causal_attn_fwd(s["q"], s["k"], s["v"], s["offsets"], save=True)
            return {"out": out, "lse": lse}
        dq, dk, dv = ops.causal_attn_bwd(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["offsets"])
        return {"dq": dq, "dk": dk, "dv": dv}
    cache = ops.KvCache(s["keys"], s["values"])
    if kind == "append":
        rotary = ops.Rotary(s["freqs"], case["layout"], s["amplitude"])
        q = ops.kv_append(cache, s["table"], s["past"], s["k"], s["v"], offsets=s["offsets"], q=s["q"], rotary=rotary)
        return {"q": q, "keys": s["keys"], "values": s["values"]}
    out, lse = ops.cache_attn(s["q"], cache, s["table"], s["lens"], max_len=s["longest"], save=True)
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------ in 64 bits

def _exact_rotated(x, freqs, at, amplitude, layout):
    """Rotation of each pair as a product of complex numbers."""
    r = 2 * len(freqs)
    turn = torch.polar(torch.full((len(at), len(freqs)), amplitude, dtype=torch.float64, device="cuda"),
                       at.double()[:, None] * freqs)[:, None]
    y = x.double()
    if layout == "half":
        z = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * turn
        pairs = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.view_as_complex(y[..., :r].reshape(*y.shape[:-1], r // 2, 2).contiguous()) * turn
        pairs = torch.view_as_real(z).reshape(*y.shape[:-1], r)
    return torch.cat([pairs, y[..., r:]], -1)


def _exact_append(case, s):
    at = torch.cat([torch.arange(p, p + m) for p, m in zip(_pasts(case).tolist(), _news(case).tolist())]).cuda()
    q, k = (_exact_rotated(s[x], s["freqs"], at, s["amplitude"], case["layout"]) for x in "qk")
    keys, values, t = s["keys"].double(), s["values"].double(), 0
    for b, (p, m) in enumerate(zip(_pasts(case).tolist(), _news(case).tolist())):
        i = torch.arange(p, p + m, device="cuda")
        page = s["table"][b].long()[i // case["page"]]
        keys[page, :, i % case["page"]], values[page, :, i % case["page"]] = k[t:t + m], s["v"][t:t + m].double()
        t += m
    return {"q": q, "keys": keys, "values": values}


def _exact_decode(case, s):
    H, kv, dh = case["heads"], case["kv"], case["dh"]
    out = torch.empty(case["B"], H, dh, dtype=torch.float64, device="cuda")
    lse = torch.empty(case["B"], H, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        page = s["table"][b, : -(-n // case["page"])].long()
        for h in range(kv):
            k, v = (s[x][page, h].reshape(-1, dh)[:n].double() for x in ("keys", "values"))
            rows = slice(h * H // kv, (h + 1) * H // kv)
            z = torch.matmul(k, (s["q"][b, rows].double() / math.sqrt(dh)).t().contiguous()).t().contiguous()
            lse[b, rows] = torch.logsumexp(z, 1)
            out[b, rows] = torch.matmul((z - lse[b, rows, None]).exp(), v)
    return {"out": out, "lse": lse}


def _exact_attn(case, s):
    H, kv, dh, T = case["heads"], case["kv"], case["dh"], s["q"].shape[0]
    new = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out, lse, dq, dk, dv = new(T, H, dh), new(H, T), new(T, H, dh), new(T, kv, dh), new(T, kv, dh)
    bwd, a = case["how"] == "bwd", 0
    for n in s["lengths"].tolist():
        hidden = torch.arange(n, device="cuda")[None, :] > torch.arange(n, device="cuda")[:, None]
        for h in range(H):
            j, r = h * kv // H, slice(a, a + n)
            q, k, v = s["q"][r, h].double() / math.sqrt(dh), s["k"][r, j].double(), s["v"][r, j].double()
            z = torch.matmul(q, k.t().contiguous()).masked_fill_(hidden, -math.inf)
            lse[h, r] = torch.logsumexp(z, 1)
            p = z.sub_(lse[h, r, None]).exp_()
            out[r, h] = torch.matmul(p, v)
            if bwd:
                g = s["dout"][r, h].double()
                dv[r, j] += torch.matmul(p.t().contiguous(), g)
                ds = p * (torch.matmul(g, v.t().contiguous()) - (g * out[r, h]).sum(1, keepdim=True))
                dq[r, h] = torch.matmul(ds, k) / math.sqrt(dh)
                dk[r, j] += torch.matmul(ds.t().contiguous(), q)
        a += n
    return {"dq": dq, "dk": dk, "dv": dv} if bwd else {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        at = s["positions"] if case["how"] == "fwd" else -s["positions"]
        return {"out": _exact_rotated(s["x"], s["freqs"], at, s["amplitude"], case["layout"])}
    return {"append": _exact_append, "decode": _exact_decode, "attn": _exact_attn}[case["kind"]](case, s)
