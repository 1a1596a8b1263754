"""torch-facing wrappers of the C ABI (buffers from torch, compute in the library).

`Jagged` holds the per-batch metadata on the device; the functions below
allocate outputs and workspace with torch and call the C entry points on the
current stream.  Nothing here computes any part of the method.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import torch

from . import hstu


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return hstu.MTGR_DTYPE_BF16
    if t.dtype == torch.float32:
        return hstu.MTGR_DTYPE_FP32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _token_stride(t: torch.Tensor, inner: int) -> int:
    """Token stride of a [T, H, dh] or [T, d] view whose inner dims are dense."""
    st, sh = t.stride(), t.shape
    if len(st) == 3:
        if st[2] != 1 or st[1] != sh[2]:
            raise ValueError("head and feature dims must be dense")
    elif len(st) == 2:
        if st[1] != 1:
            raise ValueError("feature dim must be dense")
    if sh[0] <= 1:
        return inner
    return st[0]


def _like_layout(t: torch.Tensor) -> torch.Tensor:
    """Uninitialised tensor with the same shape and strides as `t` (gradients share the
    token stride of their primal, e.g. column slices of one fused projection)."""
    return torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device)


@dataclass
class Jagged:
    """Device metadata of a jagged batch of users: offsets [B+1] int32, seg [T] int8, ts [T] int32."""
    offsets: torch.Tensor
    seg: torch.Tensor
    ts: torch.Tensor
    max_seqlen: int

    @property
    def num_users(self) -> int:
        return self.offsets.numel() - 1

    @property
    def total_tokens(self) -> int:
        return self.seg.numel()

    @staticmethod
    def from_host(offsets, seg, ts, device="cuda") -> "Jagged":
        off = torch.as_tensor(offsets).to(torch.int32)
        lens = off[1:] - off[:-1]
        max_len = int(lens.max()) if lens.numel() else 0
        return Jagged(off.to(device), torch.as_tensor(seg).to(torch.int8).to(device),
                      torch.as_tensor(ts).to(torch.int32).to(device), max_len)


def attn_problem(jag: Jagged, q, k, v, out, rab=None, alpha: float = 1.0,
                 flags: int = 0) -> hstu.HstuProblem:
    T, H, dh = q.shape
    row = H * dh
    nb = 0 if rab is None else rab.shape[1]
    # (a tensor given for several arguments, as by attn_plan, has one stride)
    lq = _token_stride(q, row)
    lk = lq if k is q else _token_stride(k, row)
    lv = lk if v is k else _token_stride(v, row)
    lo = lq if out is q else _token_stride(out, row)
    return hstu.HstuProblem(jag.num_users, jag.max_seqlen, T, H, dh, _dtype_code(q), alpha, nb, flags,
                            lq or row, lk or row, lv or row, lo or row)


def validate_batch(jag: Jagged, group_ids=None, num_groups: int = 0, scratch=None) -> None:
    """Debugging aid (synchronises): checks offsets, seg and optional group ids on the device
    through mtgr_debug_validate_inputs; raises hstu.MtgrError naming the first bad index."""
    p = hstu.attn_problem(jag.num_users, jag.total_tokens, jag.max_seqlen, 1, 16)
    if scratch is None:
        scratch = torch.empty(hstu.MTGR_VALIDATE_SCRATCH_BYTES, dtype=torch.uint8, device=jag.offsets.device)
    hstu.mtgr_debug_validate_inputs(p, jag.offsets, jag.seg, group_ids, num_groups, scratch, scratch.numel())


def attn_plan(q, jag: Jagged, workspace=None, rab=None, backward: bool = False):
    """Builds the batch plan (tile summaries + work list) once; pass the returned workspace
    with planned=True to attn_fwd / attn_bwd for every layer on the same batch.  backward=True
    allocates the larger workspace with which the backward stores dS instead of recomputing."""
    p = attn_problem(jag, q, q, q, q, rab)
    if workspace is None:
        workspace = workspace_for(p, q.device, backward)
    hstu.mtgr_hstu_attn_plan(p, jag.offsets, jag.seg, jag.ts, workspace, workspace.numel())
    return workspace


def workspace_for(problem: hstu.HstuProblem, device, backward: bool = False) -> torch.Tensor:
    n = hstu.mtgr_hstu_attn_workspace_size(problem, backward)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def attn_fwd(q, k, v, jag: Jagged, rab=None, alpha: float = 1.0, out=None, workspace=None,
             planned: bool = False, cand_rows: bool = False):
    """Eq. 5 forward: returns out [T, H, dh] (same dtype as q).  cand_rows=True forms only the
    candidate tokens' rows (the other rows of `out` are left as they were).

    A row's fp32 sums are in an order that the batch's sizes decide (total tokens, users, heads, and
    jag.max_seqlen), so the same user can differ in a result's last bit between batches."""
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    flags = (hstu.MTGR_ATTN_PLANNED if planned else 0) | (hstu.MTGR_FWD_CAND_ROWS if cand_rows else 0)
    p = attn_problem(jag, q, k, v, out, rab, alpha, flags)
    if workspace is None:
        workspace = workspace_for(p, q.device)
    hstu.mtgr_hstu_attn_fwd(p, jag.offsets, jag.seg, jag.ts, q, k, v, rab, out, workspace,
                            workspace.numel())
    return out


@dataclass
class UserCache:
    """The user-side tokens (U | S | R) of a batch of users held across serving requests: their
    layout, this layer's keys and values [Tc, H, dh], and the cache's plan (tile summaries and
    token codes, built once by user_cache())."""
    jag: Jagged
    k: torch.Tensor
    v: torch.Tensor
    plan: torch.Tensor


def user_cache(k, v, jag: Jagged) -> UserCache:
    """Plans a user-side cache (mtgr_hstu_attn_plan on its layout) for attn_fwd_cached."""
    return UserCache(jag, k, v, attn_plan(k, jag))


def attn_fwd_cached(q, k, v, jag: Jagged, cache: UserCache, rab=None, alpha: float = 1.0, out=None,
                    workspace=None, planned: bool = False):
    """Candidate rows of a request (q, k, v, jag: the candidates) against the users' cached
    user-side keys and values (mtgr_hstu_attn_fwd_cached).  Returns out [Tq, H, dh]."""
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    p = attn_problem(jag, q, k, v, out, rab, alpha, hstu.MTGR_ATTN_PLANNED if planned else 0)
    pc = attn_problem(cache.jag, cache.k, cache.k, cache.v, cache.k)
    if workspace is None:
        workspace = workspace_for(p, q.device)
    hstu.mtgr_hstu_attn_fwd_cached(p, jag.offsets, jag.seg, jag.ts, q, k, v, rab, out, pc, cache.jag.offsets,
                                   cache.jag.ts, cache.k, cache.v, cache.plan, cache.plan.numel(), workspace,
                                   workspace.numel())
    return out


def attn_bwd(q, k, v, dout, jag: Jagged, rab=None, alpha: float = 1.0, need_drab: bool = True,
             grads=None, workspace=None, planned: bool = False, parts: str = "all", act=None):
    """Backward of Eq. 5: returns (dq, dk, dv, drab-or-None).

    parts: "all"; "dq" or "dkdv" (one side only); or the two halves of the stored-dS path as
    two calls on one backward-size workspace: "dkdv_keep_ds" (dk, dv, drab and the dS blocks)
    then "dq_from_ds" (dq from them; drab is not formed again).

    act = (h, bias), h [T, 3 H dh] as q | k | v: q, k, v are silu(h + bias), and the gradients returned
    are those of h (bf16, head_dim >= 32)."""
    flags = (hstu.MTGR_ATTN_PLANNED if planned else 0) | {
        "all": 0, "dq": hstu.MTGR_BWD_SKIP_DKDV, "dkdv": hstu.MTGR_BWD_SKIP_DQ,
        "dkdv_keep_ds": hstu.MTGR_BWD_SKIP_DQ | hstu.MTGR_BWD_KEEP_DS,
        "dq_from_ds": hstu.MTGR_BWD_SKIP_DKDV | hstu.MTGR_BWD_DS_READY}[parts]
    if parts == "dq_from_ds":
        need_drab = False
    if grads is None:
        dq, dk, dv = (_like_layout(x) for x in (q, k, v))
        drab = torch.empty_like(rab) if (rab is not None and need_drab) else None
    else:
        dq, dk, dv, drab = grads
        if not need_drab:
            drab = None
    p = attn_problem(jag, q, k, v, dout, rab, alpha, flags)
    row = q.shape[1] * q.shape[2]
    if _token_stride(dq, row) != p.ld_q or _token_stride(dk, row) != p.ld_k or _token_stride(dv, row) != p.ld_v:
        raise ValueError("gradients must share the layout of q, k, v")
    if workspace is None:
        workspace = workspace_for(p, q.device, backward=True)
    if act is not None:
        h, bias = act
        if h.shape != (q.shape[0], 3 * row) or h.dtype != q.dtype or \
                (bias is not None and (bias.shape != (3 * row,) or bias.dtype != torch.float32 or not bias.is_contiguous())):
            raise ValueError("act: h is [T, 3 H dh] of the type of q, bias [3 H dh] fp32")
        hstu.mtgr_hstu_attn_bwd_act(p, jag.offsets, jag.seg, jag.ts, q, k, v, rab, dout, h, _token_stride(h, 3 * row),
                                    bias, dq, dk, dv, drab, workspace, workspace.numel())
        return dq, dk, dv, drab
    hstu.mtgr_hstu_attn_bwd(p, jag.offsets, jag.seg, jag.ts, q, k, v, rab, dout, dq, dk, dv, drab,
                            workspace, workspace.numel())
    return dq, dk, dv, drab


def gln_fwd(x, u, group_ids, gamma, beta, eps: float = 1e-5, y=None, stats=None):
    """Gate + Group-LN forward: returns (y, mean, rstd)."""
    T, d = x.shape
    if y is None:
        y = torch.empty((T, d), dtype=x.dtype, device=x.device)
    if stats is None:
        mean = torch.empty(T, dtype=torch.float32, device=x.device)
        rstd = torch.empty(T, dtype=torch.float32, device=x.device)
    else:
        mean, rstd = stats
    p = hstu.gln_problem(T, d, gamma.shape[0], _dtype_code(x), eps, _token_stride(x, d),
                         _token_stride(u, d) if u is not None else d, _token_stride(y, d))
    hstu.mtgr_group_layernorm_fwd(p, x, u, group_ids, gamma, beta, y, mean, rstd)
    return y, mean, rstd


def gln_bwd(dy, x, u, group_ids, gamma, mean, rstd, eps: float = 1e-5, grads=None, workspace=None,
            residual=None):
    """Gate + Group-LN backward: returns (dx, du-or-None, dgamma, dbeta).  `residual` (only without
    a gate) is added to dx before its rounding."""
    if residual is not None and u is not None:
        raise ValueError("a residual goes with the Group-LN without a gate")
    T, d = x.shape
    if grads is None:
        dx = _like_layout(x)
        du = _like_layout(u) if u is not None else None
        dgamma = torch.empty_like(gamma)
        dbeta = torch.empty_like(gamma)
    else:
        dx, du, dgamma, dbeta = grads
    p = hstu.gln_problem(T, d, gamma.shape[0], _dtype_code(x), eps, _token_stride(x, d),
                         _token_stride(residual if u is None else u, d) if u is not None or residual is not None else d,
                         _token_stride(dy, d))
    if _token_stride(dx, d) != p.ld_x or (du is not None and _token_stride(du, d) != p.ld_u):
        raise ValueError("gradients must share the layout of x, u")
    if workspace is None:
        n = hstu.mtgr_group_layernorm_workspace_size(p, True)
        workspace = torch.empty(max(n, 256), dtype=torch.uint8, device=x.device)
    if residual is not None:
        if residual.shape != x.shape or residual.dtype != x.dtype:
            raise ValueError("the residual has the shape and type of x")
        hstu.mtgr_group_layernorm_bwd_add(p, dy, x, residual, group_ids, gamma, mean, rstd, dx, dgamma, dbeta,
                                          workspace, workspace.numel())
        return dx, None, dgamma, dbeta
    hstu.mtgr_group_layernorm_bwd(p, dy, x, u, group_ids, gamma, mean, rstd, dx, du, dgamma, dbeta,
                                  workspace, workspace.numel())
    return dx, du, dgamma, dbeta


def gln_workspace(x, groups: int) -> torch.Tensor:
    T, d = x.shape
    p = hstu.gln_problem(T, d, groups, _dtype_code(x))
    n = hstu.mtgr_group_layernorm_workspace_size(p, True)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=x.device)


_GEMM_LAYOUTS = {"nn": hstu.MTGR_GEMM_NN, "nt": hstu.MTGR_GEMM_NT, "tn": hstu.MTGR_GEMM_TN}


def _row_ld(t: torch.Tensor) -> int:
    if t.dim() != 2 or t.dtype != torch.bfloat16 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("GEMM operands are 2-D bf16 with a dense inner dim")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def gemm(a, b, layout: str = "nn", out=None, bias=None, residual=None, silu_out=None, colsum=None,
         workspace=None):
    """bf16 product through mtgr_gemm_bf16: 'nn' a @ b, 'nt' a @ b.T, 'tn' a.T @ b, with the
    encoder layer's fused epilogues (bias + SiLU into `silu_out`, or bias + residual) and, for
    'tn', the fp32 column sums of b into `colsum`.  Returns `out`."""
    lay = _GEMM_LAYOUTS[layout]
    if layout == "nn":
        (M, K), N = a.shape, b.shape[1]
    elif layout == "nt":
        (M, K), N = a.shape, b.shape[0]
    else:
        (K, M), N = a.shape, b.shape[1]
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=a.device)
    epi = hstu.MTGR_GEMM_EPI_NONE
    if silu_out is not None:
        epi = hstu.MTGR_GEMM_EPI_BIAS_SILU
    elif residual is not None:
        epi = hstu.MTGR_GEMM_EPI_BIAS_RESIDUAL
    ws_bytes = 0
    if layout == "tn":
        ws_bytes = hstu.mtgr_gemm_workspace_size(lay, M, N, K)
        if workspace is None or workspace.numel() < ws_bytes:
            workspace = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device=a.device)
        ws_bytes = workspace.numel()
    hstu.mtgr_gemm_bf16(lay, M, N, K, a, _row_ld(a), b, _row_ld(b), out, _row_ld(out), epi, bias,
                        residual, _row_ld(residual) if residual is not None else 0, silu_out,
                        _row_ld(silu_out) if silu_out is not None else 0, colsum, workspace, ws_bytes)
    return out


def add(a, b, out=None):
    """out = a + b through mtgr_add (2-D, dense inner dim)."""
    if out is None:
        out = torch.empty_like(a)
    rows, cols = a.shape
    hstu.mtgr_add(rows, cols, _dtype_code(a), a, _token_stride(a, cols), b, _token_stride(b, cols), out,
                  _token_stride(out, cols))
    return out


# ------------------------------------------------------------------ feed-forward block, dropout, softmax loss

def _device() -> int:
    """The current device; the operands below have to be on it (the stream is its current one)."""
    return torch._C._cuda_getDevice() if torch.cuda.is_initialized() else -2     # (no tensor's device number)


def _matrix(name: str, t, rows: int, cols: int, dtype, dev: int, like: Optional[int] = None) -> int:
    """Checks a 2-D operand (shape, type, device, dense rows that do not overlap) and returns its row stride;
    `like`: the row stride that a gradient shares with its primal."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != (rows, cols):
        got = f"{list(t.shape)} {t.dtype}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise ValueError(f"{name} is [{rows}, {cols}] of {dtype}, got {got}")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, not on the current device")
    ld, inner = t.stride()
    if inner != 1 and cols > 1:
        raise ValueError(f"the rows of {name} are not dense")
    if rows <= 1:
        ld = cols
    elif ld < cols:
        raise ValueError(f"the rows of {name} overlap")
    if like is not None and ld != like:
        raise ValueError(f"{name} must share the row stride of its primal")
    return ld


def _vector(name: str, t, n: int, dtypes, dev: int) -> None:
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} is a dense [{n}] of {' or '.join(str(d) for d in dtypes)}")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, not on the current device")


def _scratch(workspace, need: int, like) -> torch.Tensor:
    """The caller's workspace, or a new one of at least `need` bytes beside the operand `like`."""
    if workspace is None:
        return torch.empty(max(need, 256), dtype=torch.uint8, device=like.device)
    if workspace.dtype is not torch.uint8 or not workspace.is_contiguous() or workspace.get_device() != like.get_device():
        raise ValueError("a workspace is a dense uint8 tensor on the device of the operands")
    return workspace


def _two_dims(name: str, t):
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} is a matrix")
    return t.shape


def gated_ffn_problem(tokens: int, dim: int, hidden: int, ld_x=None, ld_w_in=None, ld_w_out=None, ld_y=None, ld_r=None,
                      ld_pre=None, ld_h=None) -> hstu.GatedFfnProblem:
    return hstu.GatedFfnProblem(tokens, dim, hidden, ld_x or dim, ld_w_in or 2 * hidden, ld_w_out or dim, ld_y or dim,
                                ld_r or dim, ld_pre or 2 * hidden, ld_h or hidden)


def gated_ffn_workspace(tokens: int, dim: int, hidden: int, device="cuda", backward: bool = False) -> torch.Tensor:
    """A workspace for gated_ffn_fwd (with save or without) or gated_ffn_bwd of these sizes."""
    n = hstu.mtgr_gated_ffn_workspace_size(gated_ffn_problem(tokens, dim, hidden),
                                           hstu.MTGR_FFN_BACKWARD if backward else hstu.MTGR_FFN_SERVING)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def gated_ffn_fwd(x, w_in, w_out, residual=None, save: bool = False, out=None, workspace=None):
    """y = (silu(x W_gate) * (x W_up)) W_out (+ residual), bf16: x [T, d], w_in [d, 2f] = gate | up columns,
    w_out [f, d]; d and f multiples of 32.  Returns y, or with save=True (y, pre [T, 2f], h [T, f]), the last two
    for gated_ffn_bwd."""
    (T, d), f = _two_dims("x", x), _two_dims("w_out", w_out)[0]
    bf, dev = torch.bfloat16, _device()
    if out is None:
        out = torch.empty((T, d), dtype=bf, device=x.device)
    pre = torch.empty((T, 2 * f), dtype=bf, device=x.device) if save else None
    h = torch.empty((T, f), dtype=bf, device=x.device) if save else None
    p = hstu.GatedFfnProblem(T, d, f, _matrix("x", x, T, d, bf, dev), _matrix("w_in", w_in, d, 2 * f, bf, dev),
                             _matrix("w_out", w_out, f, d, bf, dev), _matrix("out", out, T, d, bf, dev),
                             _matrix("residual", residual, T, d, bf, dev) if residual is not None else d, 2 * f, f)
    need = hstu.mtgr_gated_ffn_workspace_size(p, hstu.MTGR_FFN_TRAINING if save else hstu.MTGR_FFN_SERVING)
    workspace = _scratch(workspace, need, x)
    hstu.mtgr_gated_ffn_fwd(p, x, w_in, w_out, residual, out, pre, h, workspace, workspace.numel())
    return (out, pre, h) if save else out


def gated_ffn_bwd(dy, x, pre, h, w_in, w_out, grads=None, workspace=None):
    """Gradients of gated_ffn_fwd: (dx, dw_in, dw_out), in the layouts of x, w_in and w_out (`grads`: the tensors to
    write).  A residual's gradient is dy itself."""
    (T, d), f = _two_dims("x", x), _two_dims("w_out", w_out)[0]
    bf, dev = torch.bfloat16, _device()
    dx, dw_in, dw_out = grads if grads is not None else (_like_layout(t) for t in (x, w_in, w_out))
    p = hstu.GatedFfnProblem(T, d, f, _matrix("x", x, T, d, bf, dev), _matrix("w_in", w_in, d, 2 * f, bf, dev),
                             _matrix("w_out", w_out, f, d, bf, dev), _matrix("dy", dy, T, d, bf, dev), d,
                             _matrix("pre", pre, T, 2 * f, bf, dev), _matrix("h", h, T, f, bf, dev))
    _matrix("dx", dx, T, d, bf, dev, p.ld_x)
    _matrix("dw_in", dw_in, d, 2 * f, bf, dev, p.ld_w_in)
    _matrix("dw_out", dw_out, f, d, bf, dev, p.ld_w_out)
    workspace = _scratch(workspace, hstu.mtgr_gated_ffn_workspace_size(p, hstu.MTGR_FFN_BACKWARD), x)
    hstu.mtgr_gated_ffn_bwd(p, dy, x, pre, h, w_in, w_out, dx, dw_in, dw_out, workspace, workspace.numel())
    return dx, dw_in, dw_out


def dropout(x, p: float, rng, site: int = 0, residual=None, out=None):
    """[residual +] dropout(x) of a [rows, cols] matrix, bf16 or fp32.  The mask follows from rng (a device int64 [2]:
    seed, step), `site` and the element alone and is not stored: the backward pass is dropout(dout, p, rng, site)
    with the same rng.  A program advances the step between its steps (rng[1] += 1)."""
    rows, cols = _two_dims("x", x)
    code, dt, dev = _dtype_code(x), x.dtype, _device()
    if out is None:
        out = torch.empty((rows, cols), dtype=dt, device=x.device)
    ld_x, ld_out = _matrix("x", x, rows, cols, dt, dev), _matrix("out", out, rows, cols, dt, dev)
    ld_r = _matrix("residual", residual, rows, cols, dt, dev) if residual is not None else cols
    _vector("rng", rng, 2, (torch.int64,), dev)
    if not 0 <= site < 1 << 32:
        raise ValueError("site is a 32-bit number")
    hstu.mtgr_dropout(rows, cols, code, x, ld_x, p, rng, site, residual, ld_r, out, ld_out)
    return out


def _softmax_loss_problem(x, w, targets, bias, scale: float) -> hstu.SoftmaxLossProblem:
    (N, d), V = _two_dims("x", x), _two_dims("w", w)[0]
    dev = _device()
    ld_x, ld_w = _matrix("x", x, N, d, torch.bfloat16, dev), _matrix("w", w, V, d, torch.bfloat16, dev)
    _vector("targets", targets, N, (torch.int64, torch.int32), dev)
    if bias is not None:
        _vector("bias", bias, V, (torch.float32,), dev)
    return hstu.SoftmaxLossProblem(N, V, d, 64 if targets.dtype == torch.int64 else 32, scale, ld_x, ld_w)


def softmax_loss_workspace(rows: int, classes: int, dim: int, device="cuda", backward: bool = False) -> torch.Tensor:
    """A workspace for softmax_loss_fwd or softmax_loss_bwd of these sizes."""
    p = hstu.SoftmaxLossProblem(rows, classes, dim, 64, 1.0, dim, dim)
    n = hstu.mtgr_softmax_loss_workspace_size(p, backward)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def softmax_loss_fwd(x, w, targets, bias=None, scale: float = 1.0, workspace=None):
    """Softmax cross entropy of the rows of x [N, d] against the classes w [V, d] (bf16), with the logits
    z = scale x w^T + bias (bias [V] fp32), which are never kept: (loss [N], lse [N]) fp32.  A row whose target lies
    outside 0 .. V-1 has no label: loss and lse 0.  A bias of -inf (or below -2.36e38) takes a class out."""
    p = _softmax_loss_problem(x, w, targets, bias, scale)
    loss = torch.empty(p.num_rows, dtype=torch.float32, device=x.device)
    lse = torch.empty_like(loss)
    workspace = _scratch(workspace, hstu.mtgr_softmax_loss_workspace_size(p), x)
    hstu.mtgr_softmax_loss_fwd(p, x, w, targets, bias, loss, lse, workspace, workspace.numel())
    return loss, lse


def softmax_loss_bwd(dloss, x, w, targets, lse, bias=None, scale: float = 1.0, grads=None, workspace=None):
    """Gradients of softmax_loss_fwd for dloss [N] fp32 (that of the mean over n labels: 1 / n) and the forward's lse:
    (dx, dw, dbias or None), dx and dw in the layouts of x and w (`grads`: the tensors to write)."""
    p = _softmax_loss_problem(x, w, targets, bias, scale)
    dev = x.get_device()
    _vector("dloss", dloss, p.num_rows, (torch.float32,), dev)
    _vector("lse", lse, p.num_rows, (torch.float32,), dev)
    if grads is None:
        grads = _like_layout(x), _like_layout(w), torch.empty_like(bias) if bias is not None else None
    dx, dw, dbias = grads
    _matrix("dx", dx, *x.shape, torch.bfloat16, dev, p.ld_x)
    _matrix("dw", dw, *w.shape, torch.bfloat16, dev, p.ld_w)
    if dbias is not None:
        _vector("dbias", dbias, p.num_classes, (torch.float32,), dev)
    workspace = _scratch(workspace, hstu.mtgr_softmax_loss_workspace_size(p, True), x)
    hstu.mtgr_softmax_loss_bwd(p, dloss, x, w, targets, bias, lse, dx, dw, dbias, workspace, workspace.numel())
    return dx, dw, dbias


# ------------------------------------------------------------------ rotary positions, causal attention, paged cache

# (The checks below run on every call and are a large part of its host time, so their way to success is short and what is
# wrong is said elsewhere.)

def _refuse(name: str, t, what: str):
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} is {what}, got {type(t).__name__}")
    raise ValueError(f"{name} is {what} on the current device, got {list(t.shape)} of {t.dtype}, strides {list(t.stride())}, on {t.device}")


def _heads(name: str, t, tokens: Optional[int], heads: Optional[int], dh: Optional[int], dtype, dev: int,
           like: Optional[int] = None) -> int:
    """Checks a [tokens, heads, head_dim] operand (shape, type, device, dense heads, token rows that do not overlap) and
    returns its token stride; None: any size; `like`: the stride that a gradient shares with its primal."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.dim() == 3 and t.get_device() == dev:
        n, h, d = t.shape
        ld, sh, se = t.stride()
        if (tokens is None or n == tokens) and (heads is None or h == heads) and (dh is None or d == dh) and \
                (se == 1 or d <= 1) and (sh == d or h <= 1):
            if n <= 1:
                ld = h * d
            if ld >= h * d and (like is None or ld == like):
                return ld
            _refuse(name, t, "rows that do not overlap" if like is None else "of the token stride of its primal")
    _refuse(name, t, f"[{tokens or 'tokens'}, {heads or 'heads'}, {dh or 'head_dim'}] of {dtype} with dense heads")


def _int32(name: str, t, n: int, dev: int) -> None:
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.int32 and t.get_device() == dev and t.dim() == 1 and
            t.shape[0] == n and t.is_contiguous()):
        _refuse(name, t, f"a dense [{n}] of int32")


def _sequences(offsets, dev: int) -> int:
    if not (isinstance(offsets, torch.Tensor) and offsets.dtype is torch.int32 and offsets.get_device() == dev and
            offsets.dim() == 1 and offsets.shape[0] >= 1 and offsets.is_contiguous()):
        _refuse("offsets", offsets, "a dense [B + 1] of int32")
    return offsets.shape[0] - 1


def _lse(t, rows: int, cols: int, dev: int) -> None:
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.float32 and t.get_device() == dev and t.shape == (rows, cols) and
            t.is_contiguous()):
        _refuse("lse", t, f"a dense [{rows}, {cols}] of fp32")


@dataclass
class Rotary:
    """Rotary positions: pair i of a head turns by freqs[i] (radians, device float64 [rot_dim / 2]) per position, and is
    multiplied by `amplitude`.  layout "half" pairs feature i with i + rot_dim / 2, "interleaved" 2 i with 2 i + 1; features
    behind rot_dim are kept."""
    freqs: torch.Tensor
    layout: str = "half"
    amplitude: float = 1.0

    def code(self, dev: int) -> int:
        f = self.freqs
        if not (isinstance(f, torch.Tensor) and f.dtype is torch.float64 and f.get_device() == dev and f.dim() == 1 and
                f.is_contiguous()):
            _refuse("freqs", f, "a dense [rot_dim / 2] of float64")
        if self.layout == "half":
            return hstu.MTGR_ROPE_HALF
        if self.layout == "interleaved":
            return hstu.MTGR_ROPE_INTERLEAVED
        raise ValueError(f"layout {self.layout!r} is neither 'half' nor 'interleaved'")


_ROPE_SCALINGS = {"none": hstu.MTGR_ROPE_NONE, "linear": hstu.MTGR_ROPE_LINEAR, "base": hstu.MTGR_ROPE_BASE,
                  "parts": hstu.MTGR_ROPE_PARTS}


def rotary(rot_dim: int, base: float = 10000.0, layout: str = "half", scaling: str = "none", factor: float = 1.0,
           trained_len: int = 0, slow: float = 1.0, fast: float = 32.0, device="cuda") -> Rotary:
    """Rotary positions of the first rot_dim features (a multiple of 16) with frequencies base^(-2 i / rot_dim), stretched
    for contexts `factor` times the trained ones by `scaling`: "linear", "base" or "parts" (mtgr_rope_frequencies)."""
    if scaling not in _ROPE_SCALINGS:
        raise ValueError(f"scaling {scaling!r} is none of {', '.join(_ROPE_SCALINGS)}")
    freqs, amplitude = hstu.mtgr_rope_frequencies(rot_dim, base, _ROPE_SCALINGS[scaling], factor, trained_len, slow, fast)
    return Rotary(torch.tensor(freqs, dtype=torch.float64, device=device), layout, amplitude)


def rope(x, rotary: Rotary, positions=None, offsets=None, inverse: bool = False, out=None):
    """x [T, heads, head_dim] (bf16 or fp32) with its heads rotated by their tokens' positions: `positions` [T] int32, or
    those inside each sequence of `offsets` [B + 1] int32 (rows behind the last are left).  inverse=True turns back: the
    gradient of x.  out may be x."""
    code, dev = _dtype_code(x), _device()
    dtype = x.dtype
    ld_x = _heads("x", x, None, None, None, dtype, dev)
    T, H, dh = x.shape
    if out is None:
        out, ld_out = x.new_empty((T, H, dh)), H * dh
    else:
        ld_out = _heads("out", out, T, H, dh, dtype, dev)
    layout = rotary.code(dev)
    if (positions is None) == (offsets is None):
        raise ValueError("either positions or offsets is given")
    B = 0
    if positions is not None:
        _int32("positions", positions, T, dev)
    else:
        B = _sequences(offsets, dev)
    p = hstu.RopeProblem(T, B, H, dh, 2 * rotary.freqs.numel(), layout, code, inverse, rotary.amplitude, ld_x, ld_out)
    hstu.mtgr_rope(p, x, positions, offsets, rotary.freqs, out)
    return out


def _causal_problem(q, k, v, offsets, scale, dev: int) -> hstu.CausalProblem:
    bf = torch.bfloat16
    ld_q = _heads("q", q, None, None, None, bf, dev)
    T, H, dh = q.shape
    ld_k = _heads("k", k, T, None, dh, bf, dev)
    Hk = k.shape[1]
    ld_v = _heads("v", v, T, Hk, dh, bf, dev)
    return hstu.CausalProblem(_sequences(offsets, dev), H, Hk, dh, T, dh ** -0.5 if scale is None else scale, 0, ld_q, ld_k,
                              ld_v, H * dh, H * dh)


def causal_attn_fwd(q, k, v, offsets, scale: Optional[float] = None, save: bool = False, out=None, lse=None):
    """Causal softmax attention of packed sequences (bf16): q [T, heads, head_dim], k and v [T, kv_heads, head_dim], heads a
    multiple of kv_heads, offsets [B + 1] int32 (a Jagged's offsets); scale: 1 / sqrt(head_dim) by default.  Returns out
    [T, heads, head_dim], or with save=True (out, lse [heads, T] fp32) for causal_attn_bwd.  Rows behind the last sequence are
    left as they were."""
    dev = _device()
    p = _causal_problem(q, k, v, offsets, scale, dev)
    T, H, dh = q.shape
    if out is None:
        out = q.new_empty((T, H, dh))
    else:
        p.ld_o = _heads("out", out, T, H, dh, torch.bfloat16, dev)
    if lse is not None:
        _lse(lse, H, T, dev)
    elif save:
        lse = torch.empty((H, T), dtype=torch.float32, device=q.device)
    hstu.mtgr_causal_attn_fwd(p, offsets, q, k, v, out, lse)
    return (out, lse) if save else out


def causal_attn_workspace(q, k, offsets) -> torch.Tensor:
    """A workspace for causal_attn_bwd of up to so many tokens and sequences."""
    n = hstu.mtgr_causal_attn_workspace_size(_causal_problem(q, k, k, offsets, None, _device()))
    return torch.empty(max(n, 256), dtype=torch.uint8, device=q.device)


def causal_attn_bwd(dout, q, k, v, out, lse, offsets, scale: Optional[float] = None, grads=None, workspace=None):
    """Gradients of causal_attn_fwd for dout, with its out and lse: (dq, dk, dv), in the layouts of q, k and v (`grads`: the
    tensors to write).  Rows behind the last sequence are left as they were."""
    bf, dev = torch.bfloat16, _device()
    p = _causal_problem(q, k, v, offsets, scale, dev)
    p.ld_o, p.ld_do = _heads("out", out, *q.shape, bf, dev), _heads("dout", dout, *q.shape, bf, dev)
    _lse(lse, q.shape[1], q.shape[0], dev)
    dq, dk, dv = grads if grads is not None else (_like_layout(t) for t in (q, k, v))
    _heads("dq", dq, *q.shape, bf, dev, p.ld_q)
    _heads("dk", dk, *k.shape, bf, dev, p.ld_k)
    _heads("dv", dv, *v.shape, bf, dev, p.ld_v)
    workspace = _scratch(workspace, hstu.mtgr_causal_attn_workspace_size(p), q)
    hstu.mtgr_causal_attn_bwd(p, offsets, q, k, v, out, lse, dout, dq, dk, dv, workspace, workspace.numel())
    return dq, dk, dv


@dataclass
class KvCache:
    """A paged cache of keys and values, bf16 [num_pages, kv_heads, page_size, head_dim] each: token p of a sequence lies in
    row p % page_size of page page_table[sequence, p // page_size]."""
    keys: torch.Tensor
    values: torch.Tensor

    @staticmethod
    def empty(num_pages: int, kv_heads: int, page_size: int, head_dim: int, device="cuda") -> "KvCache":
        keys = torch.empty((num_pages, kv_heads, page_size, head_dim), dtype=torch.bfloat16, device=device)
        return KvCache(keys, torch.empty_like(keys))

    def struct(self, dev: int) -> hstu.KvCachePages:
        k, v = self.keys, self.values
        for name, t in (("keys", k), ("values", v)):
            if not (isinstance(t, torch.Tensor) and t.dtype is torch.bfloat16 and t.get_device() == dev and t.dim() == 4 and
                    t.is_contiguous()):
                _refuse(name, t, "a cache's dense [num_pages, kv_heads, page_size, head_dim] of bf16")
        n, h, size, dh = shape = k.shape
        if v.shape != shape:
            raise ValueError(f"keys {list(k.shape)} and values {list(v.shape)} of the cache differ")
        return hstu.KvCachePages(n, size, h, dh, 0, k.data_ptr(), v.data_ptr())


def _page_table(t, dev: int):
    """(num_seqs, max_pages, row stride) of a page table."""
    if isinstance(t, torch.Tensor) and t.dtype is torch.int32 and t.get_device() == dev and t.dim() == 2:
        B, n = t.shape
        ld, inner = t.stride()
        if B <= 1:
            ld = n
        if ld >= n and (inner == 1 or n <= 1):
            return B, n, ld
    _refuse("page_table", t, "[num_seqs, max_pages] of int32 with dense rows that do not overlap")


def kv_append(cache: KvCache, page_table, past, k, v, offsets=None, q=None, rotary: Optional[Rotary] = None, q_out=None):
    """Appends new tokens to a paged cache: rows offsets[b] .. offsets[b + 1] - 1 of k and v [N, kv_heads, head_dim] (without
    offsets: row b) become tokens past[b], past[b] + 1, .. of sequence b.  With `rotary`, k is rotated on the way by its
    position in the sequence, and q [N, heads, head_dim] by the same; returns the rotated q (q_out, which may be q), or None
    without q.  past [B] int32; a sequence whose past is negative is left alone, with its rows of q_out, as are tokens past the
    columns of the page table."""
    bf, dev = torch.bfloat16, _device()
    c = cache.struct(dev)
    B, pages, ld_table = _page_table(page_table, dev)
    _int32("past", past, B, dev)
    Hk, dh = c.kv_heads, c.head_dim
    ld_k = _heads("k", k, None, Hk, dh, bf, dev)
    N = k.shape[0]
    ld_v = _heads("v", v, N, Hk, dh, bf, dev)
    if offsets is not None and _sequences(offsets, dev) != B:
        raise ValueError(f"offsets are those of {offsets.numel() - 1} sequences, page_table of {B}")
    H = ld_q = ld_q_out = 0
    if q is not None:
        ld_q = _heads("q", q, N, None, dh, bf, dev)
        H = q.shape[1]
        if q_out is None:
            q_out, ld_q_out = q.new_empty((N, H, dh)), H * dh
        else:
            ld_q_out = _heads("q_out", q_out, N, H, dh, bf, dev)
    elif q_out is not None:
        raise ValueError("q_out goes with q")
    rot, layout, amplitude, freqs = 0, 0, 1.0, None
    if rotary is not None:
        freqs = rotary.freqs
        layout, rot, amplitude = rotary.code(dev), 2 * freqs.numel(), rotary.amplitude
    p = hstu.KvAppendProblem(N, B, H, pages, rot, layout, amplitude, ld_table, ld_q, ld_q_out, ld_k, ld_v)
    hstu.mtgr_kv_append(p, c, page_table, past, offsets, q, k, v, freqs, q_out)
    return q_out


def cache_attn_workspace(cache: KvCache, num_seqs: int, heads: int, max_len: int) -> torch.Tensor:
    """A workspace for cache_attn of up to num_seqs sequences and any max_len up to this one."""
    c = cache.struct(_device())
    p = hstu.CacheAttnProblem(num_seqs, heads, -(-max(max_len, 1) // c.page_size), 1.0, max_len, 0, 0, 0)
    n = hstu.mtgr_cache_attn_workspace_size(p, c)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=cache.keys.device)


def cache_attn(q, cache: KvCache, page_table, lens, scale: Optional[float] = None, max_len: Optional[int] = None,
               save: bool = False, out=None, workspace=None):
    """One query token of each sequence, q [B, heads, head_dim] (bf16), against tokens 0 .. lens[b] - 1 of its cache: out
    [B, heads, head_dim], or with save=True (out, lse [B, heads] fp32).  lens [B] int32 on the device; max_len, their bound,
    should be tight (by default what the page table holds).  A sequence without tokens gets zeros and an lse of -inf."""
    bf, dev = torch.bfloat16, _device()
    c = cache.struct(dev)
    B, pages, ld_table = _page_table(page_table, dev)
    dh = c.head_dim
    ld_q = _heads("q", q, B, None, dh, bf, dev)
    H = q.shape[1]
    _int32("lens", lens, B, dev)
    if out is None:
        out, ld_o = q.new_empty((B, H, dh)), H * dh
    else:
        ld_o = _heads("out", out, B, H, dh, bf, dev)
    lse = torch.empty((B, H), dtype=torch.float32, device=q.device) if save else None
    p = hstu.CacheAttnProblem(B, H, pages, dh ** -0.5 if scale is None else scale,
                              pages * c.page_size if max_len is None else max_len, ld_table, ld_q, ld_o)
    need = hstu.mtgr_cache_attn_workspace_size(p, c)
    if need or workspace is not None:
        workspace = _scratch(workspace, need, q)
        need = workspace.numel()
    hstu.mtgr_cache_attn(p, c, page_table, lens, q, out, lse, workspace, need)
    return (out, lse) if save else out
