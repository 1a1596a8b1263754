"""Refusals of the feed-forward, dropout and softmax-loss entry points (include/mtgr_block.h) on the CPU: every
bad argument is a status before any device call.  Pointers are fake addresses that nothing reads."""
import ctypes

import pytest
import torch

from paper_2505_18654_amd import hstu, ops
from tests.block_ref import philox_words

FAKE = 0x7f0000000000
BIG = 1 << 40
NULL, INVALID, UNSUPPORTED, SMALL = (hstu.MTGR_ERROR_NULL_POINTER, hstu.MTGR_ERROR_INVALID_ARGUMENT,
                                     hstu.MTGR_ERROR_UNSUPPORTED, hstu.MTGR_ERROR_WORKSPACE_TOO_SMALL)


def status_of(call, *args, **kw):
    with pytest.raises(hstu.MtgrError) as e:
        call(*args, **kw)
    assert hstu.mtgr_last_error_message()
    return e.value.status


def test_struct_layouts():
    assert ctypes.sizeof(hstu.GatedFfnProblem) == 72 and hstu.GatedFfnProblem.ld_x.offset == 16
    assert ctypes.sizeof(hstu.SoftmaxLossProblem) == 48 and hstu.SoftmaxLossProblem.ld_x.offset == 32


# ------------------------------------------------------------------ gated feed-forward block

def ffn(**kw):
    base = dict(tokens=100, dim=64, hidden=96)
    strides = {k: kw.pop(k) for k in list(kw) if k.startswith("ld_")}
    base.update(kw)
    return ops.gated_ffn_problem(**base, **strides)


def ffn_fwd(p, **kw):
    a = dict(x=FAKE, w_in=FAKE, w_out=FAKE, residual=None, y=FAKE, pre=None, h=None, workspace=FAKE,
             workspace_bytes=BIG, stream=0)
    a.update(kw)
    hstu.mtgr_gated_ffn_fwd(p, **a)


def ffn_bwd(p, **kw):
    a = {n: FAKE for n in ("dy", "x", "pre", "h", "w_in", "w_out", "dx", "dw_in", "dw_out", "workspace")}
    a.update(workspace_bytes=BIG, stream=0)
    a.update(kw)
    hstu.mtgr_gated_ffn_bwd(p, **a)


@pytest.mark.parametrize("kw, status", [
    (dict(tokens=-1), INVALID), (dict(tokens=1 << 31), INVALID), (dict(dim=0), INVALID), (dict(hidden=-32), INVALID),
    (dict(dim=48), UNSUPPORTED), (dict(hidden=40), UNSUPPORTED), (dict(dim=1 << 20), UNSUPPORTED),
    (dict(tokens=1 << 30, hidden=4096), UNSUPPORTED),
    (dict(ld_x=56), INVALID), (dict(ld_x=68), INVALID), (dict(ld_x=1 << 22), UNSUPPORTED), (dict(ld_w_in=128), INVALID),
    (dict(ld_w_out=63), INVALID), (dict(ld_y=32), INVALID),
])
def test_ffn_problem_refused(kw, status):
    assert status_of(ffn_fwd, ffn(**kw)) == status
    assert status_of(ffn_bwd, ffn(**kw)) == status


@pytest.mark.parametrize("kw, status", [
    (dict(x=None), NULL), (dict(w_in=None), NULL), (dict(w_out=None), NULL), (dict(y=None), NULL),
    (dict(x=FAKE + 8), INVALID), (dict(y=FAKE + 2), INVALID), (dict(residual=FAKE + 4), INVALID),
    (dict(pre=FAKE), NULL), (dict(h=FAKE), NULL), (dict(pre=FAKE + 8, h=FAKE), INVALID),
    (dict(workspace=None), NULL), (dict(workspace=FAKE + 16), INVALID), (dict(workspace_bytes=100 * 96 * 2 - 1), SMALL),
])
def test_ffn_forward_refused(kw, status):
    assert status_of(ffn_fwd, ffn(), **kw) == status


@pytest.mark.parametrize("name", ["dy", "x", "pre", "h", "w_in", "w_out", "dx", "dw_in", "dw_out"])
def test_ffn_backward_refuses_each_matrix(name):
    assert status_of(ffn_bwd, ffn(), **{name: None}) == NULL
    assert status_of(ffn_bwd, ffn(), **{name: FAKE + 4}) == INVALID


def test_ffn_backward_workspace():
    need = hstu.mtgr_gated_ffn_workspace_size(ffn(), hstu.MTGR_FFN_BACKWARD)
    assert need >= 100 * 2 * 96 * 2
    assert status_of(ffn_bwd, ffn(), workspace_bytes=need - 1) == SMALL
    assert status_of(ffn_bwd, ffn(), workspace=None) == NULL


def test_ffn_null_problem_and_empty():
    L = hstu.lib()
    n = ctypes.c_size_t(7)
    assert L.mtgr_gated_ffn_workspace_size(None, 0, ctypes.byref(n)) == NULL
    assert L.mtgr_gated_ffn_workspace_size(ctypes.byref(ffn()), 0, None) == NULL
    assert L.mtgr_gated_ffn_fwd(None, *[None] * 8, 0, None) == NULL
    assert L.mtgr_gated_ffn_bwd(None, *[None] * 10, 0, None) == NULL
    assert L.mtgr_gated_ffn_workspace_size(ctypes.byref(ffn()), 3, ctypes.byref(n)) == INVALID
    assert hstu.mtgr_gated_ffn_workspace_size(ffn(tokens=0)) == 0
    for T in (1, 100, 700, 5000, 70000):                 # the forward that keeps h needs no more than serving
        p = ffn(tokens=T, dim=512, hidden=1408)
        keep = hstu.mtgr_gated_ffn_workspace_size(p, hstu.MTGR_FFN_TRAINING)
        assert keep <= hstu.mtgr_gated_ffn_workspace_size(p) - 2 * T * 1408
    ffn_fwd(ffn(tokens=0), x=None, w_in=None, w_out=None, y=None, workspace=None, workspace_bytes=0)


# ------------------------------------------------------------------ dropout

def drop(**kw):
    a = dict(rows=10, cols=64, dtype=hstu.MTGR_DTYPE_BF16, x=FAKE, ld_x=64, prob=0.1, rng=FAKE, site=0, residual=None,
             ld_residual=0, out=FAKE, ld_out=64, stream=0)
    a.update(kw)
    hstu.mtgr_dropout(**a)


@pytest.mark.parametrize("kw, status", [
    (dict(dtype=5), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(cols=12), INVALID),
    (dict(dtype=hstu.MTGR_DTYPE_FP32, cols=6), INVALID), (dict(prob=-0.1), INVALID), (dict(prob=1.0), INVALID),
    (dict(prob=float("nan")), INVALID), (dict(x=None), NULL), (dict(out=None), NULL), (dict(rng=None), NULL),
    (dict(rng=FAKE + 4), INVALID), (dict(x=FAKE + 8), INVALID), (dict(ld_x=56), INVALID), (dict(ld_out=68), INVALID),
    (dict(residual=FAKE, ld_residual=32), INVALID), (dict(residual=FAKE + 2, ld_residual=64), INVALID),
    (dict(ld_x=1 << 22), UNSUPPORTED), (dict(rows=1 << 44), INVALID),
])
def test_dropout_refused(kw, status):
    assert status_of(drop, **kw) == status


def test_generator_known_answer():
    # Random123's known answer of philox4x32 with 7 rounds for an all-zero counter and key: pins the oracle
    assert [int(v) for v in philox_words(0, 0, 0, 4)] == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]


def test_dropout_of_no_rows():
    drop(rows=0, x=None, out=None, rng=None)


# ------------------------------------------------------------------ softmax loss

def loss_problem(**kw):
    a = dict(num_rows=50, num_classes=70, dim=64, target_bits=64, scale=1.0, ld_x=64, ld_w=64)
    a.update(kw)
    return hstu.SoftmaxLossProblem(**a)


def loss_fwd(p, **kw):
    a = dict(x=FAKE, w=FAKE, targets=FAKE, bias=None, loss=FAKE, lse=FAKE, workspace=FAKE, workspace_bytes=BIG, stream=0)
    a.update(kw)
    hstu.mtgr_softmax_loss_fwd(p, **a)


def loss_bwd(p, **kw):
    a = dict(dloss=FAKE, x=FAKE, w=FAKE, targets=FAKE, bias=None, lse=FAKE, dx=FAKE, dw=FAKE, dbias=None,
             workspace=FAKE, workspace_bytes=BIG, stream=0)
    a.update(kw)
    hstu.mtgr_softmax_loss_bwd(p, **a)


@pytest.mark.parametrize("kw, status", [
    (dict(num_rows=-1), INVALID), (dict(num_rows=1 << 24), INVALID), (dict(num_classes=-1), INVALID),
    (dict(num_classes=1 << 30), INVALID), (dict(num_classes=0), INVALID), (dict(dim=0), UNSUPPORTED),
    (dict(dim=40), UNSUPPORTED), (dict(dim=2080, ld_x=2080, ld_w=2080), UNSUPPORTED), (dict(target_bits=16), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(ld_x=56), INVALID),
    (dict(ld_w=68), INVALID), (dict(ld_w=1 << 22), UNSUPPORTED),
])
def test_loss_problem_refused(kw, status):
    if kw.get("num_classes") != 0:
        assert status_of(loss_bwd, loss_problem(**kw)) == status
    assert status_of(loss_fwd, loss_problem(**kw)) == status


@pytest.mark.parametrize("kw, status", [
    (dict(x=None), NULL), (dict(w=None), NULL), (dict(targets=None), NULL), (dict(lse=None), NULL),
    (dict(x=FAKE + 8), INVALID), (dict(w=FAKE + 2), INVALID), (dict(targets=FAKE + 4), INVALID),
    (dict(bias=FAKE + 2), INVALID), (dict(lse=FAKE + 1), INVALID), (dict(workspace=None), NULL),
    (dict(workspace=FAKE + 128), INVALID), (dict(workspace_bytes=100), SMALL),
])
def test_loss_pointers_refused(kw, status):
    assert status_of(loss_fwd, loss_problem(), **kw) == status
    assert status_of(loss_bwd, loss_problem(), **kw) == status


@pytest.mark.parametrize("kw, status", [
    (dict(dloss=None), NULL), (dict(dx=None), NULL), (dict(dw=None), NULL), (dict(dloss=FAKE + 2), INVALID),
    (dict(dx=FAKE + 4), INVALID), (dict(dw=FAKE + 4), INVALID), (dict(dbias=FAKE + 2), INVALID),
])
def test_loss_backward_refused(kw, status):
    assert status_of(loss_bwd, loss_problem(), **kw) == status


def test_loss_of_nothing():
    loss_fwd(loss_problem(num_rows=0), x=None, w=None, targets=None, loss=None, lse=None, workspace=None)
    loss_bwd(loss_problem(num_rows=0, num_classes=0), dloss=None, x=None, w=None, targets=None, lse=None, dx=None,
             dw=None, workspace=None)
    assert hstu.mtgr_softmax_loss_workspace_size(loss_problem(num_rows=0)) == 0


def test_loss_workspace_stays_bounded():
    """The workspace follows rows and pieces, not rows x classes: a hundred times the classes of a long batch
    takes a few more bytes (the class bias), and is far below the logits in bf16.  A piece has at most 4 GB, 104
    blocks of 256 classes at 80,000 rows; the first set's 391 blocks are four equal pieces of 98, so that the second
    one's may be 6 blocks larger."""
    sizes = [hstu.mtgr_softmax_loss_workspace_size(loss_problem(num_rows=80000, num_classes=v), True)
             for v in (100_000, 10_000_000)]
    assert sizes[0] < 2 * 80000 * 100_000
    assert sizes[1] - sizes[0] < 6 * 256 * 2 * 80000 + (64 << 20 | 4 * 10_000_000)


# ------------------------------------------------------------------ wrappers

def test_wrappers_refuse_host_tensors_and_wrong_shapes():
    bf = torch.bfloat16
    x, w_in, w_out = torch.zeros(4, 32, dtype=bf), torch.zeros(32, 128, dtype=bf), torch.zeros(64, 32, dtype=bf)
    with pytest.raises(ValueError, match="device"):
        ops.gated_ffn_fwd(x, w_in, w_out)
    with pytest.raises(ValueError, match="x is"):
        ops.gated_ffn_fwd(x.float(), w_in, w_out)
    with pytest.raises(ValueError, match="matrix"):
        ops.gated_ffn_fwd(x[0], w_in, w_out)
    with pytest.raises(ValueError, match="device"):
        ops.dropout(x, 0.1, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError):
        ops.dropout(x.half(), 0.1, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="device"):
        ops.softmax_loss_fwd(x, x, torch.zeros(4, dtype=torch.int64))
