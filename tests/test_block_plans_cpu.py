"""Which kernels the sizes of the GPU tests run on (CPU only: the library's host code chooses)."""
import ctypes

import pytest

from paper_2505_18654_amd import hstu, ops
from tests import block_shapes as S
from tests.test_block_cpu import INVALID, NULL, ffn, loss_problem


def holds(want, got):
    assert {k: got[k] for k in want} == want, got
    return got


def ffn_kernels(shape):
    p = ops.gated_ffn_problem(*shape)
    return (hstu.mtgr_debug_gated_ffn_kernels(p, hstu.MTGR_FFN_SERVING, residual=True),
            hstu.mtgr_debug_gated_ffn_kernels(p, hstu.MTGR_FFN_TRAINING), hstu.mtgr_debug_gated_ffn_kernels(p, hstu.MTGR_FFN_BACKWARD))


def loss_kernels(N, V, d, labels):
    p = hstu.SoftmaxLossProblem(N, V, d, 64, 1.0, d, d)
    return tuple(hstu.mtgr_debug_softmax_loss_kernels(p, b, labels) for b in (False, True))


@pytest.mark.parametrize("shape, want", [*S.FFN.items(), (S.FFN_LONG, S.FFN_LONG_KERNELS)])
def test_ffn_shapes_reach_their_kernels(shape, want):
    for w, g in zip(want, ffn_kernels(shape)):
        holds(w, g)


def test_ffn_shapes_reach_every_kernel():
    got = [ffn_kernels(s) for s in S.FFN]
    tiles = lambda name: name.split("/")[0]
    for k in (0, 1):
        assert {tiles(g[k]["hidden"]) for g in got} == {"rows", "128x128", "256x256"}
        assert {tiles(g[k]["out"]) for g in got} == {"rows", "128x128", "256x256"} | ({"256x128"} if k else set())
        assert {g[k]["h"] for g in got if g[k]["hidden"] == "256x256"} == {"cached", "streamed"}
    assert {g[2]["dpre"] for g in got} == {"128x128", "256x256"} and {g[2]["together"] for g in got} == {"0", "1"}
    assert {g[2]["store"] for g in got if g[2]["dpre"] == "256x256"} == {"cached", "streamed"}
    apart = [g[2] for g in got if g[2]["together"] == "0"]
    assert {tiles(g["dx"]) for g in apart} == {"128x128", "256x256"}
    assert {tiles(g["dw_out"]) for g in apart} == {"128x128", "256x256"}


@pytest.mark.parametrize("shape, want", S.LOSS.items())
def test_loss_shapes_reach_their_kernels(shape, want):
    for w, g in zip(want, loss_kernels(*shape)):
        holds(w, g)


@pytest.mark.parametrize("shape", S.CARRIED_RUN)
def test_statistics_are_carried_over_tiles(shape):
    N = shape[0]
    got = loss_kernels(*shape, N)[0]
    assert got["logits"] == ("256x256" if shape is S.CARRIED_WIDE else "registers")
    assert int(got["run"]) == S.CARRIED_RUN[shape] and got["pieces"] == "1"


def test_refusals():
    L, text = hstu.lib(), ctypes.create_string_buffer(256)
    p, q = ctypes.byref(ffn()), ctypes.byref(loss_problem())
    assert L.mtgr_debug_gated_ffn_kernels(None, 0, 0, text, 256) == NULL
    assert L.mtgr_debug_gated_ffn_kernels(p, 0, 0, None, 256) == NULL
    assert L.mtgr_debug_gated_ffn_kernels(p, 3, 0, text, 256) == INVALID
    assert L.mtgr_debug_gated_ffn_kernels(ctypes.byref(ffn(tokens=0)), 0, 0, text, 256) == INVALID
    assert L.mtgr_debug_softmax_loss_kernels(None, 0, 0, text, 256) == NULL
    assert L.mtgr_debug_softmax_loss_kernels(q, 0, 50, None, 256) == NULL
    assert L.mtgr_debug_softmax_loss_kernels(q, 0, 51, text, 256) == INVALID
    assert L.mtgr_debug_softmax_loss_kernels(q, 0, -1, text, 256) == INVALID
    assert L.mtgr_debug_softmax_loss_kernels(ctypes.byref(loss_problem(num_rows=0)), 0, 0, text, 256) == INVALID
    for n in (0, 1, 20):                                 # too short: a status, and nothing written past the end
        short = ctypes.create_string_buffer(b"\x7f" * 64, 64)
        assert L.mtgr_debug_gated_ffn_kernels(p, 0, 0, short, n) == INVALID
        assert L.mtgr_debug_softmax_loss_kernels(q, 1, 50, short, n) == INVALID
        assert short.raw[n:] == b"\x7f" * (64 - n)
