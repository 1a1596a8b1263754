"""Rotary positions against their 64-bit definition, element by element (bounds: tests/causal_ref.py)."""
import pytest
import torch

from paper_2505_18654_amd import ops
from tests.block_ref import U, half_step, within
from tests.causal_ref import heads, offsets_of, rotate

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def stored(x):
    return half_step(x) if x.dtype == BF else U * x.double().abs()


def check(x, rot, positions, got, sign=1):
    want, bound = rotate(x, rot.freqs, sign * positions.double(), rot.amplitude, rot.layout)
    within("rope", got, want, stored(got) + bound * (1 + 2.0 ** -7))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T, H, dh, rot, dtype", [
    (1, 1, 16, 16, BF), (1, 8, 128, 128, BF), (7, 3, 64, 48, BF), (64, 32, 128, 64, BF), (333, 5, 72, 16, BF),
    (1000, 12, 128, 96, BF), (20011, 2, 64, 64, BF), (1, 1, 16, 16, F32), (5, 3, 64, 32, F32), (313, 4, 136, 112, F32),
    (9001, 6, 128, 128, F32), (3, 2, 1024, 1024, BF),
])
def test_rotation(T, H, dh, rot, dtype, layout):
    print(f"[rope] T={T} H={H} dh={dh} rot={rot} {dtype} {layout}", flush=True)
    x = heads((T, H, dh), 3, dtype=dtype)
    pos = torch.randint(0, 40000, (T,), generator=torch.Generator().manual_seed(4), dtype=torch.int32).cuda()
    r = ops.rotary(rot, layout=layout)
    y = ops.rope(x, r, positions=pos)
    check(x, r, pos, y)
    check(x, r, pos, ops.rope(x, r, positions=pos, inverse=True), -1)
    z = x.clone()
    assert ops.rope(z, r, positions=pos, out=z) is z and torch.equal(z, y)
    torch.cuda.synchronize()


@pytest.mark.parametrize("scaling", ["linear", "base", "parts"])
def test_scaled(scaling):
    x = heads((129, 4, 64), 5)
    pos = torch.arange(129, dtype=torch.int32).cuda() * 511
    r = ops.rotary(64, base=500000.0, scaling=scaling, factor=16.0, trained_len=4096)
    check(x, r, pos, ops.rope(x, r, positions=pos))
    check(x, r, pos, ops.rope(x, r, positions=pos, inverse=True), -1)


def test_far_and_negative_positions():
    x = heads((8, 2, 64), 6, dtype=F32)
    pos = torch.tensor([0, -1, 1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, -12345678, 1000000007], dtype=torch.int32).cuda()
    for layout in ("half", "interleaved"):
        r = ops.rotary(64, layout=layout)
        check(x, r, pos, ops.rope(x, r, positions=pos))
        check(x, r, pos, ops.rope(x, r, positions=pos, inverse=True), -1)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_columns_of_a_projection(dtype):
    x, out = heads((130, 6, 64), 7, wide=4, dtype=dtype), heads((130, 6, 64), 8, wide=2, dtype=dtype)
    whole = out.as_strided((130, 8, 64), out.stride())
    tail = whole[:, 6:].clone()
    pos = torch.arange(130, dtype=torch.int32).cuda()
    r = ops.rotary(32)
    ops.rope(x, r, positions=pos, out=out)
    check(x, r, pos, out)
    assert torch.equal(whole[:, 6:], tail)
    y = x.clone()
    z = heads((130, 6, 64), 7, wide=4, dtype=dtype)
    rest = z.as_strided((130, 10, 64), z.stride())[:, 6:].clone()
    ops.rope(z, r, positions=pos, out=z)
    check(y, r, pos, z)
    assert torch.equal(z.as_strided((130, 10, 64), z.stride())[:, 6:], rest)


@pytest.mark.parametrize("lengths", [[5], [1, 0, 3, 0, 0, 200, 1], [0, 0], [17] * 100])
def test_positions_of_sequences(lengths):
    n = sum(lengths)
    x, out = heads((n + 9, 3, 32), 9), heads((n + 9, 3, 32), 10)
    before = out.clone()
    r = ops.rotary(32)
    ops.rope(x, r, offsets=offsets_of(lengths), out=out)
    pos = torch.cat([torch.arange(m) for m in lengths]).cuda()
    check(x[:n], r, pos, out[:n])
    assert torch.equal(out[n:], before[n:])                      # rows behind the last sequence


def test_nothing():
    x = heads((0, 3, 32), 1)
    assert ops.rope(x, ops.rotary(16), positions=torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 3, 32)


def test_infinities_stay_in_their_pair():
    x = heads((4, 2, 32), 11)
    x[1, 0, 3], x[2, 1, 31] = float("inf"), float("nan")
    r = ops.rotary(16)
    pos = torch.arange(4, dtype=torch.int32).cuda()
    y = ops.rope(x, r, positions=pos)
    bad = ~torch.isfinite(y.float())
    assert bad.sum() == 3 and bad[1, 0, 3] and bad[1, 0, 11] and bad[2, 1, 31]


def test_streams_and_graph():
    x = heads((100, 4, 64), 12)
    pos = torch.arange(100, dtype=torch.int32).cuda()
    r = ops.rotary(64)
    want = ops.rope(x, r, positions=pos)
    out = torch.zeros_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ops.rope(x, r, positions=pos, out=out)
    side.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ops.rope(x, r, positions=pos, out=out)
    for i in range(3):
        pos += 7
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ops.rope(x, r, positions=pos))
