"""Causal attention of packed sequences against its 64-bit definition, element by element (bounds: tests/causal_ref.py)."""
import pytest
import torch

from paper_2505_18654_amd import ops
from tests.block_ref import half_step, within
from tests.causal_ref import causal, causal_back, heads, offsets_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def batch(lengths, H, Hk, dh, seed=1, wide=0, more=0, size=1.0):
    T = sum(lengths) + more
    return (heads((T, H, dh), seed, size, wide), heads((T, Hk, dh), seed + 1, size, wide), heads((T, Hk, dh), seed + 2, 1.0, wide),
            heads((T, H, dh), seed + 3, 1.0, wide))


def check(lengths, H, Hk, dh, wide=0, more=0, scale=None, size=1.0, seed=1):
    print(f"[causal] lengths={lengths[:8]}.. {len(lengths)} H={H} Hk={Hk} dh={dh} wide={wide} more={more}", flush=True)
    q, k, v, dout = batch(lengths, H, Hk, dh, seed, wide, more, size)
    o, n, s = offsets_of(lengths), sum(lengths), dh ** -0.5 if scale is None else scale
    out, lse = ops.causal_attn_fwd(q, k, v, o, scale=scale, save=True)
    torch.cuda.synchronize()
    want, wl, eo, el = causal(q[:n], k[:n], v[:n], lengths, s)
    within("out", out[:n], want, half_step(out[:n]) + eo * (1 + 2.0 ** -7))
    within("lse", lse[:, :n], wl, el)
    assert torch.equal(ops.causal_attn_fwd(q, k, v, o, scale=scale)[:n], out[:n])
    print("[causal] backward", flush=True)
    got = dict(zip(("dq", "dk", "dv"), ops.causal_attn_bwd(dout, q, k, v, out, lse, o, scale=scale)))
    torch.cuda.synchronize()
    for x, (g, b) in causal_back(dout[:n], q[:n], k[:n], v[:n], out[:n], lse[:, :n], lengths, s).items():
        within(x, got[x][:n], g, half_step(got[x][:n]) + b * (1 + 2.0 ** -7))
    for x, (g, b) in causal_back(dout[:n], q[:n], k[:n], v[:n], want, wl, lengths, s, exact_out=True).items():
        within(x + " of the definition", got[x][:n], g, half_step(got[x][:n]) + b * (1 + 2.0 ** -7))
    again = ops.causal_attn_bwd(dout, q, k, v, out, lse, o, scale=scale)
    assert all(torch.equal(a[:n], got[x][:n]) for a, x in zip(again, got))      # the same order of sums each time


LENGTHS = [[1], [2], [31], [32], [33], [63, 64, 65], [127, 128, 129], [1, 1, 1, 0, 5, 0], [300, 1, 77], [513]]


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_lengths(lengths, dh):
    check(lengths, 2, 1, dh)


@pytest.mark.parametrize("H, Hk, dh", [(1, 1, 128), (4, 4, 64), (6, 2, 128), (3, 3, 32), (8, 1, 64), (24, 8, 32), (10, 2, 128)])
def test_head_layouts(H, Hk, dh):
    check([150, 40], H, Hk, dh)


def test_columns_of_a_projection_and_rows_behind():
    check([100, 31, 200], 4, 2, 64, wide=3, more=37)
    check([257], 2, 2, 128, wide=1, more=1)


def test_long():
    check([3001, 2], 2, 1, 128)
    check([5000], 1, 1, 64)


# more tiles than the kernels for few take: sequences around the edges of tiles, cut-up long ones among them
@pytest.mark.parametrize("H, Hk, dh", [(8, 2, 128), (16, 16, 64), (12, 1, 64), (16, 4, 32)])
def test_batches(H, Hk, dh):
    check([1, 1500, 0, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 191, 193, 2, 2000, 300], H, Hk, dh, more=5)
    check([700] * 6 + [64] * 10, H, Hk, dh, wide=2)


def test_many_sequences():
    check([3, 1, 0, 7, 2] * 40, 2, 1, 32)
    check([1, 0, 2] * 1700, 1, 1, 32)                    # the search for a tile's sequence takes three steps


@pytest.mark.parametrize("size, scale", [(1.0, 0.5), (4.0, 0.3), (0.0, 1.0), (1.0, 1e-30)])
def test_scales(size, scale):
    check([130, 5], 2, 1, 64, scale=scale, size=size)


def test_falling_and_rising_scores():
    """Keys whose scores grow or shrink along the sequence, so that the running maximum moves at every tile or never."""
    for up in (True, False):
        n, dh = 700, 64
        q, k, v, _ = batch([n], 1, 1, dh)
        ramp = torch.linspace(0, 40, n).cuda()
        q = torch.zeros_like(q)
        q[..., 0] = 8.0
        k[..., 0] = (ramp if up else ramp.flip(0))[:, None].bfloat16()
        o = offsets_of([n])
        out, lse = ops.causal_attn_fwd(q, k, v, o, save=True)
        want, wl, eo, el = causal(q, k, v, [n], dh ** -0.5)
        within("out", out, want, half_step(out) + eo * (1 + 2.0 ** -7))
        within("lse", lse, wl, el)


@pytest.mark.parametrize("H, lengths", [(2, [500, 600]), (32, [1100])])
def test_offsets_past_32_bits(H, lengths):
    """Rows that lie 2^22 - 8 elements apart, the last ones 2^32 elements and more behind the first, against dense ones."""
    n, ld, dh = sum(lengths), (1 << 22) - 8, 32
    q, k, v, dout = batch(lengths, H, H, dh)
    o = offsets_of(lengths)
    out, lse = ops.causal_attn_fwd(q, k, v, o, save=True)
    want = ops.causal_attn_bwd(dout, q, k, v, out, lse, o)

    def far():
        room = torch.empty((n - 1) * ld + 5 * H * dh, dtype=torch.bfloat16, device="cuda")
        return [room.as_strided((n, H, dh), (ld, dh, 1), i * H * dh) for i in range(5)]

    q2, k2, v2, dout2, out2 = far()
    for a, b in ((q2, q), (k2, k), (v2, v), (dout2, dout)):
        a.copy_(b)
    _, lse2 = ops.causal_attn_fwd(q2, k2, v2, o, save=True, out=out2)
    assert torch.equal(out2, out) and torch.equal(lse2, lse)
    grads = far()[:3]
    ops.causal_attn_bwd(dout2, q2, k2, v2, out2, lse2, o, grads=grads)
    assert all(torch.equal(a, b) for a, b in zip(grads, want))
    r = ops.rotary(32)
    ops.rope(q2, r, offsets=o, out=q2)
    assert torch.equal(q2, ops.rope(q, r, offsets=o))


def test_rows_behind_are_left():
    lengths = [40, 0, 90]
    q, k, v, dout = batch(lengths, 2, 1, 64, more=50)
    n, o = sum(lengths), offsets_of(lengths)
    for t in (q, k, v, dout):
        t[n:] = float("nan")
    out, lse = torch.full_like(q, 7.0), torch.full((2, n + 50), 7.0, device="cuda")
    ops.causal_attn_fwd(q, k, v, o, save=True, out=out, lse=lse)
    assert (out[n:] == 7).all() and (lse[:, n:] == 7).all() and torch.isfinite(out.float()).all()
    grads = [torch.full_like(t, 7.0) for t in (q, k, v)]
    ops.causal_attn_bwd(dout, q, k, v, out, lse, o, grads=grads)
    assert all((g[n:] == 7).all() and torch.isfinite(g.float()).all() for g in grads)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_other_sequences_do_not_matter(bad):
    lengths = [70, 33, 129]
    q, k, v, dout = batch(lengths, 2, 1, 64)
    o = offsets_of(lengths)
    out, lse = ops.causal_attn_fwd(q, k, v, o, save=True)
    grads = ops.causal_attn_bwd(dout, q, k, v, out, lse, o)
    q2, k2, v2, g2 = (t.clone() for t in (q, k, v, dout))
    for t in (q2, k2, v2, g2):
        t[70:103] = bad
    out2, lse2 = ops.causal_attn_fwd(q2, k2, v2, o, save=True)
    grads2 = ops.causal_attn_bwd(g2, q2, k2, v2, out2, lse2, o)
    for a, b in [(out, out2), *zip(grads, grads2)]:
        assert torch.equal(a[:70], b[:70]) and torch.equal(a[103:], b[103:])
    assert torch.equal(lse[:, :70], lse2[:, :70]) and torch.equal(lse[:, 103:], lse2[:, 103:])


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("n, at", [(1, 0), (90, 89), (200, 150), (300, 64), (129, 128), (128, 127)])
def test_later_tokens_do_not_matter(n, at, dh):
    """Infinities and NaN in the keys and values of a token reach its own and later outputs alone."""
    q, k, v, _ = batch([n], 2, 1, dh)
    o = offsets_of([n])
    lse = ops.causal_attn_fwd(q, k, v, o, save=True)[1]
    want, _, eo, _ = causal(q, k, v, [n], dh ** -0.5)
    for t, bad in ((v, float("nan")), (v, float("inf")), (k, float("nan"))):
        keep = t[at].clone()
        t[at, :, 5] = bad
        out2, lse2 = ops.causal_attn_fwd(q, k, v, o, save=True)
        t[at] = keep
        assert torch.isfinite(out2[:at].float()).all()
        within("before", out2[:at], want[:at], half_step(out2[:at]) + eo[:at] * (1 + 2.0 ** -7))
        assert torch.equal(lse2[:, :at], lse[:, :at])
        if t is v:
            assert not torch.isfinite(out2[at:, :, 5].float()).any()
            rest = [c for c in range(dh) if c != 5]
            assert torch.isfinite(out2[at:][..., rest].float()).all()
        else:
            assert torch.isnan(out2[at:].float()).all()


@pytest.mark.parametrize("H", [2, 128])          # (the kernels for few tiles and for many)
@pytest.mark.parametrize("scale", [0.5, 2.0])
def test_scores_of_minus_infinity(H, scale):
    """Keys whose scores are minus infinity, a block of 32 of them and more before the first other one, weigh nothing."""
    n, gone = 300, 70
    q, k, v, _ = batch([n], H, H, 32)
    q[..., 0] = q[..., 0].abs() + 0.5
    k[:gone, :, 0] = -torch.inf
    out, lse = ops.causal_attn_fwd(q, k, v, offsets_of([n]), scale=scale, save=True)
    want, wl, eo, el = causal(q[gone:], k[gone:], v[gone:], [n - gone], scale)
    within("out", out[gone:], want, half_step(out[gone:]) + eo * (1 + 2.0 ** -7))       # (adding a zero rounds nothing)
    within("lse", lse[:, gone:], wl, el)
    assert torch.isnan(out[:gone].float()).all()


def test_inputs_of_nan_alone():
    """Nothing is finite and nothing is redone key by key."""
    for lengths, H in (([6000], 1), ([6000], 8)):
        q, k, v, _ = batch(lengths, H, 1, 64)
        v.fill_(float("nan"))
        out, lse = ops.causal_attn_fwd(q, k, v, offsets_of(lengths), save=True)
        torch.cuda.synchronize()
        assert torch.isnan(out.float()).all() and torch.isfinite(lse).all()


def test_nothing():
    q, k, v, dout = batch([], 2, 1, 64)
    out, lse = ops.causal_attn_fwd(q, k, v, offsets_of([]), save=True)
    assert out.shape == (0, 2, 64) and lse.shape == (2, 0)
    assert [g.shape[0] for g in ops.causal_attn_bwd(dout, q, k, v, out, lse, offsets_of([0, 0]))] == [0, 0, 0]
    q, k, v, _ = batch([5], 2, 1, 64)
    out = torch.full_like(q, 3.0)
    ops.causal_attn_fwd(q, k, v, offsets_of([0, 0]), out=out)
    assert (out == 3).all()


def test_streams_and_graph():
    lengths = [100, 31]
    q, k, v, dout = batch(lengths, 4, 2, 64)
    o = offsets_of(lengths)

    def step(out, lse, grads, ws):
        ops.causal_attn_fwd(q, k, v, o, save=True, out=out, lse=lse)
        ops.causal_attn_bwd(dout, q, k, v, out, lse, o, grads=grads, workspace=ws)

    out, lse = torch.zeros_like(q), torch.zeros(4, 131, device="cuda")
    grads, ws = [torch.zeros_like(t) for t in (q, k, v)], ops.causal_attn_workspace(q, k, o)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out, lse, grads, ws)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out, lse, grads, ws)
    for i in range(3):
        q.copy_(heads(q.shape, 50 + i))
        ws.fill_(255)                                    # a workspace may hold anything
        g.replay()
        torch.cuda.synchronize()
        o2, l2 = ops.causal_attn_fwd(q, k, v, o, save=True)
        g2 = ops.causal_attn_bwd(dout, q, k, v, o2, l2, o)
        assert torch.equal(out, o2) and torch.equal(lse, l2) and all(torch.equal(a, b) for a, b in zip(grads, g2))


# ------------------------------------------------------------------ the kernels for few tiles and for many

FEW_TILES = 1024       # tiles of 32 rows, of all heads, that the kernels for few take at most
SIDES = [(2, "few"), (128, "many")]


def on_side(side, lengths, H, more=0):
    assert ((sum(lengths) + more) // 32 + len(lengths)) * H > FEW_TILES if side == "many" else \
        ((sum(lengths) + more) // 32 + len(lengths)) * H <= FEW_TILES


@pytest.mark.parametrize("H, side", SIDES)
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("n, at", [(300, 250), (300, 33), (270, 1)])
def test_outputs_keep_their_bits_whatever_follows(n, at, dh, H, side):
    """Tokens from `at` on of other values and sizes, 60 times the scores among them: outputs and log-sums before are the same."""
    on_side(side, [n], H)
    q, k, v, _ = batch([n], H, H // 2, dh)
    o = offsets_of([n])
    out, lse = ops.causal_attn_fwd(q, k, v, o, save=True)
    for size in (0.0, 7.0, 60.0):
        q2, k2, v2 = q.clone(), k.clone(), v.clone()
        q2[at:] *= size
        k2[at:] = k2[at:].flip(0)
        v2[at:] *= -size
        out2, lse2 = ops.causal_attn_fwd(q2, k2, v2, o, save=True)
        assert torch.equal(out2[:at], out[:at]) and torch.equal(lse2[:, :at], lse[:, :at])


@pytest.mark.parametrize("H, side", SIDES)
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("n, at", [(300, 150), (300, 64), (257, 256), (289, 287)])
def test_later_values_do_not_matter(n, at, dh, H, side):
    """Infinities and NaN among a token's values reach its own and later outputs, and of those their feature alone; a NaN in its
    key reaches them all.  On the kernels for few tiles and for many."""
    on_side(side, [n], H)
    q, k, v, _ = batch([n], H, 2, dh)
    o = offsets_of([n])
    out, lse = ops.causal_attn_fwd(q, k, v, o, save=True)
    want, _, eo, _ = causal(q, k, v, [n], dh ** -0.5)
    lone = heads_of_key(H, 1)
    for t, bad in ((v, float("nan")), (v, float("inf")), (k, float("nan"))):
        t2 = t.clone()
        t2[at, 1, 5] = bad
        out2, lse2 = ops.causal_attn_fwd(q, k if t is v else t2, t2 if t is v else v, o, save=True)
        same = torch.ones(n, H, dh, dtype=torch.bool, device="cuda")
        if t is v:
            same[at:, lone, 5] = False
            hit = out2[at:, lone, 5]
            assert (hit == bad).all() if bad == bad else torch.isnan(hit).all()
            within("before", out2[:at], want[:at], half_step(out2[:at]) + eo[:at] * (1 + 2.0 ** -7))
            # (the products' own values but in the half of 32 tokens that holds the infinity)
            same[at - at % 32:at, lone, 5] = False
            assert torch.equal(lse2, lse)
        else:
            same[at:, lone] = False
            assert torch.isnan(out2[at:, lone]).all() and torch.equal(lse2[:, :at], lse[:, :at])
        assert torch.equal(out2[same], out[same])


def heads_of_key(H, j, Hk=2):
    return slice(j * H // Hk, (j + 1) * H // Hk)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("H, side", SIDES)
def test_infinities_in_several_places(H, side, dh):
    """Infinities of either sign before, in and behind a row's half: their sum by the definition, NaN where signs meet."""
    n = 270
    on_side(side, [n], H)
    q, k, v, _ = batch([n], H, 2, dh)
    for at, f, x in ((10, 1, torch.inf), (100, 1, -torch.inf), (101, 2, -torch.inf), (103, 2, -torch.inf), (120, 2, torch.nan),
                     (200, 3, torch.inf), (201, 3, -torch.inf), (269, 4, torch.inf), (0, 6, -torch.inf)):
        v[at, :, f] = x
    out = ops.causal_attn_fwd(q, k, v, offsets_of([n]))
    row = torch.arange(n, device="cuda")
    for f, spans in ((1, [(10, torch.inf), (100, torch.nan)]), (2, [(101, -torch.inf), (120, torch.nan)]),
                     (3, [(200, torch.inf), (201, torch.nan)]), (4, [(269, torch.inf)]), (6, [(0, -torch.inf)])):
        assert torch.isfinite(out[:spans[0][0], :, f]).all(), f
        for (a, x), (b, _) in zip(spans, spans[1:] + [(n, 0)]):
            part = out[(row >= a) & (row < b)][..., f]
            assert torch.isnan(part).all() if x != x else (part == x).all(), (f, a)
    rest = [c for c in range(dh) if c not in (1, 2, 3, 4, 6)]
    v[...] = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    want, _, eo, _ = causal(q, k, v, [n], dh ** -0.5)
    within("rest", out[..., rest], want[..., rest], half_step(out[..., rest]) + eo[..., rest] * (1 + 2.0 ** -7))
    for f, end in ((1, 10), (2, 101), (3, 200), (4, 269)):
        within(f"feature {f}", out[:end, :, f], want[:end, :, f], half_step(out[:end, :, f]) + eo[:end, :, f] * (1 + 2.0 ** -7))


@pytest.mark.parametrize("n, H, dh", [(2000, 2, 128), (8000, 8, 128)])
def test_one_infinity_does_not_hold_up_the_pass(n, H, dh):
    """Its half of 32 tokens is redone by products: the pass takes 4.6 and 2.5 times as long, where keys one by one took 295 and
    330 times; 25 times is refused."""
    q, k, v, _ = batch([n], H, 1, dh)
    o = offsets_of([n])

    def least():
        t = []
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in "ab")
            a.record()
            ops.causal_attn_fwd(q, k, v, o)
            b.record()
            b.synchronize()
            t.append(a.elapsed_time(b))
        return min(t)

    plain = least()
    for at in (n - 1, n // 2):
        v2 = v.clone()
        v[at, :, 3] = torch.inf
        assert least() < 25 * plain
        v = v2


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_other_sequences_do_not_matter_in_large_batches(bad, dh):
    """As above, on the kernels for many tiles, with sequences of several pieces of the backward's work among them."""
    lengths, H = [70, 33, 1500, 129, 300, 64], 32
    on_side("many", lengths, H)
    q, k, v, dout = batch(lengths, H, 4, dh)
    o, at = offsets_of(lengths), [0, 70, 103, 1603, 1732, 2032, 2096]
    out, lse = ops.causal_attn_fwd(q, k, v, o, save=True)
    grads = ops.causal_attn_bwd(dout, q, k, v, out, lse, o)
    for hit in ([1], [2], [0, 3, 5]):
        q2, k2, v2, g2 = (t.clone() for t in (q, k, v, dout))
        keep = torch.ones(2096, dtype=torch.bool, device="cuda")
        for i in hit:
            keep[at[i]:at[i + 1]] = False
            for t in (q2, k2, v2, g2):
                t[at[i]:at[i + 1]] = bad
        out2, lse2 = ops.causal_attn_fwd(q2, k2, v2, o, save=True)
        grads2 = ops.causal_attn_bwd(g2, q2, k2, v2, out2, lse2, o)
        for a, b in [(out, out2), *zip(grads, grads2)]:
            assert torch.equal(a[keep], b[keep])
        assert torch.equal(lse[:, keep], lse2[:, keep])


@pytest.mark.parametrize("dh", [32, 64, 128])
def test_rows_behind_are_left_in_large_batches(dh):
    lengths, H = [40, 0, 90, 300], 128
    on_side("many", lengths, H, 50)
    q, k, v, dout = batch(lengths, H, 16, dh, more=50)
    n, o = sum(lengths), offsets_of(lengths)
    for t in (q, k, v, dout):
        t[n:] = float("nan")
    out, lse = torch.full_like(q, 7.0), torch.full((H, n + 50), 7.0, device="cuda")
    ops.causal_attn_fwd(q, k, v, o, save=True, out=out, lse=lse)
    assert (out[n:] == 7).all() and (lse[:, n:] == 7).all() and torch.isfinite(out).all()
    grads = [torch.full_like(t, 7.0) for t in (q, k, v)]
    ops.causal_attn_bwd(dout, q, k, v, out, lse, o, grads=grads)
    assert all((g[n:] == 7).all() and torch.isfinite(g).all() for g in grads)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("H, side", SIDES)
@pytest.mark.parametrize("shape", ["rising", "falling", "steps", "one peak"])
def test_moving_maximum(shape, H, side, dh):
    """Scores that pass the reference by more than 2^8 at every second half, never, now and then, or once in the middle: outputs,
    log-sums and gradients."""
    n = 350
    on_side(side, [n], H)
    q, k, v, dout = batch([n], H, 2, dh)
    ramp = torch.linspace(0, 40, n)
    x = {"rising": ramp, "falling": ramp.flip(0), "steps": 9.0 * (torch.arange(n) // 70), "one peak": 40.0 * (torch.arange(n) == 170)}[shape]
    q[..., 0], k[..., 0] = 8.0 * dh ** 0.5 / 8, x.cuda()[:, None].bfloat16()
    q[..., 1:] *= 0.25
    o, s = offsets_of([n]), dh ** -0.5
    out, lse = ops.causal_attn_fwd(q, k, v, o, save=True)
    want, wl, eo, el = causal(q, k, v, [n], s)
    within("out", out, want, half_step(out) + eo * (1 + 2.0 ** -7))
    within("lse", lse, wl, el)
    got = dict(zip(("dq", "dk", "dv"), ops.causal_attn_bwd(dout, q, k, v, out, lse, o)))
    for name, (g, b) in causal_back(dout, q, k, v, out, lse, [n], s).items():
        within(name, got[name], g, half_step(got[name]) + b * (1 + 2.0 ** -7))
