"""The paged cache: appending to it, and single tokens against it (bounds: tests/causal_ref.py)."""
import pytest
import torch

from paper_2505_18654_amd import ops
from tests.block_ref import half_step, within
from tests.causal_ref import attend, heads, offsets_of, rotate

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def make_cache(lengths, Hk, page, dh, seed=1, spare=3, columns=None):
    """A cache of these lengths, pages in random order, what no token holds NaN; also k, v of each sequence."""
    g = torch.Generator().manual_seed(seed)
    pages = [-(-n // page) for n in lengths]
    total = sum(pages) + spare
    order = torch.randperm(total, generator=g)
    table = torch.full((len(lengths), columns or max(pages + [1])), -7, dtype=torch.int32)
    c = ops.KvCache.empty(total, Hk, page, dh)
    c.keys.fill_(NAN)
    c.values.fill_(NAN)
    ks, vs, at = [], [], 0
    for b, n in enumerate(lengths):
        table[b, :pages[b]] = order[at:at + pages[b]].int()
        at += pages[b]
        ks.append(heads((n, Hk, dh), 1000 * seed + 2 * b))
        vs.append(heads((n, Hk, dh), 1000 * seed + 2 * b + 1))
        i = torch.arange(n)
        p, r = table[b].long()[i // page].cuda(), (i % page).cuda()
        c.keys[p, :, r], c.values[p, :, r] = ks[-1], vs[-1]
    return c, table.cuda(), ks, vs


def lens_of(lengths):
    return torch.tensor(lengths, dtype=torch.int32).cuda()


def expect(q, ks, vs, scale):
    B, H, dh = q.shape
    out, eo = torch.zeros(B, H, dh, dtype=torch.float64, device="cuda"), torch.zeros(B, H, dh, dtype=torch.float64, device="cuda")
    lse, el = torch.full((B, H), -torch.inf, dtype=torch.float64, device="cuda"), torch.zeros(B, H, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, Hk = ks[b].shape[:2]
        for h in range(H if n else 0):
            j = h // (H // Hk)
            o, s, a, e = attend(q[b:b + 1, h], ks[b][:, j], vs[b][:, j], scale, torch.zeros(1, n, dtype=torch.bool, device="cuda"))
            out[b, h], lse[b, h], eo[b, h], el[b, h] = o[0], s[0], a[0], e[0]
    return out, lse, eo, el


def compare(q, ks, vs, out, lse, scale):
    want, wl, eo, el = expect(q, ks, vs, scale)
    within("out", out, want, half_step(out) + eo * (1 + 2.0 ** -7))
    empty = torch.isinf(wl)
    assert torch.equal(torch.isinf(lse) & (lse < 0), empty) and (out[empty] == 0).all()
    within("lse", lse[~empty], wl[~empty], el[~empty])


def check(lengths, H, Hk, dh, page, scale=None, max_len=None, wide=0):
    print(f"[cache] {lengths[:6]} of {len(lengths)} H={H} Hk={Hk} dh={dh} page={page} max_len={max_len}", flush=True)
    c, table, ks, vs = make_cache(lengths, Hk, page, dh)
    q = heads((len(lengths), H, dh), 77, wide=wide)
    out, lse = ops.cache_attn(q, c, table, lens_of(lengths), scale=scale, max_len=max_len, save=True)
    torch.cuda.synchronize()
    compare(q, ks, vs, out, lse, dh ** -0.5 if scale is None else scale)
    assert torch.equal(ops.cache_attn(q, c, table, lens_of(lengths), scale=scale, max_len=max_len), out)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_lengths(page, dh):
    check([1, 2, 15, 16, 17, 31, 32, 33, 0, 63, 64, 65, 127, 128, 129, 500], 4, 2, dh, page)


@pytest.mark.parametrize("H, Hk, dh", [(1, 1, 128), (8, 8, 64), (6, 2, 128), (32, 1, 64), (33, 1, 64), (40, 1, 32), (70, 2, 128),
                                       (24, 8, 32), (15, 3, 128)])
def test_head_layouts(H, Hk, dh):
    check([77, 300, 5], H, Hk, dh, 32, wide=2)


@pytest.mark.parametrize("n", [1, 411, 2048, 2049, 20011])
def test_one_sequence(n):
    check([n], 8, 2, 128, 64, max_len=n)
    check([n], 3, 1, 64, 16)


def test_many_sequences_and_long_ones_among_short():
    check([5, 1, 40] * 60, 4, 2, 64, 16)
    check([3, 9000, 1, 70], 8, 4, 128, 128, max_len=9000)
    check([3, 9000, 1, 70], 8, 4, 32, 4096)


def test_max_len_bounds_the_lengths():
    c, table, ks, vs = make_cache([100, 40], 1, 32, 64)
    q = heads((2, 2, 64), 5)
    out, lse = ops.cache_attn(q, c, table, lens_of([100, 40]), max_len=50, save=True)
    compare(q, [k[:50] for k in ks], [v[:50] for v in vs], out, lse, 0.125)
    out, lse = ops.cache_attn(q, c, table, lens_of([100, 40]), max_len=0, save=True)
    assert (out == 0).all() and torch.isinf(lse).all()
    out, lse = ops.cache_attn(q, c, table, lens_of([-5, 2 ** 31 - 1]), max_len=40, save=True)
    assert (out[0] == 0).all() and torch.isinf(lse[0]).all()
    compare(q[1:], [ks[1]], [vs[1]], out[1:], lse[1:], 0.125)


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("bad", [-1, 1 << 30])
def test_entries_without_a_page(page, bad):
    """Tokens whose entry is no page count as absent; pages that the cache has follow and precede them."""
    n = 5 * page + 3
    c, table, ks, vs = make_cache([n, n, n, n, 17], 2, page, 64)
    lost = [[0], [1], [2, 5], [0, 1, 2, 3, 4, 5], [1] if page == 16 else []]
    keep = []
    for b, cols in enumerate(lost):
        m = torch.ones(ks[b].shape[0], dtype=torch.bool)
        for j in cols:
            table[b, j] = bad
            m[j * page:(j + 1) * page] = False
        keep.append(m.cuda())
    q = heads((5, 4, 64), 6)
    out, lse = ops.cache_attn(q, c, table, lens_of([n, n, n, n, 17]), save=True)
    compare(q, [k[m] for k, m in zip(ks, keep)], [v[m] for v, m in zip(vs, keep)], out, lse, 0.125)


@pytest.mark.parametrize("n, gone", [(300, 40), (3000, 2500)])
@pytest.mark.parametrize("scale", [0.5, 2.0])
def test_scores_of_minus_infinity(n, gone, scale):
    """Keys whose scores are minus infinity, whole tiles and chunks of them, weigh nothing."""
    c, table, ks, vs = make_cache([n], 2, 32, 64)
    q = heads((1, 4, 64), 9)
    q[..., 0] = q[..., 0].abs() + 0.5
    i = torch.arange(gone, device="cuda")
    c.keys[table[0].long()[i // 32], :, i % 32, 0] = -torch.inf
    out, lse = ops.cache_attn(q, c, table, lens_of([n]), scale=scale, save=True)
    compare(q, [ks[0][gone:]], [vs[0][gone:]], out, lse, scale)


def test_table_and_output_strides():
    c, table, ks, vs = make_cache([70, 20], 2, 16, 64)
    big = torch.full((2, table.shape[1] + 5), 9999, dtype=torch.int32, device="cuda")
    big[:, :table.shape[1]] = table
    q, out = heads((2, 4, 64), 5), heads((2, 4, 64), 8, wide=3)
    whole = out.as_strided((2, 7, 64), out.stride())
    rest = whole[:, 4:].clone()
    ops.cache_attn(q, c, big[:, :table.shape[1]], lens_of([70, 20]), out=out)
    assert torch.equal(out, ops.cache_attn(q, c, table, lens_of([70, 20]))) and torch.equal(whole[:, 4:], rest)


def test_pages_past_32_bits():
    """The last pages of a cache of 2^32 elements and more, against a small cache."""
    dh, page, n = 128, 4096, 5000
    small, table, ks, vs = make_cache([n], 1, page, dh, spare=0)
    many = (1 << 32) // (page * dh) + 4
    big = ops.KvCache.empty(many, 1, page, dh)
    last = torch.tensor([[many - 1, many - 3]], dtype=torch.int32).cuda()
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    ops.kv_append(big, last, zero, ks[0], vs[0], offsets=offsets_of([n]))
    for i in range(2):
        rows = min(page, n - i * page)
        for a, b in ((big.keys, small.keys), (big.values, small.values)):
            assert torch.equal(a[int(last[0, i]), :, :rows], b[int(table[0, i]), :, :rows])
    q = heads((1, 2, dh), 4)
    a, b = (ops.cache_attn(q, c, t, lens_of([n]), save=True) for c, t in ((big, last), (small, table)))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_no_sequences():
    c = ops.KvCache.empty(1, 1, 16, 64)
    table = torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    assert ops.cache_attn(heads((0, 2, 64), 1), c, table, lens_of([])).shape == (0, 2, 64)
    k = heads((0, 1, 64), 1)
    assert ops.kv_append(c, table, lens_of([]), k, k) is None


# ------------------------------------------------------------------ append

def check_append(past, new, H, Hk, dh, page, rot, layout="half", scaling="none", more=0, single=False, wide=1):
    print(f"[append] past={past} new={new} H={H} Hk={Hk} dh={dh} page={page} rot={rot} {layout}", flush=True)
    full = [max(p, 0) + n for p, n in zip(past, new)]
    c, table, _, _ = make_cache(full, Hk, page, dh)
    c.keys.copy_(heads((c.keys.shape[0] * Hk, page, dh), 31).view(c.keys.shape))
    c.values.copy_(heads((c.keys.shape[0] * Hk, page, dh), 32).view(c.keys.shape))
    keys, values = c.keys.clone(), c.values.clone()
    N = sum(new) + more
    q, k, v = heads((N, H, dh), 41, wide=wide), heads((N, Hk, dh), 42, wide=wide), heads((N, Hk, dh), 43, wide=wide)
    r = ops.rotary(rot, layout=layout, scaling=scaling, factor=4.0, trained_len=1024) if rot else None
    q_out = torch.full((N, H, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    got = ops.kv_append(c, table, lens_of(past), k, v, offsets=None if single else offsets_of(new), q=q, rotary=r, q_out=q_out)
    torch.cuda.synchronize()
    assert got is q_out
    want_q, written, t = torch.full_like(q_out, 7.0), torch.zeros(c.keys.shape, dtype=torch.bool, device="cuda"), 0
    for b, (p, n) in enumerate(zip(past, new)):
        rows = slice(t, t + n)
        t += n
        if p < 0 or n == 0:
            continue
        i = torch.arange(p, p + n, device="cuda")
        pages, row = table[b].long()[i // page], i % page
        want_k, bound_k = rotate(k[rows], r.freqs, i, r.amplitude, layout) if r else (k[rows].double(), 0.0)
        want, bound = rotate(q[rows], r.freqs, i, r.amplitude, layout) if r else (q[rows].double(), 0.0)
        got_k = c.keys[pages, :, row]
        within("k", got_k, want_k, half_step(got_k) * bool(r) + bound_k * (1 + 2.0 ** -7))
        within("q", q_out[rows], want, half_step(q_out[rows]) * bool(r) + bound * (1 + 2.0 ** -7))
        assert torch.equal(c.values[pages, :, row], v[rows])
        written[pages, :, row] = True
        want_q[rows] = q_out[rows]
    assert torch.equal(q_out, want_q)                                        # rows of no live sequence are left
    assert torch.equal(c.keys[~written], keys[~written]) and torch.equal(c.values[~written], values[~written])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("page, dh, rot", [(16, 32, 32), (32, 64, 16), (64, 128, 128), (128, 72, 64), (16, 8, 0), (4096, 128, 96)])
def test_append(page, dh, rot, layout):
    check_append([0, 5, 31, -1, 100, 0, 15], [3, 1, 40, 6, 0, 70, 17], 4, 2, dh, page, rot, layout, more=4)


@pytest.mark.parametrize("B", [1, 3, 64, 300])
def test_append_one_token_each(B):
    past = [(37 * b) % 90 for b in range(B)]
    if B > 2:
        past[1] = -3
    check_append(past, [1] * B, 8, 2, 128, 32, 128, scaling="parts", single=True)
    check_append(past, [1] * B, 3, 3, 64, 16, 32, "interleaved")


def test_append_prompts():
    check_append([0, 700, 12], [2000, 1, 900], 6, 3, 128, 64, 128)


def test_append_where_there_is_no_page():
    c, table, _, _ = make_cache([40, 40, 40], 1, 16, 32)
    table[1, 1], table[2, 1] = -1, c.keys.shape[0]
    keys, values = c.keys.clone(), c.values.clone()
    k, v, q = heads((60, 1, 32), 1), heads((60, 1, 32), 2), heads((60, 2, 32), 3)
    # sequence 0 runs past the table (3 columns of 16), 1 and 2 have no second page
    out = torch.full_like(q, 7.0)
    ops.kv_append(c, table, lens_of([38, 10, 10]), k, v, offsets=offsets_of([20, 20, 20]), q=q, q_out=out)
    torch.cuda.synchronize()
    t = table.long().cpu()
    got = lambda b, i: (c.keys[t[b, i // 16], :, i % 16], c.values[t[b, i // 16], :, i % 16])  # noqa: E731
    written = torch.zeros(keys.shape, dtype=torch.bool, device="cuda")
    for b, row0, tokens in ((0, 0, range(38, 48)), (1, 20, list(range(10, 16))), (2, 40, list(range(10, 16)))):
        for i in tokens:
            a, d = got(b, i)
            r = row0 + i - tokens[0]
            assert torch.equal(a, k[r]) and torch.equal(d, v[r])
            written[t[b, i // 16], :, i % 16] = True
    assert torch.equal(c.keys[~written].isnan(), keys[~written].isnan()) and (c.values[~written].isnan() == values[~written].isnan()).all()
    assert torch.equal(out[:10], q[:10]) and (out[10:20] == 7).all() and torch.equal(out[20:], q[20:])


def test_generation_step_by_step():
    """A prompt through the causal attention, then tokens one by one through the cache, captured and replayed: each step's
    output is the causal attention's last row over the whole sequence."""
    lengths, steps, H, Hk, dh, page = [40, 7, 129], 5, 4, 2, 64, 16
    B, r = len(lengths), ops.rotary(64)
    room = [n + steps for n in lengths]
    c, table, _, _ = make_cache(room, Hk, page, dh)
    c.keys.fill_(NAN)
    c.values.fill_(NAN)
    qs, ks, vs = ([heads((n, h, dh), s + b) for b, n in enumerate(room)] for h, s in ((H, 100), (Hk, 200), (Hk, 300)))
    first = lambda x: torch.cat([t[:n] for t, n in zip(x, lengths)])  # noqa: E731
    o, past = offsets_of(lengths), torch.zeros(B, dtype=torch.int32, device="cuda")
    q = ops.kv_append(c, table, past, first(ks), first(vs), offsets=o, q=first(qs), rotary=r)
    assert torch.equal(q, ops.rope(first(qs), r, offsets=o))
    prompt = ops.causal_attn_fwd(q, ops.rope(first(ks), r, offsets=o), first(vs), o)
    past.copy_(lens_of(lengths))
    last, _ = ops.cache_attn(torch.stack([q[int(o[b + 1]) - 1] for b in range(B)]), c, table, past, save=True)
    for b in range(B):
        within("prompt", last[b], prompt[int(o[b + 1]) - 1].double(), 8 * half_step(prompt[int(o[b + 1]) - 1]) + 2.0 ** -6)
    tq, tk, tv = (torch.zeros((B, h, dh), dtype=torch.bfloat16, device="cuda") for h in (H, Hk, Hk))
    out, rq = torch.zeros_like(tq), torch.zeros_like(tq)
    longest = max(room)
    ws = ops.cache_attn_workspace(c, B, H, longest)

    def step():
        ops.kv_append(c, table, past, tk, tv, q=tq, rotary=r, q_out=rq)
        past.add_(1)
        ops.cache_attn(rq, c, table, past, max_len=longest, out=out, workspace=ws)

    g = torch.cuda.CUDAGraph()
    keep = past.clone()
    with torch.cuda.graph(g):
        step()
    past.copy_(keep)
    for i in range(steps):
        for t, x in ((tq, qs), (tk, ks), (tv, vs)):
            t.copy_(torch.stack([x[b][lengths[b] + i] for b in range(B)]))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        for b in range(B):
            n = lengths[b] + i + 1
            one = offsets_of([n])
            rk, rqq = ops.rope(ks[b][:n], r, offsets=one), ops.rope(qs[b][:n], r, offsets=one)
            want, _, eo, _ = expect(rqq[-1:], [rk], [vs[b][:n]], dh ** -0.5)
            within("step", out[b], want[0], half_step(out[b]) + eo[0] * (1 + 2.0 ** -7))


# ------------------------------------------------------------------ infinite values

@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("n", [1, 17, 31, 32, 33, 300, 3000])
def test_infinite_values_stay_infinite(n, dh):
    """An infinite value of a sequence's first or last token is the sum, with its sign, of its feature and of no other, wherever
    the sequence ends in a tile of keys."""
    for at in {0, n - 1}:
        c, table, ks, vs = make_cache([n], 2, 16, dh)
        page, row = int(table[0, at // 16]), at % 16
        c.values[page, 0, row, 5], c.values[page, 1, row, dh - 1] = torch.inf, -torch.inf
        q = heads((1, 4, dh), 9)
        out, lse = ops.cache_attn(q, c, table, lens_of([n]), save=True)
        assert (out[0, :2, 5] == torch.inf).all() and (out[0, 2:, dh - 1] == -torch.inf).all()
        want, wl, eo, el = expect(q, ks, vs, dh ** -0.5)             # (of the values without infinities)
        keep = torch.isfinite(out)
        assert int((~keep).sum()) == 4
        within("out", out[keep], want[keep], half_step(out[keep]) + eo[keep] * (1 + 2.0 ** -7))
        within("lse", lse, wl, el)


@pytest.mark.parametrize("page", [16, 32])
def test_infinite_values_beside_missing_pages(page):
    """The tokens on either side of a missing page hold an infinity: copies of them stand in for the absent ones."""
    n, lost = 6 * page, 3
    c, table, ks, vs = make_cache([n], 2, page, 64)
    q = heads((1, 4, 64), 9)
    c.values[int(table[0, lost - 1]), :, page - 1, 3] = torch.inf
    c.values[int(table[0, lost + 1]), :, 0, 40] = -torch.inf
    table[0, lost] = -1
    m = torch.ones(n, dtype=torch.bool, device="cuda")
    m[lost * page:(lost + 1) * page] = False
    out = ops.cache_attn(q, c, table, lens_of([n]))
    assert (out[..., 3] == torch.inf).all() and (out[..., 40] == -torch.inf).all()
    want, _, eo, _ = expect(q, [ks[0][m]], [vs[0][m]], 0.125)
    keep = torch.isfinite(out)
    assert int((~keep).sum()) == 8
    within("out", out[keep], want[keep], half_step(out[keep]) + eo[keep] * (1 + 2.0 ** -7))


@pytest.mark.parametrize("H, Hk, dh, B", [(8, 2, 128, 2), (8, 2, 64, 9), (40, 1, 32, 3)])
def test_one_workspace_for_a_session(H, Hk, dh, B):
    """A workspace for the longest history serves every step before, with a tight max_len, and every smaller batch; nothing is
    written behind it."""
    lengths = [9000 - 700 * b for b in range(B)]
    c, table, ks, vs = make_cache(lengths, Hk, 64, dh)
    n = ops.cache_attn_workspace(c, B, H, 9000).numel()
    room = torch.full((n + 4096,), 93, dtype=torch.uint8, device="cuda")
    ws = room[:n]
    q = heads((B, H, dh), 5)
    for longest in (1, 1024, 1025, 1152, 1153, 4096, 4097, 8192, 8193, 9000):
        for m in sorted({1, B // 2, B}):
            some = [min(longest, x) for x in lengths[:m]]
            out, lse = ops.cache_attn(q[:m], c, table[:m], lens_of(some), max_len=longest, save=True, workspace=ws)
            assert (room[n:] == 93).all()
            if longest in (1153, 8193):
                compare(q[:m], [k[:x] for k, x in zip(ks, some)], [v[:x] for v, x in zip(vs, some)], out, lse, dh ** -0.5)


@pytest.mark.parametrize("H, Hk, dh", [(40, 1, 128), (70, 2, 64), (33, 1, 32)])
def test_many_query_heads_over_several_chunks(H, Hk, dh):
    """More query heads of a key head than one product has columns, and more keys than one workgroup takes."""
    check([5000, 1, 0, 2049], H, Hk, dh, 32, max_len=5000)
