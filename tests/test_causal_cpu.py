"""Refusals of the entry points of include/mtgr_causal.h on the CPU (every bad argument is a status before any device call;
pointers are fake addresses that nothing reads), the rotary frequencies, and the 64-bit definitions that the GPU tests
compare with, against differences."""
import ctypes
import math

import pytest
import torch

from paper_2505_18654_amd import hstu, ops
from tests.causal_ref import causal, causal_back, rotate

FAKE = 0x7f0000000000
BIG = 1 << 40
NULL, INVALID, UNSUPPORTED, SMALL = (hstu.MTGR_ERROR_NULL_POINTER, hstu.MTGR_ERROR_INVALID_ARGUMENT,
                                     hstu.MTGR_ERROR_UNSUPPORTED, hstu.MTGR_ERROR_WORKSPACE_TOO_SMALL)
INF, NAN = float("inf"), float("nan")


def status_of(call, *args, **kw):
    with pytest.raises(hstu.MtgrError) as e:
        call(*args, **kw)
    assert hstu.mtgr_last_error_message()
    return e.value.status


def test_struct_layouts():
    for t, size, field, offset in ((hstu.RopeProblem, 56, "ld_x", 40), (hstu.CausalProblem, 72, "ld_q", 32),
                                   (hstu.KvCachePages, 40, "keys", 24), (hstu.KvAppendProblem, 72, "ld_table", 32),
                                   (hstu.CacheAttnProblem, 48, "max_len", 16)):
        assert ctypes.sizeof(t) == size and getattr(t, field).offset == offset, t


# ------------------------------------------------------------------ rotary positions

def rope(**kw):
    a = dict(x=FAKE, positions=FAKE, offsets=None, freqs=FAKE, out=FAKE, stream=0)
    args = {n: kw.pop(n) for n in list(kw) if n in a}
    a.update(args)
    p = dict(num_tokens=10, num_seqs=2, heads=4, head_dim=64, rot_dim=64, layout=0, dtype=0, inverse=0, amplitude=1.0, ld_x=256,
             ld_out=256)
    p.update(kw)
    hstu.mtgr_rope(hstu.RopeProblem(**p), **a)


@pytest.mark.parametrize("kw, status", [
    (dict(num_tokens=-1), INVALID), (dict(num_tokens=1 << 31), INVALID), (dict(num_seqs=-1), INVALID),
    (dict(num_tokens=1 << 30), UNSUPPORTED), (dict(num_tokens=1 << 29, dtype=1, ld_x=512), UNSUPPORTED),
    (dict(heads=0), INVALID), (dict(heads=65536), INVALID), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED),
    (dict(head_dim=1032), UNSUPPORTED), (dict(rot_dim=0), UNSUPPORTED), (dict(rot_dim=24), UNSUPPORTED),
    (dict(rot_dim=80), UNSUPPORTED), (dict(rot_dim=-16), UNSUPPORTED), (dict(layout=2), INVALID), (dict(dtype=7), UNSUPPORTED),
    (dict(amplitude=INF), INVALID), (dict(amplitude=NAN), INVALID), (dict(ld_x=255), INVALID), (dict(ld_x=260), INVALID),
    (dict(ld_x=1 << 22), UNSUPPORTED), (dict(ld_out=128), INVALID), (dict(x=None), NULL), (dict(out=None), NULL),
    (dict(x=FAKE + 8), INVALID), (dict(positions=None), NULL), (dict(offsets=FAKE), INVALID),
    (dict(positions=FAKE + 2), INVALID), (dict(positions=None, offsets=FAKE + 1), INVALID), (dict(freqs=None), NULL),
    (dict(freqs=FAKE + 4), INVALID), (dict(ld_out=512), INVALID),            # in place with another stride
])
def test_rope_refused(kw, status):
    assert status_of(rope, **kw) == status


def test_rope_of_nothing():
    rope(num_tokens=0, x=None, out=None, positions=None)
    rope(num_seqs=0, positions=None, offsets=FAKE)


@pytest.mark.parametrize("kw", [
    dict(rot_dim=8), dict(rot_dim=1040), dict(base=1.0), dict(base=INF), dict(base=NAN), dict(scaling=4), dict(scaling=-1),
    dict(scaling=1, factor=0.5), dict(scaling=2, factor=INF), dict(scaling=3, factor=NAN), dict(scaling=3, factor=2.0),
    dict(scaling=3, factor=2.0, trained_len=100, slow=-1.0), dict(scaling=3, factor=2.0, trained_len=100, slow=2.0, fast=2.0),
    dict(scaling=3, factor=2.0, trained_len=100, fast=INF),
])
def test_frequencies_refused(kw):
    a = dict(rot_dim=64, base=1e4)
    a.update(kw)
    assert status_of(hstu.mtgr_rope_frequencies, **a) in (INVALID, UNSUPPORTED)


def test_frequencies():
    r, base, s, L = 64, 10000.0, 8.0, 1024
    plain = [base ** (-2 * i / r) for i in range(r // 2)]
    near = lambda got, want: all(abs(g - w) <= 1e-14 * w for g, w in zip(got, want, strict=True))  # noqa: E731
    f, a = hstu.mtgr_rope_frequencies(r, base)
    assert near(f, plain) and a == 1.0
    f, a = hstu.mtgr_rope_frequencies(r, base, hstu.MTGR_ROPE_LINEAR, s)
    assert near(f, [x / s for x in plain]) and a == 1.0
    f, a = hstu.mtgr_rope_frequencies(r, base, hstu.MTGR_ROPE_BASE, s)
    assert f[0] == 1.0 and abs(f[-1] * s / plain[-1] - 1) < 1e-12 and a == 1.0
    f, a = hstu.mtgr_rope_frequencies(r, base, hstu.MTGR_ROPE_PARTS, s, L, 1.0, 32.0)
    for got, x in zip(f, plain):
        turns = L * x / (2 * math.pi)
        keep = 0.0 if turns <= 1 else 1.0 if turns >= 32 else (turns - 1) / 31
        assert abs(got - x * (keep + (1 - keep) / s)) <= 1e-13 * x
    assert abs(a - (0.1 * math.log(s) + 1)) < 1e-7 and f[0] == plain[0] and abs(f[-1] * s / plain[-1] - 1) < 1e-12
    assert ops.rotary(16, device="cpu").freqs.dtype == torch.float64
    with pytest.raises(ValueError):
        ops.rotary(16, scaling="longer", device="cpu")


# ------------------------------------------------------------------ causal attention

def causal_problem(**kw):
    p = dict(num_seqs=3, heads=4, kv_heads=2, head_dim=64, total_tokens=100, scale=0.125, reserved=0, ld_q=256, ld_k=128,
             ld_v=128, ld_o=256, ld_do=256)
    p.update(kw)
    return hstu.CausalProblem(**p)


FWD = dict(offsets=FAKE, q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=FAKE, stream=0)
BWD = dict(FWD, workspace=FAKE, workspace_bytes=BIG, dout=FAKE, dq=FAKE, dk=FAKE, dv=FAKE)


def split(base, kw):
    a = {n: kw.get(n, v) for n, v in base.items()}
    return {n: v for n, v in kw.items() if n not in base}, a


def causal_fwd(**kw):
    p, a = split(FWD, kw)
    hstu.mtgr_causal_attn_fwd(causal_problem(**p), **a)


def causal_bwd(**kw):
    p, a = split(BWD, kw)
    hstu.mtgr_causal_attn_bwd(causal_problem(**p), **a)


@pytest.mark.parametrize("call", [causal_fwd, causal_bwd])
@pytest.mark.parametrize("kw, status", [
    (dict(num_seqs=-1), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(kv_heads=3), INVALID),
    (dict(kv_heads=8), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=16), UNSUPPORTED),
    (dict(head_dim=256), UNSUPPORTED), (dict(total_tokens=-1), INVALID), (dict(total_tokens=1 << 30), INVALID),
    (dict(total_tokens=1 << 29, heads=64, kv_heads=64), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(scale=3e38), INVALID), (dict(reserved=1), INVALID),
    (dict(num_seqs=2 ** 31 - 1), UNSUPPORTED), (dict(num_seqs=(1 << 24) - (1 << 17), heads=1, kv_heads=1), UNSUPPORTED),
    (dict(ld_q=255), INVALID), (dict(ld_q=260), INVALID), (dict(ld_k=127), INVALID), (dict(ld_v=1 << 22), UNSUPPORTED),
    (dict(ld_o=248), INVALID), (dict(offsets=None), NULL), (dict(offsets=FAKE + 2), INVALID), (dict(q=None), NULL),
    (dict(k=None), NULL), (dict(v=FAKE + 2), INVALID), (dict(out=None), NULL), (dict(lse=FAKE + 2), INVALID),
])
def test_causal_refused(call, kw, status):
    assert status_of(call, **kw) == status


@pytest.mark.parametrize("kw, status", [
    (dict(lse=None), NULL), (dict(dout=None), NULL), (dict(ld_do=128), INVALID), (dict(dq=None), NULL), (dict(dk=None), NULL),
    (dict(dv=FAKE + 8), INVALID), (dict(workspace=None), NULL), (dict(workspace=FAKE + 64), INVALID),
    (dict(workspace_bytes=1599), SMALL),
])
def test_causal_backward_refused(kw, status):
    assert status_of(causal_bwd, **kw) == status


def test_largest_launch():
    most = (1 << 24) - (1 << 17)
    assert hstu.mtgr_causal_attn_workspace_size(causal_problem(num_seqs=most - 1, heads=1, kv_heads=1)) > 0
    p = hstu.CacheAttnProblem(num_seqs=2048, heads=4094, max_pages=1 << 25, scale=0.125, max_len=(1 << 31) - 4097,
                              ld_table=1 << 25, ld_q=0, ld_o=0)
    assert hstu.mtgr_cache_attn_workspace_size(p, pages(page_size=4096, kv_heads=4094)) > 0


def test_causal_of_nothing():
    for call in (causal_fwd, causal_bwd):
        call(total_tokens=0, q=None, k=None, v=None, out=None, offsets=None)
        call(num_seqs=0, q=None, offsets=None)


# ------------------------------------------------------------------ paged cache

def pages(**kw):
    c = dict(num_pages=9, page_size=32, kv_heads=2, head_dim=64, reserved=0, keys=FAKE, values=FAKE)
    c.update(kw)
    return hstu.KvCachePages(**c)


APPEND = dict(page_table=FAKE, past=FAKE, offsets=FAKE, q=FAKE, k=FAKE, v=FAKE, freqs=FAKE, q_out=FAKE, stream=0)


def append(cache=None, **kw):
    p, a = split(APPEND, kw)
    base = dict(num_tokens=10, num_seqs=3, heads=4, max_pages=5, rot_dim=64, layout=0, amplitude=1.0, ld_table=5, ld_q=256,
                ld_q_out=256, ld_k=128, ld_v=128)
    base.update(p)
    hstu.mtgr_kv_append(hstu.KvAppendProblem(**base), cache or pages(), **a)


BAD_CACHE = [(dict(num_pages=0), INVALID), (dict(num_pages=1 << 31), INVALID), (dict(page_size=8), UNSUPPORTED),
             (dict(page_size=48), UNSUPPORTED), (dict(page_size=8192), UNSUPPORTED), (dict(page_size=-32), UNSUPPORTED),
             (dict(kv_heads=0), INVALID), (dict(reserved=1), INVALID), (dict(keys=None), NULL), (dict(values=None), NULL),
             (dict(values=FAKE + 8), INVALID)]


@pytest.mark.parametrize("kw, status", BAD_CACHE + [(dict(head_dim=60), UNSUPPORTED), (dict(head_dim=1032), UNSUPPORTED)])
def test_append_cache_refused(kw, status):
    assert status_of(append, cache=pages(**kw)) == status


@pytest.mark.parametrize("kw, status", [
    (dict(num_tokens=-1), INVALID), (dict(num_tokens=1 << 31), INVALID), (dict(num_seqs=-1), INVALID), (dict(heads=-1), INVALID),
    (dict(max_pages=0), INVALID), (dict(rot_dim=24), UNSUPPORTED), (dict(rot_dim=80), UNSUPPORTED), (dict(layout=5), INVALID),
    (dict(amplitude=NAN), INVALID), (dict(ld_table=4), INVALID), (dict(ld_q=252), INVALID), (dict(ld_q_out=1 << 22), UNSUPPORTED),
    (dict(ld_k=64), INVALID), (dict(ld_v=132), INVALID), (dict(offsets=None), INVALID), (dict(offsets=FAKE + 2), INVALID),
    (dict(page_table=None), NULL), (dict(past=None), NULL), (dict(past=FAKE + 1), INVALID), (dict(k=None), NULL),
    (dict(v=None), NULL), (dict(q=None), NULL), (dict(q_out=None), NULL), (dict(heads=0), INVALID), (dict(freqs=None), NULL),
    (dict(ld_q=512), INVALID), (dict(num_tokens=1 << 30), UNSUPPORTED),
])
def test_append_refused(kw, status):
    assert status_of(append, **kw) == status


def test_append_of_nothing():
    append(num_tokens=0, page_table=None)
    append(num_seqs=0, page_table=None)


def cache_attn(cache=None, **kw):
    p, a = split(dict(page_table=FAKE, lens=FAKE, q=FAKE, out=FAKE, lse=FAKE, workspace=FAKE, workspace_bytes=BIG, stream=0), kw)
    base = dict(num_seqs=3, heads=4, max_pages=5, scale=0.125, max_len=160, ld_table=5, ld_q=256, ld_o=256)
    base.update(p)
    hstu.mtgr_cache_attn(hstu.CacheAttnProblem(**base), cache or pages(), **a)


@pytest.mark.parametrize("kw, status", BAD_CACHE + [(dict(head_dim=96), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED)])
def test_cache_attn_cache_refused(kw, status):
    assert status_of(cache_attn, cache=pages(**kw)) == status


@pytest.mark.parametrize("kw, status", [
    (dict(num_seqs=-1), INVALID), (dict(num_seqs=65536), INVALID), (dict(heads=0), INVALID), (dict(heads=3), INVALID),
    (dict(num_seqs=4096, heads=32768), UNSUPPORTED), (dict(num_seqs=4096, heads=2048), UNSUPPORTED),
    (dict(max_pages=0), INVALID), (dict(scale=0.0), INVALID), (dict(scale=NAN), INVALID), (dict(max_len=-1), INVALID),
    (dict(max_len=161), INVALID), (dict(max_pages=1 << 30, ld_table=1 << 30, max_len=1 << 31), INVALID), (dict(ld_table=4), INVALID),
    (dict(ld_q=128), INVALID), (dict(ld_o=252), INVALID), (dict(page_table=None), NULL), (dict(page_table=FAKE + 2), INVALID),
    (dict(lens=None), NULL), (dict(q=None), NULL), (dict(out=FAKE + 2), INVALID), (dict(lse=FAKE + 2), INVALID),
    (dict(workspace=None, max_pages=5000, ld_table=5000, max_len=150000), NULL),
    (dict(workspace_bytes=256, max_pages=5000, ld_table=5000, max_len=150000), SMALL),
    (dict(workspace=FAKE + 16, max_pages=5000, ld_table=5000, max_len=150000), INVALID),
])
def test_cache_attn_refused(kw, status):
    assert status_of(cache_attn, **kw) == status


def test_cache_attn_of_nothing():
    cache_attn(num_seqs=0, page_table=None, q=None)


# ------------------------------------------------------------------ the definitions

def random(*shape, seed=1):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def test_gradients_of_the_definition():
    """causal_back against autograd and against central differences of causal."""
    lengths, H, Hk, dh, scale = [5, 1, 0, 7], 4, 2, 8, 0.4
    T = sum(lengths)
    q, k, v, g = random(T, H, dh), random(T, Hk, dh, seed=2), random(T, Hk, dh, seed=3), random(T, H, dh, seed=4)
    out, lse = causal(q, k, v, lengths, scale)[:2]
    grads = causal_back(g, q, k, v, out, lse, lengths, scale)
    for i, (name, t) in enumerate((("dq", q), ("dk", k), ("dv", v))):
        d = random(*t.shape, seed=7 + i)
        h = 1e-6
        up, down = ([x + s * h * d if x is t else x for x in (q, k, v)] for s in (1, -1))
        slope = ((causal(*up, lengths, scale)[0] - causal(*down, lengths, scale)[0]) * g).sum() / (2 * h)
        assert abs(slope - (grads[name][0] * d).sum()) < 1e-7 * (grads[name][0].abs() * d.abs()).sum()
    a = 0
    for n in lengths:
        if n == 0:
            continue
        x = [t[a:a + n].clone().requires_grad_() for t in (q, k, v)]
        kk, vv = (t.repeat_interleave(H // Hk, 1) for t in x[1:])
        z = torch.einsum("ihd,jhd->hij", x[0], kk) * scale
        p = torch.softmax(z.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -INF), -1)
        (torch.einsum("hij,jhd->ihd", p, vv) * g[a:a + n]).sum().backward()
        for t, name in zip(x, ("dq", "dk", "dv")):
            assert torch.allclose(t.grad, grads[name][0][a:a + n], atol=1e-12)
        a += n


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_of_the_definition(layout):
    """Scores of rotated queries and keys depend on the distance alone, lengths are kept, and turning back undoes it."""
    f = torch.tensor(hstu.mtgr_rope_frequencies(16, 100.0)[0], dtype=torch.float64)
    x, y = random(1, 1, 24, seed=5), random(1, 1, 24, seed=6)
    at = lambda t, p: rotate(t, f, torch.tensor([p]), 1.0, layout)[0]  # noqa: E731
    assert torch.allclose((at(x, 9) * at(y, 4)).sum(), (at(x, 105) * at(y, 100)).sum())
    assert torch.allclose(at(x, 77).norm(), x.norm()) and torch.allclose(at(at(x, 31), -31), x)
    assert torch.equal(at(x, 5)[..., 16:], x[..., 16:])


# ------------------------------------------------------------------ the torch-facing checks

def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("call", [
    lambda: ops.rope(bf(4, 2, 32), ops.rotary(16, device="cpu"), positions=i32(4)),                      # not on the device
    lambda: ops.rope(torch.zeros(4, 2, 32, dtype=torch.float16), ops.rotary(16, device="cpu"), positions=i32(4)),
    lambda: ops.causal_attn_fwd(bf(4, 2, 64), bf(4, 2, 64), bf(4, 2, 64), i32(2)),
    lambda: ops.causal_attn_fwd(bf(4, 128), bf(4, 2, 64), bf(4, 2, 64), i32(2)),
    lambda: ops.causal_attn_bwd(bf(4, 2, 64), bf(4, 2, 64), bf(4, 2, 64), bf(4, 2, 64), bf(4, 2, 64), torch.zeros(2, 4), i32(2)),
    lambda: ops.kv_append(ops.KvCache.empty(2, 1, 16, 32, device="cpu"), i32(1, 2), i32(1), bf(1, 1, 32), bf(1, 1, 32)),
    lambda: ops.cache_attn(bf(1, 2, 32), ops.KvCache.empty(2, 1, 16, 32, device="cpu"), i32(1, 2), i32(1)),
])
def test_operands_refused_before_the_library(call):
    with pytest.raises((ValueError, TypeError)):
        call()


@pytest.fixture
def on_cpu(monkeypatch):
    """The checks as if the CPU were the current device; no entry point of the library is reached."""
    monkeypatch.setattr(ops, "_device", lambda: -1)
    for name in ("mtgr_rope", "mtgr_causal_attn_fwd", "mtgr_causal_attn_bwd", "mtgr_kv_append", "mtgr_cache_attn"):
        monkeypatch.setattr(hstu, name, lambda *a, **k: None)


ROT = lambda: ops.rotary(16, device="cpu")  # noqa: E731
CACHE = lambda: ops.KvCache.empty(3, 2, 16, 32, device="cpu")  # noqa: E731


def test_operands_accepted(on_cpu):
    assert ops.rope(bf(4, 2, 32), ROT(), positions=i32(4)).shape == (4, 2, 32)
    assert ops.causal_attn_fwd(bf(4, 6, 96)[:, :4, :64].contiguous(), bf(4, 2, 64), bf(4, 2, 64), i32(3)).shape == (4, 4, 64)
    out = ops.kv_append(CACHE(), i32(3, 2), i32(3), bf(3, 2, 32), bf(3, 2, 32), q=bf(3, 4, 32), rotary=ROT())
    assert out.shape == (3, 4, 32)
    assert [t.shape for t in ops.cache_attn(bf(3, 4, 32), CACHE(), i32(3, 2), i32(3), save=True)] == [(3, 4, 32), (3, 4)]


@pytest.mark.parametrize("call", [
    lambda: ops.rope(bf(4, 2, 32), ROT()),
    lambda: ops.rope(bf(4, 2, 32), ROT(), positions=i32(4), offsets=i32(2)),
    lambda: ops.rope(bf(4, 2, 32), ROT(), positions=i32(5)),
    lambda: ops.rope(bf(4, 2, 32), ROT(), positions=torch.zeros(4, dtype=torch.int64)),
    lambda: ops.rope(bf(4, 2, 32), ROT(), offsets=torch.zeros(0, dtype=torch.int32)),
    lambda: ops.rope(bf(4, 2, 32), ops.Rotary(torch.zeros(8)), positions=i32(4)),
    lambda: ops.rope(bf(4, 2, 32), ops.Rotary(ROT().freqs, "diagonal"), positions=i32(4)),
    lambda: ops.rope(bf(4, 2, 64)[..., ::2], ROT(), positions=i32(4)),
    lambda: ops.rope(bf(4, 2, 64)[..., :32], ROT(), positions=i32(4)),                     # heads with gaps
    lambda: ops.rope(bf(1, 2, 32).expand(4, 2, 32), ROT(), positions=i32(4)),              # rows that overlap
    lambda: ops.rope(bf(4, 2, 32), ROT(), positions=i32(4), out=bf(4, 3, 32)),
    lambda: ops.causal_attn_fwd(bf(4, 2, 64), bf(5, 2, 64), bf(5, 2, 64), i32(2)),
    lambda: ops.causal_attn_fwd(bf(4, 2, 64), bf(4, 2, 32), bf(4, 2, 32), i32(2)),
    lambda: ops.causal_attn_fwd(bf(4, 2, 64), bf(4, 2, 64), bf(4, 1, 64), i32(2)),
    lambda: ops.causal_attn_fwd(bf(4, 2, 64), bf(4, 2, 64), bf(4, 2, 64), i32(2, 2)),
    lambda: ops.causal_attn_fwd(bf(4, 2, 64), bf(4, 2, 64), bf(4, 2, 64), i32(2), lse=torch.zeros(4, 2)),
    lambda: ops.causal_attn_bwd(*[bf(4, 2, 64)] * 5, torch.zeros(4, 2), i32(2)),
    lambda: ops.causal_attn_bwd(*[bf(4, 2, 64)] * 5, torch.zeros(2, 4), i32(2), grads=(bf(4, 3, 64)[:, :2], bf(4, 2, 64), bf(4, 2, 64))),
    lambda: ops.KvCache(bf(3, 2, 16, 32), bf(3, 2, 16, 64)).struct(-1),
    lambda: ops.KvCache(bf(3, 2, 16, 64)[..., :32], bf(3, 2, 16, 32)).struct(-1),
    lambda: ops.KvCache(torch.zeros(3, 2, 16, 32), torch.zeros(3, 2, 16, 32)).struct(-1),
    lambda: ops.kv_append(CACHE(), i32(3), i32(3), bf(3, 2, 32), bf(3, 2, 32)),
    lambda: ops.kv_append(CACHE(), i32(3, 2), i32(2), bf(3, 2, 32), bf(3, 2, 32)),
    lambda: ops.kv_append(CACHE(), i32(3, 2), i32(3), bf(3, 3, 32), bf(3, 3, 32)),
    lambda: ops.kv_append(CACHE(), i32(3, 2), i32(3), bf(3, 2, 32), bf(4, 2, 32)),
    lambda: ops.kv_append(CACHE(), i32(3, 2), i32(3), bf(3, 2, 32), bf(3, 2, 32), offsets=i32(3)),
    lambda: ops.kv_append(CACHE(), i32(3, 2), i32(3), bf(3, 2, 32), bf(3, 2, 32), q_out=bf(3, 2, 32)),
    lambda: ops.kv_append(CACHE(), i32(3, 2), i32(3), bf(3, 2, 32), bf(3, 2, 32), q=bf(2, 4, 32)),
    lambda: ops.cache_attn(bf(2, 4, 32), CACHE(), i32(3, 2), i32(3)),
    lambda: ops.cache_attn(bf(3, 4, 64), CACHE(), i32(3, 2), i32(3)),
    lambda: ops.cache_attn(bf(3, 4, 32), CACHE(), i32(3, 2), i32(2)),
    lambda: ops.cache_attn(bf(3, 4, 32), CACHE(), i32(1, 2).expand(3, 2), i32(3)),
    lambda: ops.cache_attn(bf(3, 4, 32), CACHE(), i32(3, 2).long(), i32(3)),
])
def test_operands_that_do_not_fit(on_cpu, call):
    with pytest.raises(ValueError):
        call()


# ------------------------------------------------------------------ workspaces of a session's largest call

@pytest.mark.parametrize("H, Hk, dh", [(8, 2, 128), (1, 1, 32), (33, 1, 64), (70, 2, 64), (32, 8, 128), (24, 24, 64), (600, 300, 32)])
def test_cache_workspace_of_the_largest_call(H, Hk, dh):
    """One sized for the longest history and the most sequences is enough for every smaller call."""
    def size(B, n):
        p = hstu.CacheAttnProblem(num_seqs=B, heads=H, max_pages=1 << 20, scale=0.125, max_len=n, ld_table=1 << 20, ld_q=0, ld_o=0)
        return hstu.mtgr_cache_attn_workspace_size(p, pages(page_size=1024, kv_heads=Hk, head_dim=dh))

    lens = sorted({0, 1, 1024, 1025, 8192, 9000, 32768, 32769, 65536, 100003, 1 << 24, (1 << 30) - 1,
                   *range(900, 40000, 331), *(2 ** i + d for i in range(10, 30) for d in (-1, 0, 1))})
    batches = [0, 1, 2, 3, 4, 5, 7, 8, 15, 31, 64, 100, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000, 4096, 10000]
    before = [0] * len(lens)
    for B in batches:
        row = [size(B, n) for n in lens]
        assert all(a <= b for a, b in zip(row, row[1:])), B
        assert all(a <= b for a, b in zip(before, row)), B
        before = row


def test_backward_workspace_of_the_largest_call():
    def size(T, B, H, Hk, dh):
        return hstu.mtgr_causal_attn_workspace_size(causal_problem(total_tokens=T, num_seqs=B, heads=H, kv_heads=Hk, head_dim=dh,
                                                                   ld_q=H * dh, ld_k=Hk * dh, ld_v=Hk * dh, ld_o=H * dh, ld_do=H * dh))

    for H, Hk, dh in ((8, 2, 128), (1, 1, 32), (16, 16, 64), (2048, 2048, 32)):
        before = [0] * 7
        for T in (0, 1, 31, 128, 129, 700, 3000, 3001, 20000, 70000, 500000):
            row = [size(T, B, H, Hk, dh) for B in (0, 1, 2, 3, 50, 64, 1000)]
            assert all(a <= b for a, b in zip(row, row[1:])) and all(a <= b for a, b in zip(before, row)), (H, T)
            before = row


def test_addresses_of_int_subclasses():
    """An address may be any int, for every entry point."""
    class Address(int):
        pass

    assert hstu._ptr(Address(FAKE)) == FAKE and hstu._ptr(FAKE) == FAKE and hstu._ptr(None) is None
    assert status_of(rope, x=Address(FAKE), out=Address(FAKE + 8)) == INVALID
    rope(num_tokens=0, x=Address(FAKE))
