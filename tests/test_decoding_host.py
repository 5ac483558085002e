"""Heads, the cache in 4 bits, attention over it and the draw of a token without a GPU: pins of the oracle, size queries, refusals."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2310_15929_amd as esp
from oracle import decoding_oracle as orc
from paper_2310_15929_amd import binding

EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -7
P = 1 << 20   # stands for device pointers a long way apart: aligned, never followed


def _at(i):
    return P + (i << 36)


@pytest.fixture(scope="module")
def ctx():
    return esp.Context(0)


# ---- oracle ---------------------------------------------------------------------------------------
def test_rotation_of_one_pair():
    x = np.array([[[3.0, 4.0, 5.0]]])
    y = orc.rotate(x, None, 0, np.array([1]), np.array([math.pi / 2]), False)
    assert np.allclose(y, [[[-4.0, 3.0, 5.0]]], atol=1e-12)
    a, b = (orc.rotate(np.arange(8.0).reshape(1, 1, 8), None, 0, np.array([2]), np.array([0.3, 0.1, 0.2, 0.5]), paired) for paired in (False, True))
    c, s = math.cos(0.2), math.sin(0.2)
    assert math.isclose(a[0, 0, 1], 1 * c - 5 * s) and math.isclose(a[0, 0, 5], 5 * c + 1 * s) and math.isclose(b[0, 0, 2], 2 * c - 3 * s) and math.isclose(b[0, 0, 3], 3 * c + 2 * s)


def test_rotation_keeps_products_of_equal_distance():
    rng = np.random.default_rng(3)
    q, k, f = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16)), np.float32(0.9) ** np.arange(8)
    one, two = ((orc.rotate(q, None, 0, np.array([p + 5]), f, False) * orc.rotate(k, None, 0, np.array([p]), f, False)).sum() for p in (0, 1000))
    assert math.isclose(one, two, rel_tol=1e-9)


@pytest.mark.parametrize("D", [1, 33, 64, 80, 128, 200, 256])
def test_rows_of_the_cache_go_back_and_forth(D):
    x = np.random.default_rng(D).standard_normal((3, 2, D))
    d, s = orc.cache_rows(x)
    assert d.shape == (3, 2, orc.row_of(D) // 2) and s.shape == (3, 2, orc.row_of(D) // 32)
    v = orc.cache_values(d, s, D)
    e, t = orc.cache_rows(v)
    assert np.array_equal(orc.cache_values(e, t, D), v) and np.abs(v - x).max() <= np.abs(x).max() / 4


def test_attention_of_one_and_of_equal_tokens():
    v = np.arange(12.0).reshape(3, 4)
    out, lse, *_ = orc.attend(np.ones((3, 4)), np.ones((3, 4)), v, 0.5, [-1, 0, 2])
    assert (out[0] == 0).all() and lse[0] == -np.inf and np.array_equal(out[1], v[0]) and np.allclose(out[2], v.mean(0)) and math.isclose(lse[2], 2 + math.log(3))


def test_worked_draw():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert orc.sample(x, 0.05)[0] == 0 and orc.sample(x, 0.3)[0] == 1 and orc.sample(x, 0.65)[0] == 2 and orc.sample(x, 0.99)[0] == 3
    assert list(orc.sample(x, 0.5, top_k=2)[2]) == [1, 3] and list(orc.sample(x, 0.5, top_p=0.75)[2]) == [1, 2, 3] and list(orc.sample(x, 0.5, min_p=0.5 - 1e-9)[2]) == [1, 2, 3]
    token, lp, kept = orc.sample(x, 0.9, top_k=3, top_p=0.5)     # 4/9 has come before the second
    assert list(kept) == [1, 3] and token == 3 and math.isclose(lp, math.log(3 / 7))
    assert orc.sample(np.array([1.0, 5.0, 5.0]), 0.9, 0.0) == (1, 0.0, [1])


# ---- sizes ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("D,row", [(1, 64), (64, 64), (65, 128), (128, 128), (129, 256), (256, 256)])
def test_cache_sizes(D, row):
    assert esp.cache_size(7, 16, 3, D) == (7 * 16 * 3 * row // 2, 7 * 16 * 3 * row // 32) and esp.cache_size(0, 16, 3, D) == (0, 0)


@pytest.mark.parametrize("call", [
    lambda: esp.cache_size(-1, 16, 1, 64), lambda: esp.cache_size(1, 8, 1, 64), lambda: esp.cache_size(1, 48, 1, 64), lambda: esp.cache_size(1, 2048, 1, 64),
    lambda: esp.cache_size(1, 16, 0, 64), lambda: esp.cache_size(1, 16, 1, 0), lambda: esp.cache_size(1, 16, 1, 257), lambda: esp.cache_size(1 << 27, 16, 1, 64),
    lambda: esp.cache_attention_workspace(4, 16, 2, 64, 3, 3, 3, 1, False), lambda: esp.cache_attention_workspace(4, 16, 2, 64, 3, 2, 4, 1, False),
    lambda: esp.cache_attention_workspace(4, 16, 2, 64, -1, 2, 4, 1, True), lambda: esp.cache_attention_workspace(4, 16, 2, 64, 1, 1, 4, -1, True),
    lambda: esp.cache_attention_workspace(4, 16, 2, 64, 1 << 22, 1, 4, 1, True), lambda: esp.cache_attention_workspace(4, 16, 2, 64, 1, 1, 4, 1 << 27, True),
    lambda: esp.sample_workspace(-1, 5), lambda: esp.sample_workspace(1, 0), lambda: esp.sample_workspace(1, (1 << 21) + 1), lambda: esp.sample_workspace(1 << 20, 1 << 20)])
def test_size_queries_refuse(call):
    with pytest.raises(esp.EsparseError):
        call()


def test_workspaces():
    assert esp.cache_attention_workspace(4, 16, 2, 64, 0, 5, 4, 100, True) == 0 and esp.sample_workspace(0, 100) == 0
    assert esp.sample_workspace(3, 50000) > 0
    one, two = (esp.cache_attention_workspace(4096, 64, 8, 128, 1, 1, 64, w, False) for w in (1, 2048))
    assert one == 0 and two > 0


@pytest.mark.parametrize("T,B,Hq,H,ragged", [(65536, 1, 64, 8, True), (1 << 20, 1, 64, 8, True), ((1 << 22) - 1, 1, 16, 16, True), (1 << 17, 1 << 17, 32, 32, False), (1, (1 << 22) - 1, 1, 1, True)])
def test_attention_of_many_rows_is_taken(T, B, Hq, H, ragged):
    """As many rows as a launch holds: 2^26 of all heads, and 2^22 heads of sequences."""
    assert esp.cache_attention_workspace(4096, 64, H, 64, T, B, Hq, 2048, ragged) >= 0
    for more in (dict(T=2 * T, B=B if ragged else 2 * B), dict(T=T if ragged else 4 * B, B=4 * B)):
        if more["T"] * Hq > 1 << 26 or more["B"] * H > 1 << 22:
            with pytest.raises(esp.EsparseError):
                esp.cache_attention_workspace(4096, 64, H, 64, more["T"], more["B"], Hq, 2048, ragged)


# ---- refusals: nothing is launched ------------------------------------------------------------------
def _rotate(ctx, rc, what=None, **change):
    a = dict(heads=(8, 2, 64, 64, 0, 1e-6), T=5, dtype=0, q=_at(0), ldq=512, qw=_at(1), k=_at(2), ldk=128, kw=_at(3), pos=_at(4), freq=_at(5), qo=_at(6), ko=None,
             v=_at(7), ldv=128, cache=(_at(8), _at(9), _at(10), _at(11), 4, 16, 2, 64), slots=_at(12))
    a.update(change)
    h, c = (binding._Heads(*a["heads"]) if a["heads"] else None), (binding._Cache(*a["cache"]) if a["cache"] else None)
    got = ctx._lib.esparse_rotate_heads(ctx._h, C.byref(h) if h else None, a["T"], a["dtype"], a["q"], a["ldq"], a["qw"], a["k"], a["ldk"], a["kw"], a["pos"], a["freq"], a["qo"], a["ko"],
                                        a["v"], a["ldv"], C.byref(c) if c else None, a["slots"])
    assert got == rc, ctx._lib.esparse_last_error(ctx._h)


CACHE = (_at(8), _at(9), _at(10), _at(11), 4, 16, 2, 64)


@pytest.mark.parametrize("change", [
    dict(heads=None), dict(T=-1), dict(T=1 << 22), dict(heads=(0, 2, 64, 64, 0, 0.0)), dict(heads=(8, 3, 64, 64, 0, 0.0)), dict(heads=(8, 2, 300, 64, 0, 0.0)),
    dict(heads=(8, 2, 0, 0, 0, 0.0)), dict(heads=(8, 2, 64, 63, 0, 0.0)), dict(heads=(8, 2, 64, 66, 0, 0.0)), dict(heads=(8, 2, 64, -2, 0, 0.0)), dict(heads=(8, 2, 64, 64, 2, 0.0)),
    dict(heads=(8, 2, 64, 64, 0, -1.0)), dict(heads=(8, 2, 64, 64, 0, math.nan)), dict(q=None), dict(qo=None), dict(k=None), dict(cache=None), dict(v=None), dict(slots=None), dict(pos=None),
    dict(freq=None), dict(ldq=511), dict(ldk=127), dict(ldv=100), dict(q=_at(0) + 1), dict(kw=_at(3) + 1), dict(pos=_at(4) + 2), dict(slots=_at(12) + 2), dict(ldq=1 << 38),
    dict(qo=_at(0)), dict(qo=_at(8)), dict(ko=_at(6) + 2), dict(ko=_at(2) + 64), dict(cache=(_at(8) + 8,) + CACHE[1:]), dict(cache=(None,) + CACHE[1:]), dict(cache=CACHE[:4] + (4, 24, 2, 64)),
    dict(cache=CACHE[:4] + (4, 16, 3, 64)), dict(cache=CACHE[:4] + (4, 16, 2, 128)), dict(cache=(_at(8), _at(8) + 16) + CACHE[2:]), dict(q=None, qo=None, qw=_at(1)),
    dict(q=None, k=None, qo=None, qw=None, kw=None, cache=None, v=None, slots=None), dict(q=_at(8) + 64), dict(v=_at(11))])
def test_rotate_heads_refuses(ctx, change):
    _rotate(ctx, EINVAL, **change)


def test_rotate_heads_of_nothing_and_of_other_types(ctx):
    _rotate(ctx, 0, T=0)
    _rotate(ctx, EUNSUPPORTED, dtype=2)
    assert ctx._lib.esparse_rotate_heads(None, None, 0, 0, *[None, 0, None] * 2, *[None] * 5, 0, None, None) == EINVAL


@pytest.mark.parametrize("rc,change", [
    (EUNSUPPORTED, dict(dtype=3)), (EINVAL, dict(cache=None)), (EINVAL, dict(T=-1)), (EINVAL, dict(slots=None)), (EINVAL, dict(k=None, v=None)), (EINVAL, dict(k=_at(8))), (EINVAL, dict(k=_at(3))),
    (EINVAL, dict(slots=_at(12) + 1)), (EINVAL, dict(v=_at(3) + 1)), (EINVAL, dict(T=1 << 21, cache=CACHE[:4] + (4, 16, 64, 64))), (0, dict(T=0))])
def test_cache_read_refuses(ctx, rc, change):
    a = dict(cache=CACHE, slots=_at(12), T=5, dtype=1, k=_at(2), v=_at(3))
    a.update(change)
    c = binding._Cache(*a["cache"]) if a["cache"] else None
    assert ctx._lib.esparse_cache_read(ctx._h, C.byref(c) if c else None, a["slots"], a["T"], a["dtype"], a["k"], a["v"]) == rc


LONG = CACHE[:4] + (4096, 64, 2, 128)


@pytest.mark.parametrize("rc,change", [
    (EUNSUPPORTED, dict(dtype=2)), (EINVAL, dict(cache=None)), (EINVAL, dict(T=6)), (EINVAL, dict(T=-1, starts=_at(5))), (EINVAL, dict(heads=7)), (EINVAL, dict(heads=0)), (EINVAL, dict(width=-1)),
    (EINVAL, dict(width=1 << 40)), (EINVAL, dict(scale=math.inf)), (EINVAL, dict(scale=1e39)), (EINVAL, dict(scale=math.nan)), (EINVAL, dict(q=None)), (EINVAL, dict(out=None)), (EINVAL, dict(lengths=None)), (EINVAL, dict(table=None)), (EINVAL, dict(ldq=1023)),
    (EINVAL, dict(q=_at(0) + 1)), (EINVAL, dict(lse=_at(2) + 2)), (EINVAL, dict(table=_at(3) + 2)), (EINVAL, dict(starts=_at(5) + 1)), (EINVAL, dict(ws=None)), (EINVAL, dict(ws=_at(6) + 128)),
    (EWORKSPACE, dict(room=-1)), (EINVAL, dict(out=_at(0))), (EINVAL, dict(out=_at(8))), (EINVAL, dict(lse=_at(1) + 4)), (EINVAL, dict(ws=_at(11))), (EINVAL, dict(ws=_at(3))), (EINVAL, dict(B=-5, T=-5)),
    (EINVAL, dict(cache=LONG[:3] + (None,) + LONG[4:])), (0, dict(T=0, B=0)), (0, dict(T=0, starts=_at(5)))])
def test_cache_attention_refuses(ctx, rc, change):
    a = dict(q=_at(0), ldq=1024, T=5, heads=8, dtype=0, cache=LONG, table=_at(3), width=900, lengths=_at(4), starts=None, B=5, scale=0.1, out=_at(1), lse=_at(2), ws=_at(6), room=0)
    a.update(change)
    c = binding._Cache(*a["cache"]) if a["cache"] else None
    need = esp.cache_attention_workspace(4096, 64, 2, 128, 5, 5, 8, 900, False) + (1 << 30 if a["starts"] else 0)
    assert need > 0
    got = ctx._lib.esparse_cache_attention(ctx._h, a["q"], a["ldq"], a["T"], a["heads"], a["dtype"], C.byref(c) if c else None, a["table"], a["width"], a["lengths"], a["starts"], a["B"], a["scale"],
                                           a["out"], a["lse"], a["ws"], need + a["room"])
    assert got == rc, ctx._lib.esparse_last_error(ctx._h)


@pytest.mark.parametrize("rc,change", [
    (EUNSUPPORTED, dict(dtype=3)), (EUNSUPPORTED, dict(V=(1 << 21) + 1, ld=1 << 22)), (EINVAL, dict(V=0)), (EINVAL, dict(R=-1)), (EINVAL, dict(R=1 << 22)), (EINVAL, dict(x=None)), (EINVAL, dict(u=None)),
    (EINVAL, dict(tokens=None)), (EINVAL, dict(ld=999)), (EINVAL, dict(ld=1 << 31)), (EINVAL, dict(x=_at(0) + 1)), (EINVAL, dict(tokens=_at(2) + 4)), (EINVAL, dict(u=_at(1) + 2)), (EINVAL, dict(t=_at(5) + 1)),
    (EINVAL, dict(k=_at(6) + 1)), (EINVAL, dict(p=_at(7) + 1)), (EINVAL, dict(m=_at(8) + 1)), (EINVAL, dict(lp=_at(3) + 2)), (EINVAL, dict(ws=None)), (EINVAL, dict(ws=_at(4) + 8)), (EWORKSPACE, dict(room=-1)),
    (EINVAL, dict(tokens=_at(0))), (EINVAL, dict(tokens=_at(3))), (EINVAL, dict(ws=_at(1))), (EINVAL, dict(lp=_at(7))), (0, dict(R=0))])
def test_sample_refuses(ctx, rc, change):
    a = dict(x=_at(0), R=4, V=1000, ld=1000, dtype=1, t=_at(5), k=_at(6), p=_at(7), m=_at(8), u=_at(1), tokens=_at(2), lp=_at(3), ws=_at(4), room=0)
    a.update(change)
    need = esp.sample_workspace(4, 1000)
    got = ctx._lib.esparse_sample(ctx._h, a["x"], a["R"], a["V"], a["ld"], a["dtype"], a["t"], a["k"], a["p"], a["m"], a["u"], a["tokens"], a["lp"], a["ws"], need + a["room"])
    assert got == rc, ctx._lib.esparse_last_error(ctx._h)


# ---- the binding refuses tensors of the wrong place, shape or type ------------------------------------
def test_binding_refuses_tensors_that_are_not_on_the_device(ctx):
    x, i = torch.zeros(2, 2, 64, dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    cache = esp.KVCache(*(torch.zeros(1, 2, 16, n, dtype=torch.uint8) for n in (32, 2, 32, 2)), 64)
    for call in (lambda: ctx.rotate_heads(x, None), lambda: ctx.cache_read(cache, i), lambda: ctx.cache_attention(x, cache, i[:, None], i), lambda: ctx.sample(x[0], torch.zeros(2))):
        with pytest.raises(ValueError, match="the context on cuda"):
            call()


def test_binding_refuses_without_tensors_that_belong_together(ctx):
    x = torch.zeros(2, 2, 64, dtype=torch.float16)
    for call in (lambda: ctx.rotate_heads(None, None), lambda: ctx.rotate_heads(x, x, v=x), lambda: ctx.rotate_heads(x, None, cache=object(), v=x, slots=x), lambda: ctx.kv_cache(0, 16, 1, 64)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(esp.EsparseError):
        ctx.kv_cache(4, 24, 1, 64)
    with pytest.raises(TypeError):
        ctx.rotate_heads(x.float(), None)
