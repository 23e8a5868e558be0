"""The 4-bit cache, its pages and rotary positions (include/dartree/serve.h, pages.h,
rotary.h) without a GPU: exported and bound, refused arguments, the table of
frequencies, and the plain forms the GPU tests compare with."""
import ctypes
import decimal
import math
import os
import re

import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests import more_ref as R

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dartree")
FAKE = 0x10000000   # 16-byte aligned address that is never dereferenced
byref = ctypes.byref
BAD, NOT, WS = D.ERR_INVALID_ARG, D.ERR_UNSUPPORTED, D.ERR_WORKSPACE


@pytest.mark.parametrize("header,bound", [("pages.h", D.PAGES_SYMBOLS), ("rotary.h", D.ROTARY_SYMBOLS)])
def test_every_declared_symbol_is_exported_and_bound(header, bound):
    syms = sorted(set(re.findall(r"^dartree_status (dartree_\w+)\(", open(os.path.join(INCLUDE, header)).read(), re.M)))
    assert syms == sorted(bound)
    for s in syms:
        assert hasattr(D.lib(), s)


def cache_params(**kw):
    p = D.CacheParams(4, 8, 128, 64, 100, 16, D.CACHE_E2M1)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_cache_in_4_bits_is_a_type_of_its_own():
    assert D.cache_validate(cache_params()) == D.OK
    for t in (2, 3, 5, -4):
        assert D.cache_validate(cache_params(type=t)) == BAD
    lib, p = D.lib(), cache_params()
    for i in range(5):
        fields = [FAKE] * 5
        for wrong in (None, FAKE + 8):
            fields[i] = wrong
            c = D.CacheC(*fields)
            assert lib.dartree_cache_write(byref(p), byref(c), 64, 16, FAKE, FAKE, 1024, None, None, None, None) == BAD
            assert lib.dartree_cache_read(byref(p), byref(c), 16, FAKE, FAKE, None, None, None) == BAD


def test_cache_memory_has_to_fit():
    p = D.CacheParams(2, 1, 128, 16, 3, 2, D.CACHE_E2M1)
    c = D.DeviceCache.alloc(p, "cpu")
    assert c.k.shape == c.v.shape == (3, 1, 16, 64) and c.k.dtype == torch.uint8
    assert c.k_exp.shape == (3, 1, 16, 4) and int(c.table.max()) == -1
    x = torch.zeros(2, 4, 1, 128, dtype=torch.bfloat16)
    c.k_exp = c.k_exp[..., 0].contiguous()
    with pytest.raises(ValueError, match="k_exp"):
        D.cache_write(p, c, x, x, 4)
    c = D.DeviceCache.alloc(p, "cpu")
    c.v = c.v.view(torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="cache v"):
        D.cache_read(p, c, x, x)
    with pytest.raises(ValueError, match="not on a GPU"):
        D.cache_read(p, D.DeviceCache.alloc(p, "cpu"), x, x)


def test_page_calls_refuse_before_any_launch():
    lib, p = D.lib(), cache_params()
    need = D.pages_workspace_size(p)
    n = ctypes.c_size_t(0)
    assert lib.dartree_pages_workspace_size(byref(p), None) == BAD and lib.dartree_pages_workspace_size(None, byref(n)) == BAD
    wide = cache_params(batch=1 << 16, max_pages=(1 << 14) + 1)
    assert lib.dartree_pages_workspace_size(byref(wide), byref(n)) == NOT
    out = FAKE + 4 * 16 * 4   # right behind the table

    def fork(p=p, table=FAKE, out=out, source=None, keep=None):
        return lib.dartree_pages_fork(p and byref(p), table, out, source, keep, None)

    assert fork(p=None) == BAD and fork(p=cache_params(page=24)) == NOT and fork(p=wide) == NOT
    assert fork(table=None) == BAD and fork(out=None) == BAD and fork(out=out + 8) == BAD
    assert fork(out=out - 16) == BAD and fork(out=FAKE - 240) == BAD                        # overlapping
    assert fork(out=FAKE, source=FAKE) == BAD and fork(source=FAKE + 4) == BAD and fork(keep=FAKE + 4) == BAD

    def reserve(table=FAKE, out=out, rows=130, start=None, counts=None, pairs=FAKE, most=16, totals=FAKE, granted=FAKE, ws=FAKE,
                size=need):
        return lib.dartree_pages_reserve(byref(p), table, out, rows, start, counts, pairs, most, totals, granted, ws, size, None)

    assert reserve(rows=0) == BAD and reserve(out=out - 16) == BAD and reserve(most=15) == BAD and reserve(most=-1) == BAD
    assert reserve(table=None) == BAD and reserve(pairs=None) == BAD and reserve(totals=None) == BAD and reserve(granted=FAKE + 4) == BAD
    assert reserve(start=FAKE + 4) == BAD and reserve(counts=FAKE + 8) == BAD
    assert reserve(ws=None) == WS and reserve(ws=FAKE + 16) == WS and reserve(size=need - 1) == WS
    assert reserve(rows=1 << 30, most=63) == BAD                                            # 16 columns, not more, of 4 requests

    def compact(table=FAKE, out=out, pairs=FAKE, most=50, totals=FAKE, ws=FAKE, size=need):
        return lib.dartree_pages_compact(byref(p), table, out, pairs, most, totals, ws, size, None)

    assert compact(most=49) == BAD and compact(pairs=None) == BAD and compact(totals=None) == BAD and compact(out=out - 4) == BAD
    assert compact(ws=None) == WS and compact(size=need - 1) == WS

    def copy(p=p, c=D.CacheC(FAKE, FAKE, FAKE, FAKE, None), pairs=FAKE, most=4, count=FAKE):
        return lib.dartree_cache_copy(p and byref(p), c and byref(c), pairs, most, count, None)

    assert copy(p=None) == BAD and copy(c=None) == BAD and copy(pairs=None) == BAD and copy(most=0) == BAD and copy(count=None) == BAD
    assert copy(c=D.CacheC(FAKE, FAKE, None, FAKE, None)) == BAD and copy(c=D.CacheC(FAKE, None, FAKE, FAKE, None)) == BAD


def test_page_tensors_have_to_fit():
    p = D.CacheParams(3, 1, 128, 16, 8, 4, D.CACHE_BF16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    t, o = i32(3, 4), i32(3, 4)
    with pytest.raises(ValueError, match="out"):
        D.pages_fork(p, t, i32(3, 5))
    with pytest.raises(ValueError, match="keep"):
        D.pages_fork(p, t, o, keep=torch.zeros(3))
    with pytest.raises(ValueError, match="pairs"):
        D.pages_reserve(p, t, o, 4, i32(3), None, i32(9), i32(2), i32(3), None)
    with pytest.raises(ValueError, match="granted"):
        D.pages_reserve(p, t, o, 4, i32(3), None, i32(9, 2), i32(2), i32(4), None)
    with pytest.raises(ValueError, match="totals"):
        D.pages_compact(p, t, o, i32(4, 2), i32(3), None)
    with pytest.raises(ValueError, match="not on a GPU"):
        D.pages_compact(p, t, o, i32(4, 2), i32(2), None)
    with pytest.raises(ValueError, match="empty"):
        D.cache_copy(p, D.DeviceCache.alloc(p, "cpu"), i32(4, 2), i32(0))


def rotary_params(**kw):
    p = D.RotaryParams(2, 5, 8, 2, 128, 128, D.ROTARY_HALF, D.BF16, 0, 0, 1.0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("field,value,code", [
    ("batch", 0, BAD), ("rows", 0, BAD), ("heads_q", -1, BAD), ("heads_kv", -1, BAD), ("head_dim", 0, BAD), ("rotary_dim", 0, BAD),
    ("rotary_dim", 5, BAD), ("rotary_dim", 130, BAD), ("layout", 2, BAD), ("type", 2, BAD), ("inverse", 2, BAD), ("inverse", -1, BAD),
    ("amplitude", math.inf, BAD), ("amplitude", math.nan, BAD), ("head_dim", 132, NOT), ("head_dim", 520, NOT),
    ("heads_q", 2049, NOT), ("heads_kv", 2049, NOT), ("rows", 1 << 23, NOT)])
def test_rotary_params_refused(field, value, code):
    p = rotary_params(**{field: value})
    assert D.lib().dartree_rotary(byref(p), FAKE, FAKE, 1 << 20, FAKE, 1 << 20, FAKE, 1 << 20, FAKE, 1 << 20, None, None, None,
                                  None) == code


def test_rotary_refuses_before_any_launch():
    lib = D.lib()

    def call(p=rotary_params(), turns=FAKE, q=FAKE, qs=1024, k=FAKE, ks=256, qo=FAKE + 4096, qos=1024, ko=FAKE + 8192, kos=256,
             positions=None, start=None, counts=None):
        return lib.dartree_rotary(p and byref(p), turns, q, qs, k, ks, qo, qos, ko, kos, positions, start, counts, None)

    assert call(p=None) == BAD and call(turns=None) == BAD and call(turns=FAKE + 8) == BAD
    assert call(q=None) == BAD and call(k=None) == BAD and call(qo=None) == BAD and call(ko=FAKE + 4) == BAD
    assert call(qs=1016) == BAD and call(ks=252) == BAD and call(qos=1028) == BAD and call(kos=0) == BAD
    assert call(qo=FAKE, qos=2048) == BAD                                                   # in place with another stride
    assert call(positions=FAKE + 4) == BAD and call(start=FAKE + 4) == BAD and call(counts=FAKE + 4) == BAD
    both = rotary_params(heads_q=0, heads_kv=0)
    assert call(p=both) == BAD


def test_rotary_tensors_have_to_fit():
    p = rotary_params()
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    q, k, t = bf(2, 5, 8, 128), bf(2, 5, 2, 128), torch.zeros(64, dtype=torch.int64)
    with pytest.raises(ValueError, match="q is"):
        D.rotary(p, t, q.float(), k, q, k)
    with pytest.raises(ValueError, match="k_out"):
        D.rotary(p, t, q, k, q, bf(2, 5, 3, 128))
    with pytest.raises(ValueError, match="neither dense"):
        D.rotary(p, t, q, bf(2, 10, 2, 128)[:, ::2].transpose(0, 1).contiguous().transpose(0, 1), q, k)
    with pytest.raises(ValueError, match="turns"):
        D.rotary(p, t[:63], q, k, q, k)
    with pytest.raises(ValueError, match="positions"):
        D.rotary(p, t, q, k, q, k, positions=torch.zeros(2, 5))
    with pytest.raises(ValueError, match="not on a GPU"):
        D.rotary(p, t, q, k, q, k)


def test_turns_refused():
    lib, out = D.lib(), (ctypes.c_uint64 * 256)()
    turns = lambda rot=128, base=1e4, s=None: lib.dartree_rotary_turns(rot, base, s and byref(s), out)
    S = D.RotaryScaling
    assert turns() == D.OK and lib.dartree_rotary_turns(128, 1e4, None, None) == BAD
    assert turns(rot=0) == BAD and turns(rot=7) == BAD and turns(rot=514) == NOT
    assert turns(base=0.0) == BAD and turns(base=-1.0) == BAD and turns(base=math.inf) == BAD and turns(base=math.nan) == BAD
    assert turns(s=S(4, 2.0, 1.0, 2.0, 8)) == BAD and turns(s=S(-1, 2.0, 1.0, 2.0, 8)) == BAD
    for rule in (D.ROTARY_LINEAR, D.ROTARY_BASE, D.ROTARY_TURNS):
        assert turns(s=S(rule, 2.0, 1.0, 2.0, 8)) == D.OK
        for factor in (0.0, -1.0, math.inf, math.nan):
            assert turns(s=S(rule, factor, 1.0, 2.0, 8)) == BAD
    assert turns(s=S(D.ROTARY_TURNS, 2.0, 2.0, 2.0, 8)) == BAD and turns(s=S(D.ROTARY_TURNS, 2.0, math.nan, 2.0, 8)) == BAD
    assert turns(s=S(D.ROTARY_TURNS, 2.0, 1.0, 2.0, 0)) == BAD and turns(s=S(D.ROTARY_PLAIN, math.nan, 0.0, 0.0, 0)) == D.OK
    radians = (ctypes.c_double * 2)(1.0, math.nan)
    assert lib.dartree_rotary_turns_of(2, radians, out) == BAD and lib.dartree_rotary_turns_of(1, radians, out) == D.OK
    assert lib.dartree_rotary_turns_of(0, radians, out) == BAD and lib.dartree_rotary_turns_of(1, None, out) == BAD


PI = decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.mark.parametrize("rot,base", [(2, 10000.0), (80, 500000.0), (128, 10000.0), (512, 1e6)])
@pytest.mark.parametrize("rule,factor,low,high,length", [(0, 1.0, 0.0, 0.0, 0), (1, 8.0, 0.0, 0.0, 0), (2, 4.0, 0.0, 0.0, 0),
                                                         (3, 4.0, 1.0, 32.0, 4096), (3, 8.0, 1.0, 4.0, 8192)])
def test_turns_follow_the_rules(rot, base, rule, factor, low, high, length):
    """Within 2^-62 of a turn of the definition in 50 digits (64 bits of mantissa, a handful of roundings)."""
    d = decimal.Decimal
    with decimal.localcontext(decimal.Context(prec=50)):
        b = d(base)
        if rule == 2 and rot > 2:
            b *= d(factor) ** (d(rot) / d(rot - 2))
        got = D.rotary_turns(rot, base, D.RotaryScaling(rule, factor, low, high, length), device="cpu")
        for i, t in enumerate(got.tolist()):
            f = b ** (d(-2 * i) / d(rot))
            if rule == 1:
                f /= d(factor)
            if rule == 3:
                s = min(max((length * f / (2 * PI) - d(low)) / (d(high) - d(low)), d(0)), d(1))
                f *= s + (1 - s) / d(factor)
            off = (d(t % (1 << 64)) - f / (2 * PI) % 1 * (1 << 64) + (1 << 63)) % (1 << 64) - (1 << 63)
            assert abs(off) <= 4
        # 1 / (2 pi) from a rounded pi and a rounded quotient: 2 * 2^-64 of 0.16 turns, a third of a unit of 2^-64 before it
        # is rounded to one, so up to 0.84 units in all
        for t, want in zip(D.rotary_turns_of([1.0, -1.0], "cpu").tolist(), (1 / (2 * PI) * 2 ** 64, -1 / (2 * PI) * 2 ** 64)):
            assert abs(d(t) - want) <= d("0.84")


def test_series_of_sine_and_cosine():
    """The kernel's series, in fp32, over an eighth of a turn either way: off by less than 2^-23."""
    f = np.float32
    exact = np.linspace(-np.pi / 4, np.pi / 4, 200001)
    a = exact.astype(f)
    q = a * a
    sn = a + (a * q) * (f(-1 / 6) + q * (f(1 / 120) + q * (f(-1 / 5040) + q * f(1 / 362880))))
    cs = f(1) + q * (f(-0.5) + q * (f(1 / 24) + q * (f(-1 / 720) + q * (f(1 / 40320) + q * f(-1 / 3628800)))))
    assert np.abs(sn - np.sin(exact)).max() < 2.0 ** -23 and np.abs(cs - np.cos(exact)).max() < 2.0 ** -23


def test_plain_forms():
    """e2m1 codes in words; pages by hand; a turned pair's length and distance."""
    assert R.values_of(*R.quantise(np.full((1, 128), 6.0))).max() == 6.0
    assert R.codes_of(np.array([0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -5.1])).tolist() == [0, 1, 2, 2, 4, 4, 6, 6, 7, 15]
    x = np.zeros(128)
    x[0], x[40], x[70], x[100] = 6.1, 1e-40, np.nan, -6.0 * 2.0 ** 125
    packed, e = R.quantise(x)
    assert e.tolist() == [128, 27, 255, 252] and R.values_of(packed, e)[100] == -6.0 * 2.0 ** 125
    table = np.array([[4, 1, -1], [4, 2, -1]], np.int32)
    out, pairs, totals, granted = R.reserve(table, 16, 6, 20, start=[10, 30])
    assert out.tolist() == [[0, 1, -1], [4, 2, 3]] and pairs == [(4, 0)] and totals == (1, 1) and granted.tolist() == [1, 1]
    out, pairs, totals, granted = R.reserve(table, 16, 6, 40, start=[0, 0], counts=[40, 16])
    assert out.tolist() == [[0, 1, 3], [5, 2, -1]] and pairs == [] and totals == (0, 0)
    out, pairs, totals, granted = R.reserve(table, 16, 5, 40, start=[0, 32], counts=[40, 1])
    assert granted.tolist() == [1, 0] and out[1].tolist() == [4, 2, -1]
    out, pairs, totals = R.compact(np.array([[5, 1, -1], [5, 9, 7]], np.int32), 9)
    assert out.tolist() == [[0, 1, -1], [0, -1, 2]] and pairs == [(5, 0), (7, 2)] and totals == (2, 3)
    assert R.fork(table, 16, source=[1, 5], keep=[17, 100]).tolist() == [[4, 2, -1], [-1, -1, -1]]
    f = R.frequencies(8)
    q, k = np.random.default_rng(0).normal(size=(2, 1, 8))
    for half in (True, False):
        dots = [float((R.rotate(q, p, f, half) * R.rotate(k, p - 7, f, half)).sum()) for p in (7, 100, 2 ** 31)]
        assert np.allclose(dots, dots[0], rtol=1e-9)
        assert np.allclose(R.rotate(R.rotate(q, 9, f, half), 9, f, half, inverse=True), q)
