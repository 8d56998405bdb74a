"""Refusals of the calls for steps over requests of any lengths, the rotary frequencies and the workspace's size: nothing is launched."""
import ctypes
import math

import numpy as np
import pytest

A = 1 << 20  # an address that is aligned and never read
NULL, SHAPE, ALIGN, CODEBOOK, LIMIT = -1, -2, -3, -4, -6


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


@pytest.fixture(scope="module")
def lib(iq):
    from paper_2608_08081_b200 import binding
    return binding


def chunk(iq, lib, batch=2, heads=8, kv=2, d=128, cap=256, bits=3, cb=None, q=A, sb=8 * 8 * 128, st=8 * 128, sh=128, ctx=A, start=None, count=None, n=8,
          window=0, sinks=0, ws=A, out=A, rot=A, cache=None, cross=False):
    s = lib._IqShape(batch, heads, kv, d, cap, bits, 0.0)
    c = cb or iq.iq_lloyd_max_codebook(d if d in (128, 256) else 128, bits if bits in (2, 3, 4) else 3).c()
    k = cache or lib._IqCache(A, A, A, A, None, 0, 0, 0)
    head = (ctypes.byref(s), rot, ctypes.byref(c), q, sb, st, sh, ctypes.byref(k), ctx, start, count, n)
    return lib._lib.iq_cross_attention(*head, ws, out, None, None, None) if cross else lib._lib.iq_chunk_attention(*head, window, sinks, ws, out, None, None, None)


@pytest.mark.parametrize("kw,code", [
    (dict(d=96), SHAPE), (dict(bits=5), SHAPE), (dict(heads=7), SHAPE), (dict(cap=100), SHAPE), (dict(n=-1), SHAPE), (dict(window=-1), SHAPE),
    (dict(sinks=-1), SHAPE), (dict(sb=-8), SHAPE), (dict(st=-8), SHAPE), (dict(start=A, count=A), SHAPE), (dict(n=(1 << 20) + 1), LIMIT),
    (dict(cap=(1 << 31) - 128), LIMIT), (dict(n=1 << 20, heads=4096, kv=2), LIMIT), (dict(batch=65535, n=1 << 20, heads=1024, kv=128, cap=1 << 30), LIMIT),
    (dict(q=None), NULL), (dict(ctx=None), NULL), (dict(ws=None), NULL), (dict(out=None), NULL), (dict(rot=None), NULL),
    (dict(q=A + 2), ALIGN), (dict(ws=A + 8), ALIGN), (dict(out=A + 4), ALIGN), (dict(sh=4), ALIGN), (dict(st=3), ALIGN), (dict(sb=4), ALIGN)])
@pytest.mark.parametrize("cross", [False, True])
def test_chunk_refusals(iq, lib, kw, code, cross):
    if cross and ("window" in kw or "sinks" in kw):
        pytest.skip("cross attention has neither")
    assert chunk(iq, lib, cross=cross, **kw) == code


def test_chunk_refuses_codebooks_that_decode_refuses(iq, lib):
    cb = iq.Codebook((-1.7, -0.3001, 0.4003, 2.0), (-1.0, 0.0, 1.0))
    assert chunk(iq, lib, bits=2, cb=cb.c()) == CODEBOOK
    assert chunk(iq, lib, bits=3, cb=cb.c()) == CODEBOOK


def test_chunk_with_nothing_to_do(iq, lib):
    assert chunk(iq, lib, batch=0, q=None, ws=None, out=None) == 0
    assert chunk(iq, lib, n=0, q=None, ws=None, out=None) == 0
    assert chunk(iq, lib, n=0, start=A, sb=-5, q=None, ws=None, out=None) == 0
    assert chunk(iq, lib, cache=lib._IqCache(A, A, None, A, None, 0, 0, 0)) == NULL
    assert chunk(iq, lib, cache=lib._IqCache(A, A, A, A, A, 192, 4, 0)) == SHAPE


def test_chunk_workspace(iq):
    a, b = iq.iq_chunk_workspace_bytes(iq.Shape(2, 8, 2, 128, 256)), iq.iq_chunk_workspace_bytes(iq.Shape(64, 64, 8, 256, 1 << 20))
    assert 0 < a < b and a % 16 == 0 and b % 16 == 0
    assert iq.iq_chunk_workspace_bytes(iq.Shape(2, 8, 3, 128, 256)) == 0
    assert iq.iq_chunk_workspace_bytes(iq.Shape(2, 8, 2, 128, (1 << 31) - 128)) == 0


def test_the_diagnostic_call_refuses_more_polls_than_the_limit(iq, lib):
    s, cb, k = lib._IqShape(1, 4, 1, 128, 128, 3, 0.0), iq.iq_lloyd_max_codebook(128, 3).c(), lib._IqCache(A, A, A, A, None, 0, 0, 0)
    assert lib._lib.iq_selftest_chunk_wait(ctypes.byref(s), A, ctypes.byref(cb), A, 512, 512, 128, ctypes.byref(k), A, None, 1, A, A, None, A, 65537, None) == LIMIT


def plan(lib, batch=2, cap=256, ctx=A, new=A, table=None, page_rows=0, pages=0, n=16, start=A):
    s = lib._IqShape(batch, 4, 1, 128, cap, 3, 0.0)
    return lib._lib.iq_plan_tokens(ctypes.byref(s), ctx, new, table, page_rows, pages, n, start, A, A, A, None, None)


@pytest.mark.parametrize("kw,code", [(dict(batch=-1), SHAPE), (dict(cap=100), SHAPE), (dict(n=-1), SHAPE), (dict(table=A), SHAPE), (dict(table=A, page_rows=192, pages=4), SHAPE),
                                     (dict(table=A, page_rows=128), SHAPE), (dict(table=A, page_rows=512, pages=4), SHAPE), (dict(ctx=None), NULL),
                                     (dict(new=None), NULL), (dict(start=None), NULL)])
def test_plan_refusals(lib, kw, code):
    assert plan(lib, **kw) == code


def rotary(iq, lib, d=128, r=None, q=A, k=2 * A, qo=3 * A, ko=4 * A, qs=(512, 128), ks=(128, 128), qos=(512, 128), kos=(128, 128), pos=A, n=4):
    s, c = lib._IqShape(1, 4, 1, d, 128, 3, 0.0), lib._IqRotary(128, 0, 1.0) if r is None else r
    return lib._lib.iq_apply_rotary(ctypes.byref(s), ctypes.byref(c), q, *qs, qo, *qos, k, *ks, ko, *kos, pos, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(d=64), SHAPE), (dict(n=-1), SHAPE), (dict(q=None, k=None, qo=None, ko=None), NULL), (dict(qo=None), NULL), (dict(k=None), NULL), (dict(pos=None), NULL),
    (dict(qs=(-8, 128)), SHAPE), (dict(kos=(128, -8)), SHAPE), (dict(qs=(512, 4)), ALIGN), (dict(ks=(12, 128)), ALIGN), (dict(q=A + 8), ALIGN), (dict(ko=A + 2), ALIGN),
    (dict(qo=A, qos=(1024, 128)), SHAPE)])
def test_rotary_refusals(iq, lib, kw, code):
    assert rotary(iq, lib, **kw) == code


def test_rotary_refuses_other_structs(iq, lib):
    assert rotary(iq, lib, r=lib._IqRotary(256, 0, 1.0)) == SHAPE and rotary(iq, lib, r=lib._IqRotary(24, 0, 1.0)) == SHAPE
    assert rotary(iq, lib, r=lib._IqRotary(0, 0, 1.0)) == SHAPE
    assert rotary(iq, lib, n=0, pos=None) == 0


@pytest.mark.parametrize("kw", [dict(rotary_dim=24), dict(rotary_dim=0), dict(rotary_dim=272), dict(base=1.0), dict(base=float("nan")), dict(scaling="linear", factor=0.5),
                                dict(scaling="parts", factor=2.0, original_len=0), dict(scaling="parts", factor=2.0, original_len=64, beta_fast=1.0),
                                dict(inv_freq=[float("inf")] * 64), dict(scaling="base", factor=float("inf"))])
def test_make_rotary_refusals(iq, kw):
    args = dict(rotary_dim=128)
    args.update(kw)
    with pytest.raises((iq.IQError, AssertionError)):
        iq.iq_make_rotary(**args)


@pytest.mark.parametrize("r", [16, 96, 128, 256])
def test_frequencies(iq, r):
    """Turns per position as 64-bit fractions, off by half a unit of 2^-64, against the formulas in 64-bit floats, which hold 53 bits and lose some
    to the powers; as the part of the turn that the floats' share leaves."""
    i = np.arange(r // 2)

    def off(rot, f):
        turns = np.array([t / 2.0 ** 64 for t in rot.turns])
        return (np.maximum(np.abs(turns - f / (2 * math.pi)) - 2.0 ** -65, 0) / (f / (2 * math.pi))).max()

    plain = 10000.0 ** (-2.0 * i / r)
    assert off(iq.iq_make_rotary(r), plain) < 1e-14
    assert off(iq.iq_make_rotary(r, scaling="linear", factor=3.0), plain / 3.0) < 1e-14
    assert off(iq.iq_make_rotary(r, scaling="base", factor=4.0, base=500.0), (500.0 * 4.0 ** (r / (r - 2))) ** (-2.0 * i / r)) < 1e-13
    parts = iq.iq_make_rotary(r, scaling="parts", factor=8.0, original_len=2048)
    low = max(math.floor(r * math.log(2048 / (2 * math.pi * 32)) / (2 * math.log(10000.0))), 0)
    high = min(math.ceil(r * math.log(2048 / (2 * math.pi)) / (2 * math.log(10000.0))), r - 1)
    k = np.clip((i - low) / max(high - low, 0.001), 0, 1)
    assert off(parts, plain / 8.0 * k + plain * (1 - k)) < 1e-14
    assert abs(parts.magnitude - (0.1 * math.log(8.0) + 1)) < 1e-7
    given = iq.iq_make_rotary(r, inv_freq=-2 * math.pi * (0.25 + i % 2), magnitude=2.0)  # backwards, and more than a turn
    # (2 pi in 64-bit floats is off by 2^-53 of itself)
    assert all(abs(t - (3 << 62)) <= 1 << 12 for t in given.turns) and given.magnitude == 2.0


def test_packed_append_refusals(iq, lib):
    s, cb, k = lib._IqShape(2, 4, 1, 128, 128, 3, 0.0), iq.iq_lloyd_max_codebook(128, 3).c(), lib._IqCache(A, A, A, A, None, 0, 0, 0)

    def call(x=A, st=128, sh=128, pos=A, start=A, rows=8, most=8):
        return lib._lib.iq_quantize_append_packed(ctypes.byref(s), A, ctypes.byref(cb), x, A, st, sh, pos, start, rows, most, ctypes.byref(k), None, None)

    assert call(start=None) == NULL and call(pos=None) == NULL and call(x=None) == NULL
    assert call(rows=-1) == SHAPE and call(most=-1) == SHAPE and call(st=-8) == SHAPE
    assert call(st=4) == ALIGN and call(x=A + 2) == ALIGN
    assert call(most=0) == 0 and call(rows=0) == 0
