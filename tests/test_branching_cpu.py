"""Refusals of the branching calls, and their host-side sizes: nothing is launched."""
import ctypes

import numpy as np
import pytest

import branching as br

A = 1 << 20  # an address that is aligned and never read


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


@pytest.fixture(scope="module")
def lib(iq):
    from paper_2608_08081_b200 import binding
    return binding


NULL, SHAPE, ALIGN, CODEBOOK, LIMIT = -1, -2, -3, -4, -6


def tree(iq, lib, batch=2, heads=8, kv=2, d=128, cap=256, bits=3, cb=None, q=A, sb=8 * 8 * 128, st=8 * 128, sh=128, ctx=A, mask=A, n_tok=None, T=8,
         window=0, sinks=0, ws=A, out=A, rot=A, cache=None):
    s = lib._IqShape(batch, heads, kv, d, cap, bits, 0.0)
    c = cb or iq.iq_lloyd_max_codebook(d if d in (128, 256) else 128, bits if bits in (2, 3, 4) else 3).c()
    k = cache or lib._IqCache(A, A, A, A, None, 0, 0, 0)
    return lib._lib.iq_tree_attention(ctypes.byref(s), rot, ctypes.byref(c), q, sb, st, sh, ctypes.byref(k), ctx, mask, n_tok, T, window, sinks, ws, out, 1,
                                      None, None, None)


@pytest.mark.parametrize("kw,code", [
    (dict(d=96), SHAPE), (dict(bits=5), SHAPE), (dict(heads=7), SHAPE), (dict(cap=100), SHAPE), (dict(T=-1), SHAPE), (dict(window=-1), SHAPE),
    (dict(sinks=-1), SHAPE), (dict(sb=-8), SHAPE), (dict(T=257), LIMIT), (dict(cap=(1 << 31) - 128), LIMIT), (dict(batch=65535, heads=4096, kv=128, T=256), LIMIT),
    (dict(q=None), NULL), (dict(ctx=None), NULL), (dict(ws=None), NULL), (dict(out=None), NULL), (dict(rot=None), NULL),
    (dict(q=A + 2), ALIGN), (dict(ws=A + 8), ALIGN), (dict(out=A + 4), ALIGN), (dict(sh=4), ALIGN), (dict(st=3), ALIGN)])
def test_tree_refusals(iq, lib, kw, code):
    assert tree(iq, lib, **kw) == code


def test_tree_refuses_codebooks_that_decode_refuses(iq, lib):
    cb = iq.Codebook((-1.7, -0.3001, 0.4003, 2.0), (-1.0, 0.0, 1.0))
    assert tree(iq, lib, bits=2, cb=cb.c()) == CODEBOOK
    assert tree(iq, lib, bits=3, cb=cb.c()) == CODEBOOK


def test_tree_with_nothing_to_do(iq, lib):
    assert tree(iq, lib, batch=0, q=None, ws=None, out=None) == 0
    assert tree(iq, lib, T=0, q=None, ws=None, out=None) == 0
    assert tree(iq, lib, cache=lib._IqCache(A, A, None, A, None, 0, 0, 0)) == NULL
    assert tree(iq, lib, cache=lib._IqCache(A, A, A, A, A, 192, 4, 0)) == SHAPE


def test_tree_workspace(iq):
    s = iq.Shape(2, 8, 2, 128, 256)
    sizes = [iq.iq_tree_workspace_bytes(s, T) for T in (1, 8, 64, 256)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and iq.iq_tree_workspace_bytes(s, 257) == 0 and iq.iq_tree_workspace_bytes(s, -1) == 0
    # a partial per item and CTA boundary, not per item times CTAs: a large batch of wide trees stays small beside its cache
    assert iq.iq_tree_workspace_bytes(iq.Shape(32, 64, 8, 128, 32768), 16) < 200 << 20


def test_keep_refusals(iq, lib):
    def keep(batch=2, cap=256, base=A, idx=A, n=4, cache=None, d=128):
        s, k = lib._IqShape(batch, 8, 2, d, cap, 3, 0.0), cache or lib._IqCache(A, A, A, A, None, 0, 0, 0)
        return lib._lib.iq_keep_rows(ctypes.byref(s), ctypes.byref(k), base, idx, None, n, None, None)
    assert keep(d=64) == SHAPE and keep(n=-1) == SHAPE and keep(n=257) == LIMIT and keep(base=None) == NULL and keep(idx=None) == NULL
    assert keep(cache=lib._IqCache(A, A + 4, A, A, None, 0, 0, 0)) == ALIGN
    assert keep(n=0, idx=None) == 0 and keep(batch=0) == 0


def test_pool_refusals(iq, lib):
    def pool(table=A, ref=A, free=A, state=A, n=4, per=2, pages=8, pr=128):
        return lib._IqPagePool(table, ref, free, state, n, per, pages, pr)
    for call in (lib._lib.iq_reserve_pages, lib._lib.iq_release_pages):
        for kw, code in ((dict(table=None), NULL), (dict(ref=None), NULL), (dict(free=None), NULL), (dict(state=None), NULL), (dict(n=-1), SHAPE),
                         (dict(n=65536), SHAPE), (dict(per=0), SHAPE), (dict(pages=0), SHAPE), (dict(pr=100), SHAPE), (dict(per=1 << 25), SHAPE),
                         (dict(n=65535, per=1 << 20), LIMIT)):
            assert call(ctypes.byref(pool(**kw)), A, A, None, None) == code, (call, kw)
        assert call(ctypes.byref(pool()), None, A, None, None) == NULL and call(ctypes.byref(pool()), A, None, None, None) == NULL
        assert call(ctypes.byref(pool(n=0)), A, A, None, None) == 0
    s, k = lib._IqShape(4, 8, 2, 128, 256, 3, 0.0), lib._IqCache(A, A, A, A, A, 128, 8, 0)

    def fork(p=pool(), shape=s, cache=k, src=A, dst=A, rows=A, n=3):
        return lib._lib.iq_fork_sequences(ctypes.byref(shape), ctypes.byref(cache), ctypes.byref(p), src, dst, rows, n, None, None)
    assert fork(n=-1) == SHAPE and fork(n=1025) == LIMIT and fork(src=None) == NULL and fork(dst=None) == NULL and fork(rows=None) == NULL
    assert fork(n=0, src=None) == 0 and fork(p=pool(pr=64)) == SHAPE and fork(cache=lib._IqCache(A, None, A, A, A, 128, 8, 0)) == NULL
    assert fork(shape=lib._IqShape(4, 8, 2, 100, 256, 3, 0.0)) == SHAPE and fork(cache=lib._IqCache(A, A, A + 1, A, A, 128, 8, 0)) == ALIGN

    def copy(cache=k, src=A, dst=A, n=3):
        return lib._lib.iq_copy_pages(ctypes.byref(s), ctypes.byref(cache), src, dst, n, None, None)
    assert copy(n=-1) == SHAPE and copy(src=None) == NULL and copy(dst=None) == NULL and copy(n=0) == 0
    assert copy(cache=lib._IqCache(A, A, A, A, None, 128, 8, 0)) == NULL and copy(cache=lib._IqCache(A, A, A, A, A, 130, 8, 0)) == SHAPE


def test_pool_sizes(iq):
    assert [iq.iq_page_pool_state_ints(n) for n in (0, -1, 1, 32, 33)] == [0, 0, 5, 5, 6]


@pytest.mark.parametrize("bits", [2, 3, 4])
def test_the_tests_packing_is_the_oracles(bits):
    import oracle
    rng = np.random.default_rng(bits)
    codes = rng.integers(0, 1 << bits, (5, 128)).astype(np.uint8)
    for row, packed in zip(codes, br.pack(codes, bits)):
        assert np.array_equal(oracle.pack_row(128, row, bits), packed)
    assert np.array_equal(br.unpack(br.pack(codes, bits), bits), codes)


def test_the_tests_attention_is_the_oracles_for_one_token():
    import oracle
    rng = np.random.default_rng(9)
    rows = br.Rows(rng, 2, 2, 256, 128, 3)
    k, ks, v, vs = rows.arrays()
    quats = rng.standard_normal((2, 32, 8)).astype(np.float32)
    lv = np.sort(rng.standard_normal(8)).astype(np.float32)
    q = rng.standard_normal((2, 1, 4, 128)).astype(np.float16)
    ctx = np.array([200, 7])
    out, lse, _, _ = br.attention(rows, None, 0, quats, lv, lv, q, ctx, [1, 1], np.ones((2, 1, 1), bool), 0, 0, 256)
    want = oracle.decode_attention(quats, lv, q[:, 0], dict(k_codes=k, k_scales=ks, v_codes=v, v_scales=vs), ctx + 1, 2)
    assert np.allclose(out[:, 0], want["out"], atol=1e-10) and np.allclose(lse[:, 0], want["lse"], atol=1e-10)
