"""iq_tree_attention where a CTA works off long pieces, many pieces, or pieces whose rows differ much in weight and length. Many sequences
share the pages of one context, so the cache stays small; a few sequences are compared with the definition in 64 bits."""
import math

import numpy as np
import pytest

import branching as br
import oracle
from test_gpu_tree import Case, dev

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


def tile_and_ctas(c):
    """(token, query head) pairs of an item and CTAs of the launch."""
    pairs = c.T * c.H // c.hk
    tile = 16 if pairs <= 16 else 32 if pairs <= 32 else 64
    return tile, torch.cuda.get_device_properties(0).multi_processor_count * (2 if c.d == 128 and tile <= 32 else 1)


def blocks_per_cta(c):
    """Blocks of 128 rows in a CTA's range (no window)."""
    tile, ctas = tile_and_ctas(c)
    items = [c.hk * -(-int(t) * (c.H // c.hk) // tile) * -(-(int(x) + int(t)) // 128) for x, t in zip(c.ctx, c.tokens)]
    return sum(items) / ctas


def shared(iq, seed, sequences=None, **kw):
    """A Case of one sequence, its pages read by as many sequences as the launch has CTAs (or `sequences`), each with queries of its own.
    The drafted tokens see the context only."""
    c = Case(iq, seed, B=1, page_rows=128, tree="any", **kw)
    B = sequences or tile_and_ctas(c)[1]
    c.B = B
    c.ctx, c.tokens, c.table = np.repeat(c.ctx, B), np.repeat(c.tokens, B), np.repeat(c.table, B, 0)
    c.see = np.zeros((B, c.T, c.T), bool)
    c.mask = dev(br.mask_words(c.see))
    c.q = c.rng.standard_normal((B, c.T, c.H, c.d)).astype(np.float16)
    c.shape = iq.Shape(B, c.H, c.hk, c.d, c.t_cap, c.bits, c.sm_scale)
    return c


def run(c):
    c.upload()
    out = torch.zeros((c.B, c.T, c.H, c.d), device="cuda")
    lse = torch.zeros((c.B, c.T, c.H), device="cuda")
    c.call(out, lse)
    torch.cuda.synchronize()
    assert c.status.tolist() == [0, 0, 0, 0]
    return out, lse


def expected(c, some):
    return br.attention(c.rows, c.table[some], c.page_rows, c.quats, c.lk, c.lv, c.q[some], c.ctx[some], c.tokens[some], c.see[some], c.window, c.sinks,
                        c.t_cap, c.sm_scale)


def off(got, want):
    """Error over all the outputs, relative to them."""
    got = got.double().cpu().numpy()
    return np.linalg.norm(got - want) / np.linalg.norm(want)


# Head counts and tokens of the three tiles.
TILES = [dict(T=2, H=8), dict(T=4, H=8), dict(T=8, H=8)]
KINDS = [dict(d=128), dict(d=256, bits=4), dict(d=128, bits=2, grid="fp16"), dict(d=256, grid="fp16")]


def ids(k):
    return "-".join(f"{a}{v}" for a, v in k.items())


@pytest.mark.parametrize("kind", KINDS, ids=ids)
@pytest.mark.parametrize("tile", TILES, ids=ids)
def test_sums_over_long_pieces(iq, tile, kind):
    """Over 150 blocks of one item to a CTA. A tensor core cuts its sums off where an fp32 addition rounds, 16 times a block, by half of
    2^-24 .. 2^-23 of the sum in the mean, always towards zero: left there for 160 blocks the sums lose 160 * 16 * 2^-25 = 8e-5, over
    the growing sum 4e-5. Taken over into fp32 sums every 16 blocks it is a tenth: with q~ and the weights (2^-18 and less of each, not
    all one way) below 1e-5."""
    c = shared(iq, 21, ctx=160 * 128, **tile, **kind)
    assert blocks_per_cta(c) > 150
    out, lse = run(c)
    some = [0, c.B // 2, c.B - 1]
    o, l, tol, tol_lse = expected(c, some)
    assert off(out[some], o) <= 1e-5
    assert np.all(np.abs(lse[some].double().cpu().numpy() - l) <= tol_lse)


def towards(c, k, score):
    """Every query's part along k (in the original space) made so large that a row whose key is k scores `score`."""
    q = c.q.astype(np.float64)
    q += (score * math.sqrt(c.d) - q @ k)[..., None] * k / (k @ k)
    c.q = q.astype(np.float16)


def bound(c, score):
    """Of the output: 2^-18 of each weight, q~ and exp2 below that, the sums as over long pieces: 1e-5; and for a row that scores much, what
    the tensor core cuts off its score (d / 16 additions of first terms, 2^-24 in the mean) and its rounding."""
    return 1e-5 + (c.d / 16 + 2) * 2.0 ** -24 * max(score, 0.0)


@pytest.mark.parametrize("kind", KINDS, ids=ids)
@pytest.mark.parametrize("tile", TILES, ids=ids)
@pytest.mark.parametrize("weight,length", [(0.99, 1e-6), (0.9999, 1e-6), (1e-12, 1e5)], ids=["sink99", "sink9999", "long"])
def test_one_row_unlike_the_others(iq, weight, length, tile, kind):
    """A row near the start of a piece of some 100 blocks has almost all of the weight and next to no value (an attention sink), or a value
    1e5 times the others' and no weight: the output is the other rows' either way. A weight's rounding may not depend on how large
    another row's weight or value is."""
    c = shared(iq, 22, ctx=100 * 128, **tile, **kind)
    c.rows.scales[0] *= np.float32(0.1)
    page, row = int(c.table[0, 0]), 5
    c.rows.scales[0][page, 0, row] = math.sqrt(c.d)
    c.rows.scales[1][page, 0, row] = math.sqrt(c.d) * length
    score = math.log(int(c.ctx[0])) + math.log(weight / (1 - weight))
    towards(c, c.lk[c.rows.codes[0][page, 0, row]].astype(np.float64) @ oracle.rotation_matrix(c.d, c.quats[0]), score)
    out, lse = run(c)
    some = [0, c.B - 1]
    o, l, tol, tol_lse = expected(c, some)
    assert off(out[some], o) <= bound(c, score)
    assert np.all(np.abs(lse[some].double().cpu().numpy() - l) <= tol_lse)


@pytest.mark.parametrize("kind", KINDS, ids=ids)
@pytest.mark.parametrize("tile", TILES, ids=ids)
def test_references_that_rise_within_a_piece(iq, tile, kind):
    """One row in some blocks of a piece of 40 scores 12 more than the last one (17 in units of log2: the references rise), before and
    after the values have been taken over into fp32 sums, and in blocks next to each other. The earlier rows have the longer values, so
    that all count: a factor that is left out, or applied to only a part, shows."""
    c = shared(iq, 23, ctx=40 * 128, **tile, **kind)
    blocks = [0, 3, 4, 20, 37]
    last = 12.0 * (len(blocks) - 1) + 4
    c.rows.scales[0] *= np.float32(0.05)
    c.rows.scales[1] *= np.float32(math.exp(last) / 100)
    first = int(c.table[0, 0])
    for i, blk in enumerate(blocks):
        page, score = int(c.table[0, blk]), 12.0 * i + 4
        c.rows.codes[0][page, 0, 77] = c.rows.codes[0][first, 0, 77]
        c.rows.scales[0][page, 0, 77] = math.sqrt(c.d) * score / last
        c.rows.scales[1][page, 0, 77] = math.sqrt(c.d) * math.exp(last - score)
    towards(c, c.lk[c.rows.codes[0][first, 0, 77]].astype(np.float64) @ oracle.rotation_matrix(c.d, c.quats[0]), last)
    out, lse = run(c)
    some = [0, c.B - 1]
    o, l, tol, tol_lse = expected(c, some)
    assert off(out[some], o) <= bound(c, last)
    assert np.all(np.abs(lse[some].double().cpu().numpy() - l) <= tol_lse)


@pytest.mark.parametrize("kw", [dict(T=1, H=64, hk=8), dict(T=3, H=64, hk=8), dict(T=5, H=64, hk=8), dict(T=1, H=16, hk=8, d=256, bits=4), dict(T=9, H=32, hk=8, d=256)], ids=ids)
def test_more_pieces_than_are_found_at_a_time(iq, kw):
    """A CTA's pieces are found sixteen at a time: here it has some forty, a block each."""
    c = shared(iq, 24, sequences=1500, ctx=1, t_cap=128, **kw)
    T = c.T
    c.ctx = c.rng.integers(0, 129 - T, c.B).astype(np.int32)
    c.table = c.rng.integers(0, c.rows.codes[0].shape[0], (c.B, 1)).astype(np.int32)
    c.see[:] = np.tril(np.ones((T, T), bool))
    c.mask = None
    assert blocks_per_cta(c) > 32
    out, lse = run(c)
    some = [0, 1, 2, 300, 301, 749, 750, 1111, 1498, 1499]
    want = expected(c, some)
    c.tokens = c.tokens[some]
    c.check(out[some], lse[some], want=want)
    # sequences that are alike in everything have the same outputs, wherever their pieces lie
    c.ctx[:], c.table[:], c.q[:] = c.ctx[7], c.table[7], c.q[7]
    c.tokens = np.full(c.B, T, np.int32)
    out, _ = run(c)
    assert bool((out == out[:1]).all())


@pytest.mark.parametrize("kw", [dict(T=2, H=8), dict(T=8, H=8, d=256, grid="fp16")], ids=ids)
def test_long_pieces_give_the_same_bits_again(iq, kw):
    """Called twice, and replayed from a graph on another stream, over a workspace that holds something else each time."""
    c = shared(iq, 25, ctx=70 * 128, **kw)
    out, lse = run(c)
    again, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
    q = dev(c.q)
    c.workspace.fill_(255)
    c.call(again, lse2, q=q)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.call(again, lse2, q=q)
    s = torch.cuda.Stream()
    for _ in range(2):
        again.zero_()
        c.workspace.fill_(255)
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kw", [dict(T=2, H=8, bits=4), dict(T=8, H=8, d=256)], ids=ids)
def test_a_wait_that_gives_up_over_levels_of_two_terms(iq, kw):
    """Limit 0, with two tiles of V levels to a block: the call ends, says so, and the next one is right."""
    c = shared(iq, 26, sequences=40, ctx=20 * 128, grid="fp16", **kw).upload()
    out = torch.zeros((c.B, c.T, c.H, c.d), device="cuda")
    iq.iq_selftest_tree_wait(c.shape, c.rot, c.cb, dev(c.q), c.cache, c.ctx_dev, c.mask, c.n_tokens, c.workspace, out, c.status, 0)
    torch.cuda.synchronize()
    assert c.status.tolist() == [2, 0, 0, 0]
    out, _ = run(c)
    some = [0, 39]
    assert off(out[some], expected(c, some)[0]) <= 1e-5


def test_two_calls_at_once(iq):
    """Two streams, each with a workspace of its own, over one cache: the results are those of the calls one after the other."""
    cases = [shared(iq, 27, ctx=30 * 128, T=4, H=8), shared(iq, 27, ctx=30 * 128, T=8, H=8, d=256, grid="fp16")]
    want = [run(c)[0] for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[torch.zeros_like(w) for _ in range(5)] for w in want]
    qs = [dev(c.q) for c in cases]
    torch.cuda.synchronize()
    for i in range(5):
        for c, s, o, q in zip(cases, streams, outs, qs):
            with torch.cuda.stream(s):
                c.call(o[i], q=q)
    torch.cuda.synchronize()
    for c, w, o in zip(cases, want, outs):
        assert c.status.tolist() == [0, 0, 0, 0] and all(torch.equal(w, x) for x in o)
