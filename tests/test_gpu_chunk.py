"""iq_chunk_attention and iq_cross_attention against their definition in 64 bits (tests/steps.py has the bounds): types, head layouts, lengths,
layouts of the tokens, windows, pages, strides, streams and graphs."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from steps import Step  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("ctx,tokens", [(0, 1), (0, 33), (5, 1), (100, 28), (127, 2), (128, 128), (300, 129), (1000, 64), (2500, 257)])
def test_one_sequence(iq, d, ctx, tokens):
    Step(iq, 1, H=4, hk=1, d=d, ctx=ctx, tokens=tokens).run()


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("H,hk", [(1, 1), (4, 1), (9, 3), (64, 8), (40, 1), (72, 1)])
@pytest.mark.parametrize("cross", [False, True])
def test_few_tokens(iq, d, H, hk, cross):
    """Up to 64 (token, head) pairs of a KV head go another way than more do, in a batch up to 16."""
    G = H // hk
    for most in (16, 17, 32, 33, 64, 65):
        n = max(1, most // G)
        Step(iq, most, B=2, H=H, hk=hk, d=d, ctx=[150, 300], tokens=[n, max(0, n - 1)], cross=cross).run()
        Step(iq, most, B=4, H=H, hk=hk, d=d, ctx=[150, 0, 300, 40], tokens=[n, 1, 70, 0], cross=cross, packed=True, window=0 if cross else 100, sinks=3).run()


@pytest.mark.parametrize("H,hk", [(1, 1), (4, 1), (32, 4), (16, 8), (7, 1), (64, 8), (24, 2)])
def test_head_layouts(iq, H, hk):
    Step(iq, 2, B=2, H=H, hk=hk, ctx=[260, 31], tokens=[45, 30]).run()


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("grid", ["int8", "fp16"])
@pytest.mark.parametrize("f16", [False, True])
def test_formats(iq, d, bits, grid, f16):
    Step(iq, 3, B=2, H=8, hk=2, d=d, bits=bits, grid=grid, f16=f16, two_sided=True, ctx=[200, 400], tokens=[70, 9], page_rows=128, packed=True).run()


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("page_rows", [0, 128, 256])
def test_ragged(iq, d, packed, page_rows):
    Step(iq, 4, B=6, H=8, hk=2, d=d, ctx=[0, 513, 40, 0, 1200, 7], tokens=[130, 1, 0, 0, 77, 300], packed=packed, page_rows=page_rows).run()


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("packed", [False, True])
def test_cross(iq, d, packed):
    Step(iq, 5, B=5, H=8, hk=4, d=d, cross=True, ctx=[1500, 0, 1, 129, 640], tokens=[20, 3, 200, 0, 1], packed=packed, page_rows=128).run()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (64, 4), (128, 128), (129, 0), (500, 130), (1000, 2000), (5000, 4)])
@pytest.mark.parametrize("d", [128, 256])
def test_windows(iq, d, window, sinks):
    Step(iq, 6, B=2, H=4, hk=2, d=d, ctx=[1400, 90], tokens=[150, 260], window=window, sinks=sinks).run()


@pytest.mark.parametrize("d", [128, 256])
def test_pages_that_no_token_sees_may_be_missing(iq, d):
    c = Step(iq, 7, B=2, H=4, hk=1, d=d, ctx=[1400, 900], tokens=[50, 20], window=300, sinks=5, page_rows=128)
    vis = c.visible().reshape(2, -1, 128).any(2)
    assert not vis.all()
    keep = c.table.copy()
    c.table[~vis] = -1
    c.upload()
    c.table = keep
    out, lse = c.outputs()
    c.call(out, lse)
    assert c.status.tolist() == [0, 0, 0, 0]
    c.check(out, lse)


def test_a_missing_page_that_is_seen_is_flagged(iq):
    c = Step(iq, 8, ctx=300, tokens=9, page_rows=128)
    c.table[0, 1] = 10 ** 6
    c.upload()
    out, _ = c.outputs()
    c.call(out)
    assert c.status.tolist()[0] == 4


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("kw", [dict(ctx=[300, 90], tokens=[50, 9]), dict(ctx=[300, 90], tokens=[50, 9], window=60, sinks=3),
                                dict(ctx=[300, 90], tokens=[50, 9], cross=True)])
def test_rows_that_are_not_seen_may_hold_anything(iq, d, kw):
    Step(iq, 9, B=2, H=4, hk=1, d=d, t_cap=640, **kw).poison().run()


@pytest.mark.parametrize("d", [128, 256])
def test_a_row_that_some_tokens_see_concerns_no_others(iq, d):
    """NaN and infinite scales in the rows of later tokens: the earlier ones do not see them."""
    c = Step(iq, 10, H=4, hk=1, d=d, ctx=200, tokens=60)
    want = c.expected()
    for i, x in ((0, np.nan), (1, np.nan), (0, np.inf), (1, np.inf)):
        c.rows.scales[i][:, :, 230 + 2 * i + int(np.isinf(x))] = x
    c.upload()
    out, _ = c.outputs()
    c.call(out)
    got = out[0].double().cpu()
    assert bool(torch.isfinite(got[:30]).all()) and not bool(torch.isfinite(got[30]).all())
    o, _, tol, _ = want[0]
    assert bool(((got[:30] - o[:30]).norm(dim=-1) <= tol[:30] + 2.0 ** -11 * o[:30].norm(dim=-1)).all())


@pytest.mark.parametrize("d", [128, 256])
def test_a_query_that_is_not_finite_concerns_its_own_output(iq, d):
    c = Step(iq, 11, H=4, hk=1, d=d, ctx=100, tokens=40)
    want = c.expected()
    c.q[0][7, 2, 5], c.q[0][9, 0, 3] = np.inf, np.nan
    c.upload()
    out, _ = c.outputs()
    c.call(out)
    got, (o, _, tol, _) = out[0].double().cpu(), want[0]
    ok = torch.ones(o.shape[:2], dtype=torch.bool)
    ok[7, 2] = ok[9, 0] = False
    assert bool(((got - o).norm(dim=-1) <= tol + 2.0 ** -11 * o.norm(dim=-1))[ok].all())
    assert bool(torch.isnan(got[~ok]).any(-1).all())


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("x", [np.inf, -np.inf, np.nan])
def test_a_query_that_is_not_finite_changes_no_bit_of_the_others(iq, d, x):
    c = Step(iq, 12, H=4, hk=1, d=d, ctx=100, tokens=70)
    res = []
    for y in (0.0, x):
        c.q[0][7, 2, 5] = c.q[0][66, 1, d - 1] = y
        c.upload()
        out, lse = c.outputs()
        c.call(out, lse)
        res.append((out, lse))
    ok = torch.ones((70, 4), dtype=torch.bool)
    ok[7, 2] = ok[66, 1] = False
    assert torch.equal(res[0][0][0].cpu()[ok], res[1][0][0].cpu()[ok])
    assert torch.equal(res[0][1][0].cpu()[ok], res[1][1][0].cpu()[ok])
    assert bool(torch.isnan(res[1][0][0].cpu()[~ok]).any(-1).all())


@pytest.mark.parametrize("d", [128, 256])
def test_tokens_behind_the_cache(iq, d):
    """Rows from t_cap on are not there: their tokens see the cache, and those with a window behind it nothing."""
    Step(iq, 12, H=4, hk=1, d=d, ctx=200, tokens=150, t_cap=256).run()
    Step(iq, 12, H=4, hk=1, d=d, ctx=200, tokens=150, t_cap=256, window=20).run()


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("kind", ["rising", "sink", "zero", "large", "tiny"])
def test_rows_unlike_the_others(iq, d, kind):
    c = Step(iq, 13, H=4, hk=1, d=d, ctx=3000, tokens=40, q_scale=8.0 if kind == "large" else 2.0)
    s = c.rows.scales
    if kind == "rising":     # scores that grow along the cache: references are raised again and again
        s[0] *= np.linspace(0.02, 6.0, s[0].shape[2], dtype=np.float32)
    elif kind == "sink":     # most of the weight on a row with next to no value
        s[0][:, :, 0] *= 12.0
        s[1][:, :, 0] = 1e-6
    elif kind == "zero":     # rows of norm zero, on either side
        s[0][:, :, ::3] = 0.0
        s[1][:, :, 1::3] = 0.0
        s[1][:, :, :130] = 0.0
    elif kind == "tiny":
        s[1] *= 1e-4
    c.run()


def test_all_values_zero(iq):
    c = Step(iq, 14, H=4, hk=1, ctx=300, tokens=9)
    c.rows.scales[1][:] = 0.0
    out = c.run()
    assert not bool(out.any())


def test_scale_given(iq):
    Step(iq, 15, H=4, hk=2, ctx=333, tokens=21, sm_scale=0.31, q_scale=0.5).run()


@pytest.mark.parametrize("d", [128, 256])
def test_strides(iq, d):
    c = Step(iq, 16, B=2, H=8, hk=2, d=d, ctx=[50, 300], tokens=[40, 17]).upload()
    wide = torch.full((2, c.places, 8 + 6, d + 16), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, :, 2:10, 8:8 + d] = c.q_dev
    out, lse = c.outputs()
    c.call(out, lse, q=wide[:, :, 2:10, 8:8 + d])
    c.check(out, lse)
    turned = c.q_dev.transpose(1, 2).contiguous().transpose(1, 2)  # heads before tokens
    again, _ = c.outputs()
    c.call(again, q=turned)
    assert torch.equal(again, out)


@pytest.mark.parametrize("kw", [dict(B=1, H=8, hk=2, ctx=9000, tokens=16), dict(B=9, H=8, hk=2, ctx=[700 * i for i in range(9)], tokens=[1, 300, 1, 1, 64, 1, 1, 500, 2], packed=True),
                                dict(B=1, H=64, hk=8, ctx=1500, tokens=300)])
@pytest.mark.parametrize("d", [128, 256])
def test_many_tiles_and_cut_ones(iq, d, kw):
    c = Step(iq, 17, d=d, **kw)
    out = c.run()
    for _ in range(3):
        again, _ = c.outputs()
        c.call(again)
        assert torch.equal(again, out)


@pytest.mark.parametrize("packed", [False, True])
def test_large_batches(iq, packed):
    """A few long sequences among many short and empty ones."""
    tokens = [0] * 500
    for b, n in ((3, 1), (40, 70), (41, 2), (200, 90), (201, 17), (499, 130)):
        tokens[b] = n
    Step(iq, 24, B=500, H=4, hk=2, ctx=[(37 * b) % 130 for b in range(500)], tokens=tokens, packed=packed).run()


def test_nothing_to_do(iq):
    c = Step(iq, 18, B=3, ctx=[5, 6, 7], tokens=[0, 0, 0], places=4).upload()
    out, lse = c.outputs()
    c.call(out, lse)
    c.check(out, lse)
    c = Step(iq, 18, B=3, ctx=[0, 0, 0], tokens=[3, 1, 2], cross=True)
    out = c.run()
    assert not bool(out[0, :3].any())


def test_starts_that_are_out_of_range(iq):
    c = Step(iq, 19, B=3, ctx=[20, 30, 40], tokens=[5, 6, 7], packed=True, spare=2).upload()
    want = c.expected()
    out, lse = c.outputs()
    c.start = torch.tensor([-3, 5, 11, 10 ** 9], dtype=torch.int32, device="cuda")   # the last one takes all places: two more tokens
    c.call(out, lse)
    assert c.status.tolist() == [0, 0, 0, 0]
    got = out.double().cpu()
    for b, (a, z) in enumerate(((0, 5), (5, 11), (11, 18))):
        o, _, tol, _ = want[b]
        assert bool(((got[a:z] - o).norm(dim=-1) <= tol + 2.0 ** -11 * o.norm(dim=-1)).all())
    c.start = torch.tensor([9, 5, 4, 2], dtype=torch.int32, device="cuda")           # each behind the next: no tokens
    out, lse = c.outputs()
    c.call(out, lse)
    assert bool((out == 7.0).all())


def test_streams_and_graphs(iq):
    c = Step(iq, 20, B=2, H=8, hk=2, ctx=[700, 90], tokens=[90, 33]).upload()
    want = c.expected()
    out, lse = c.outputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.call(out, lse, stream=side)
    side.synchronize()
    c.check(out, lse, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.call(out, lse)
    # other lengths and queries in the same buffers
    c.ctx = np.array([1, 600], np.int32)
    c.q = [(0.5 * c.rng.standard_normal(x.shape)).astype(np.float16) for x in c.q]
    c.ctx_dev.copy_(torch.from_numpy(c.ctx))
    c.q_dev.copy_(c.queries())
    out.fill_(7.0)
    lse.fill_(7.0)
    g.replay()
    torch.cuda.synchronize()
    c.check(out, lse)


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("tokens", [3, 70])
def test_rows_behind_4_gib(iq, d, tokens):
    """Pages at the end of a pool whose arrays of codes pass 2^32 bytes: the same bits as from a small pool."""
    c = Step(iq, 29, H=4, hk=1, d=d, ctx=300, tokens=tokens, page_rows=128)
    want = c.run()
    small = (c.cache.k_codes, c.cache.k_scales, c.cache.v_codes, c.cache.v_scales)
    n = small[0].shape[0]
    pages = (1 << 32) // (small[0].nbytes // n) + n + 1
    big = []
    for x in small:
        y = torch.empty((pages,) + x.shape[1:], dtype=x.dtype, device="cuda")
        y[pages - n:] = x
        big.append(y)
    c.cache = iq.Cache(*big, c.cache.block_table + (pages - n), 128)
    out, _ = c.outputs()
    c.call(out)
    assert c.status.tolist() == [0, 0, 0, 0]
    assert torch.equal(out, want)


def test_two_calls_at_once(iq):
    a, b = Step(iq, 21, H=32, hk=8, ctx=1500, tokens=200).upload(), Step(iq, 22, B=3, H=16, hk=8, d=256, ctx=700, tokens=60).upload()
    oa, ob = a.outputs(), b.outputs()
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        a.call(*oa, stream=s)
        b.call(*ob, stream=t)
    torch.cuda.synchronize()
    a.check(*oa)
    b.check(*ob)


def test_a_wait_that_gives_up_ends_the_call_and_says_so(iq):
    for d in (128, 256):
        c = Step(iq, 23, H=8, hk=2, d=d, ctx=900, tokens=100).upload()
        out, lse = c.outputs()
        iq.iq_selftest_chunk_wait(c.shape, c.rot, c.cb, c.q_dev, c.cache, c.ctx_dev, c.workspace, out, c.status, 0)
        torch.cuda.synchronize()
        assert c.status.tolist()[0] == 2
        c.status.zero_()
        out, lse = c.outputs()
        c.call(out, lse)
        assert c.status.tolist() == [0, 0, 0, 0]
        c.check(out, lse)
