"""Long contexts that one pair of CTAs works through from end to end: what the values lose to the tensor core's sums, and to weights that
binary16 has no place for, does not grow with the rows."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import oracle  # noqa: E402
from steps import Step, attention  # noqa: E402

pytestmark = pytest.mark.gpu
SEGMENT = 8192  # rows after which sums and references begin anew, at most


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


def step(iq, d, ctx, cross):
    """80 tiles of 64 heads over one KV head: some 148 / 2 pairs of CTAs have a tile each, uncut or cut once."""
    return Step(iq, 41, H=64, hk=1, d=d, ctx=ctx, tokens=320, cross=cross)


def shrunk(c, out, at, causal):
    """By how much the outputs of tokens `at` are shorter than the definition's along it, in the mean over the heads; and the lse's distance."""
    res = []
    for t in at:
        q = [c.q[0][t:t + 1]]
        o, lse, _, _ = attention(c.rows, None, 0, c.quats, c.lk, c.lv, q, c.ctx + (t if causal else 0), [1], causal, 0, 0, c.t_cap)[0]
        got = out[0][0, t].double().cpu()
        res.append(((got * o[0]).sum(-1) / o[0].square().sum(-1) - 1, out[1][0, t].double().cpu() - lse[0]))
    return torch.stack([r[0] for r in res]), torch.stack([r[1] for r in res])


@pytest.mark.parametrize("d,cross", [(128, False), (256, False), (128, True)])
def test_values_of_one_sign(iq, d, cross):
    """A product adds 16 rows and cuts the sum so far towards zero, by 2^-23 of it at most: 512 products in a segment (those of the
    weights' second terms come before the first of the same rows and are given no share of their own). All else rounds to nearest,
    independently from row to row, and averages out over the 64 heads: 2^-16 is allowed for it (an output's own rounding is 2^-11 / sqrt(3) of
    an element, some 2^-18.4 of the mean over a token's 64 d). Over the whole context it would be 8192 products, a cut of 2^-11.4 or so."""
    c = step(iq, d, 131072 - 320, cross)
    c.rows.codes[1] |= 1 << (c.bits - 1)  # the upper half of the levels
    c.upload()
    out = c.outputs()
    c.call(*out)
    assert c.status.tolist() == [0, 0, 0, 0]
    less, off = shrunk(c, out, (0, 319), not cross)
    assert float(less.mean(-1).abs().max()) <= SEGMENT / 16 * 2.0 ** -23 + 2.0 ** -16, less.mean(-1).tolist()
    assert float(off.abs().max()) <= 2.0 ** -14


@pytest.mark.parametrize("d,cross", [(128, False), (256, False), (128, True)])
def test_many_small_weights_beside_a_large_one(iq, d, cross):
    """Row 0 has most of the weight, each other row 2^-25.5 of it and the opposite value: together 2^-8.5, which is more than any rounding. What
    is left out lies in the segment of the large one: 8191 times 2^-25 of it at most; an output's own rounding along its direction is
    below 2^-13 (2^-11 / sqrt(3) of an element, independently, over the d elements)."""
    c = step(iq, d, 131072 - 320, cross)
    low = 25.5 * math.log(2)
    a = c.rows.codes[1][:, :, :1]
    c.rows.codes[1][:] = (1 << c.bits) - 1 - a
    c.rows.codes[1][:, :, 0] = a[:, :, 0]
    c.rows.scales[1][:] = math.sqrt(d)
    c.rows.codes[0][:] = (1 << c.bits) - 1
    c.rows.scales[0][:] = 0.0
    rot = np.asarray(oracle.rotation_matrix(d, c.quats[0]), np.float64)
    q = (rot.T @ np.full(d, 0.5)).astype(np.float16)
    c.q = [np.broadcast_to(q, c.q[0].shape).copy()]
    score = float((rot @ q.astype(np.float64)).sum() * c.lk[-1] / math.sqrt(d)) / math.sqrt(d)  # of a row whose scale is 1
    c.rows.scales[0][:, :, 0] = low / score
    c.upload()
    out = c.outputs()
    c.call(*out)
    less, off = shrunk(c, out, (0, 319), not cross)
    assert float(less.abs().max()) <= SEGMENT * 2.0 ** -25 + 2.0 ** -13, less[:, :4].tolist()
    assert float(off.abs().max()) <= 2.0 ** -14


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("kind", ["random", "rising", "falling", "late", "empty"])
def test_segments_with_references_of_their_own(iq, d, kind):
    """References that rise, fall, begin late (rows of V scale 0 before count as 2^-60) and segments that tokens do not see, by the bounds of the other tests."""
    kw = dict(window=9000, sinks=40) if kind == "empty" else {}
    c = Step(iq, 42, H=64, hk=1, d=d, ctx=30000, tokens=90, **kw)
    s = c.rows.scales
    if kind == "rising":
        s[0] *= np.linspace(0.02, 4.0, s[0].shape[2], dtype=np.float32)
    elif kind == "falling":
        s[0] *= np.linspace(4.0, 0.02, s[0].shape[2], dtype=np.float32)
    elif kind == "late":
        s[0][:, :, :20000] = 0.0
        s[1][:, :, :20000] = 0.0
    c.upload()
    out, lse = c.outputs()
    c.call(out, lse)
    assert c.status.tolist() == [0, 0, 0, 0]
    keep = [0, 1, 40, 88, 89]  # (tokens are worked out alike; the definition takes its time)
    full, c.q = c.q, [c.q[0][keep]]
    want = [attention(c.rows, None, 0, c.quats, c.lk, c.lv, [full[0][t:t + 1]], c.ctx + t, [1], True, c.window, c.sinks, c.t_cap)[0] for t in keep]
    for (o, l, tol, tol_lse), t in zip(want, keep):
        e = (out[0, t].double().cpu() - o[0]).norm(dim=-1)
        assert bool((e <= tol[0] + 2.0 ** -11 * o[0].norm(dim=-1) + 2.0 ** -25 * math.sqrt(d)).all()), (t, float((e / tol[0]).max()))
        assert bool(((lse[0, t].double().cpu() - l[0]).abs() <= tol_lse[0]).all())
    again, _ = c.outputs()
    c.call(again)
    assert torch.equal(again, out)
