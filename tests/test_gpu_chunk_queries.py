"""Tokens whose queries differ in size by powers of two: one factor scales all 128 (token, head) pairs of a CTA, and the small ones keep their bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from steps import Step, attention  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("power", [4, 8, 12, 16, 20])
@pytest.mark.parametrize("kind", ["one_large", "one_small", "every_other"])
def test_large_queries_beside_small_ones(iq, d, power, kind):
    """The scores of the small tokens are of the usual size (by the scale of the scores), so that an error of their queries shows. An element of
    a rotated query is off by 2^-22 of itself (two terms of 11 bits), or by half a step of binary16's subnormals, 2^-25, where the largest element of the 128 pairs'
    queries is 2^8 at least: 2^-33 of that. Over d elements the second is 2^-33 sqrt(d) largest |k| sm in a score; the rest as in the other tests."""
    n = 70
    small = 2.0 ** -8 if power < 16 else 2.0 ** -12
    c = Step(iq, 61, H=4, hk=1, d=d, ctx=500, tokens=n, q_scale=small, sm_scale=2.0 / small / math.sqrt(d))
    big = {"one_large": [33], "one_small": [t for t in range(n) if t != 33], "every_other": list(range(0, n, 2))}[kind]
    c.q[0][big] = (c.q[0][big].astype(np.float32) * 2.0 ** power).astype(np.float16)
    assert np.isfinite(c.q[0]).all()
    c.upload()
    out, lse = c.outputs()
    c.call(out, lse)
    assert c.status.tolist() == [0, 0, 0, 0]
    o, l, tol, tol_lse = attention(c.rows, None, 0, c.quats, c.lk, c.lv, c.q, c.ctx, c.tokens, True, 0, 0, c.t_cap, c.sm_scale)[0]
    largest = float(np.abs(c.q[0].astype(np.float32)).max())
    kn = float(np.linalg.norm(c.lk[c.rows.codes[0][0, 0]] * c.rows.scales[0][0, 0][:, None], axis=-1).max()) / math.sqrt(d)
    vn = float(np.linalg.norm(c.lv[c.rows.codes[1][0, 0]] * c.rows.scales[1][0, 0][:, None], axis=-1).max()) / math.sqrt(d)
    dz = 2.0 ** -33 * math.sqrt(d) * largest * kn * c.sm_scale
    keep = [t for t in range(n) if t not in big]
    e = (out[0].double().cpu() - o).norm(dim=-1)
    lim = tol + 2 * dz * vn + 2.0 ** -11 * o.norm(dim=-1) + 2.0 ** -25 * math.sqrt(d)
    assert bool((e <= lim).all()), float((e / lim).max())
    assert bool(((lse[0].double().cpu() - l).abs() <= tol_lse + dz).all())
    if power <= 16:  # (then dz is below 2^-12 of a score of the size of |q| |k| sm: the outputs' own rounding is most of the error)
        assert float(e[keep].square().sum().sqrt() / o[keep].norm()) <= 2.4e-4
