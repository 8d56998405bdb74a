"""Starts of packed sequences that hold anything: they count as brought into the places of the step, at the ends of the 32-bit range too."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from steps import Step  # noqa: E402

pytestmark = pytest.mark.gpu
LEAST, MOST = -(1 << 31), (1 << 31) - 1


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


def clamped(starts, places):
    return [max(0, min(x, places)) for x in starts]


@pytest.mark.parametrize("tokens", [[3, 2, 4], [90, 70, 33]])
@pytest.mark.parametrize("starts", [[0, LEAST, LEAST + 1, 5], [LEAST, 4, LEAST, MOST], [MOST, LEAST, 2, LEAST], [7, LEAST, MOST, MOST], [-1, -7, 6, MOST - 1]])
@pytest.mark.parametrize("cross", [False, True])
def test_attention(iq, tokens, starts, cross):
    """The same bits as with the starts brought into range on the host; places that are nobody's are left as they are."""
    c = Step(iq, 33, B=3, H=4, hk=1, ctx=[200, 130, 40], tokens=tokens, packed=True, cross=cross, t_cap=512).upload()
    c.q_dev = torch.where(c.q_dev.isnan(), 0.5, c.q_dev)
    got, want = c.outputs(), c.outputs()
    c.start = torch.tensor(clamped(starts, c.places), dtype=torch.int32, device="cuda")
    c.call(*want)
    c.start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    c.call(*got)
    assert c.status.tolist() == [0, 0, 0, 0]
    mine = np.zeros(c.places, int)
    at = clamped(starts, c.places)
    for a, z in zip(at, at[1:]):
        mine[a:max(a, z)] += 1
    one, none = torch.from_numpy(mine == 1).cuda(), torch.from_numpy(mine == 0).cuda()
    for x, y in zip(got, want):
        assert torch.equal(x[one], y[one])  # (places of two sequences hold the results of either)
        assert bool((x[none] == 7.0).all()) and bool((y[none] == 7.0).all())


@pytest.mark.parametrize("rows,most", [(12, 6), (300, 290)])
@pytest.mark.parametrize("starts", [[0, LEAST, LEAST + 1, 5], [LEAST, 4, LEAST, MOST], [MOST, LEAST, 2, LEAST], [7, LEAST, MOST, MOST]])
def test_append(iq, rows, most, starts):
    d, hk, B = 128, 2, 3
    shape, cb = iq.Shape(B, 4, hk, d, 512), iq.iq_lloyd_max_codebook(d, 3)
    rot = torch.empty(iq.iq_rotation_floats(d, hk), dtype=torch.float32, device="cuda")
    iq.iq_make_rotation(d, hk, 5, None, rot)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    k, v = (torch.randn((rows, hk, d), generator=gen, device="cuda").half() for _ in range(2))
    pos = torch.tensor([5, 128, 120], dtype=torch.int32, device="cuda")
    caches = []
    for s in (starts, clamped(starts, rows)):
        cache = iq.new_cache(shape)
        for x in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales):
            x.zero_()
        iq.iq_quantize_append_packed(shape, rot, cb, k, v, pos, torch.tensor(s, dtype=torch.int32, device="cuda"), most, cache)
        caches.append(cache)
    a, b = caches
    for x, y in ((a.k_codes, b.k_codes), (a.v_codes, b.v_codes), (a.k_scales, b.k_scales), (a.v_scales, b.v_scales)):
        assert torch.equal(x, y)
