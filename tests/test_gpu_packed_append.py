"""Packed rows that a call's n_new_max leaves out: the others are appended as ever, those are flagged and counted, on both of the append's paths."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


@pytest.mark.parametrize("d,bits", [(128, 3), (256, 4)])
@pytest.mark.parametrize("lens,most", [([3, 1, 9], 1), ([3, 8, 0], 3), ([300, 129, 1], 130), ([40, 500, 41], 40), ([2, 1, 1], 2), ([1, 0, 2], 1000)])
def test_rows_behind_the_limit(iq, d, bits, lens, most):
    B, hk, t_cap = len(lens), 2, 768
    shape, cb = iq.Shape(B, 4, hk, d, t_cap, bits), iq.iq_lloyd_max_codebook(d, bits)
    rot = torch.empty(iq.iq_rotation_floats(d, hk), dtype=torch.float32, device="cuda")
    iq.iq_make_rotation(d, hk, 5, None, rot)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    k, v = (torch.randn((sum(lens), hk, d), generator=gen, device="cuda").half() for _ in range(2))
    starts = np.concatenate(([0], np.cumsum(lens)))
    pos = torch.tensor([5, 200, 120], dtype=torch.int32, device="cuda")
    caches, status = [], [torch.zeros(4, dtype=torch.int32, device="cuda") for _ in range(2)]
    for c in range(2):
        cache = iq.new_cache(shape)
        for x in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales):
            x.zero_()
        caches.append(cache)
    iq.iq_quantize_append_packed(shape, rot, cb, k, v, pos, torch.tensor(starts, dtype=torch.int32, device="cuda"), most, caches[0], status[0])
    # the same rows without those behind the limit
    keep = np.concatenate([np.arange(s, s + min(n, most)) for s, n in zip(starts, lens)])
    short = [min(n, most) for n in lens]
    kk, vv = (x[torch.from_numpy(keep).cuda()].contiguous() for x in (k, v))
    iq.iq_quantize_append_packed(shape, rot, cb, kk, vv, pos, torch.tensor(np.concatenate(([0], np.cumsum(short))), dtype=torch.int32, device="cuda"), most,
                                 caches[1], status[1])
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[1], name))
    left = sum(lens) - sum(short)
    a, b = status[0].tolist(), status[1].tolist()
    assert b[0] == 0 and b[2] == 0
    assert a[0] == (1 if left else 0) and a[2] == 2 * hk * left and a[1] == b[1]
