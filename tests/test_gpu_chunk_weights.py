"""What the weights lose on their way through the tensor cores stays far below the outputs' own rounding, for many tokens as for few."""
import pytest

torch = pytest.importorskip("torch")
from steps import Step  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("kw", [dict(H=8, hk=2, ctx=1000, tokens=64), dict(H=16, hk=4, ctx=0, tokens=700), dict(B=3, H=8, hk=2, ctx=[900, 300, 1200], tokens=[90, 200, 40], cross=True),
                                dict(H=8, hk=2, ctx=3000, tokens=200, window=1000, sinks=5), dict(H=8, hk=2, ctx=1500, tokens=100, bits=4, grid="fp16", f16=True),
                                dict(H=8, hk=2, ctx=1500, tokens=100, bits=2, two_sided=True), dict(H=4, hk=1, ctx=1500, tokens=5)])
def test_outputs_are_off_by_their_own_rounding(iq, d, kw):
    """r: the norm of what the definition's outputs lose when they are rounded to binary16. A kernel that is exact but for that is r off; one
    that is off by e more, independently, sqrt(r^2 + e^2). 2^-16 of the outputs is allowed beside r (e below 8e-5 of r's 2.1e-4): two terms of a
    weight hold 22 bits (2^-23), a tensor-core sum of these lengths is cut by 1.5e-5 at most (128 products of 2^-23). One term of 11 bits
    makes e 1.2e-4 to 1.9e-4: the rounding of a weight is 2^-12 / sqrt(3) of it in the mean square and more just above a power of two."""
    c = Step(iq, 51, d=d, **kw).upload()
    out, _ = c.outputs()
    c.call(out)
    got, _ = c.split(out)
    far = size = own = 0.0
    for x, (o, _, _, _) in zip(got, c.expected()):
        far, own, size = far + float((x.double() - o).square().sum()), own + float((o.half().double() - o).square().sum()), size + float(o.square().sum())
    far, own = (far / size) ** 0.5, (own / size) ** 0.5
    assert 1.9e-4 < own < 2.3e-4
    assert far <= own + 2.0 ** -16, (far, own)


@pytest.mark.parametrize("d", [128, 256])
def test_a_token_alone_and_among_others(iq, d):
    """The last token's output when 64 come with it and when it comes alone (another kernel, other sums): two roundings of nearly the same value. They
    differ by a step in as many elements as the distance e before rounding is parts of a step: e / 2^-11 in the mean; e is below 2^-15 (both
    kernels' sums and exponents), one element in sixteen then. One term of 11 bits: one in three."""
    c = Step(iq, 52, H=32, hk=8, d=d, ctx=1200, tokens=65).upload()
    out, _ = c.outputs()
    c.call(out)
    last = c.q_dev[:, -1:].contiguous()
    alone = torch.empty_like(last)
    iq.iq_chunk_attention(c.shape, c.rot, c.cb, last, c.cache, c.ctx_dev + 64, c.workspace, alone)
    assert float((alone != out[:, -1:]).float().mean()) < 1 / 16
