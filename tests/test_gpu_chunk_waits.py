"""Waits of the chunk attention kernel that give up at any place: the call ends, says so, and leaves nothing behind that the next call meets."""
import pytest

torch = pytest.importorskip("torch")
from steps import Step  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("kw", [dict(H=8, hk=2, ctx=900, tokens=100), dict(B=3, H=16, hk=4, ctx=[3000, 0, 700], tokens=[600, 400, 90]), dict(H=4, hk=1, ctx=6000, tokens=70),
                                dict(H=16, hk=1, ctx=20000, tokens=600)])
def test_waits_that_give_up_at_any_place(iq, d, kw):
    """Limits from no poll at all upwards run out in different roles and pieces. The outputs are then invalid; the call returns, with the flag
    where a wait ran out, and the same call without a limit of that kind is right behind it."""
    c = Step(iq, 31, d=d, **kw).upload()
    want = c.expected()
    for polls in (0, 0, 0, 0, 1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 65536):
        out, lse = c.outputs()
        c.status.zero_()
        iq.iq_selftest_chunk_wait(c.shape, c.rot, c.cb, c.q_dev, c.cache, c.ctx_dev, c.workspace, out, c.status, polls)
        torch.cuda.synchronize()
        flags = c.status.tolist()
        assert flags[1:] == [0, 0, 0] and flags[0] in ((2,) if polls == 0 else (0,) if polls == 65536 else (0, 2))
        c.status.zero_()
        out, lse = c.outputs()
        c.call(out, lse)
        assert c.status.tolist() == [0, 0, 0, 0]
        c.check(out, lse, want)
