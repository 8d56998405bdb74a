"""Pages that no drafted token's window reaches are not needed, wherever the window's edge falls in a block."""
import numpy as np
import pytest

import branching as br
from test_gpu_tree import Case, dev

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


@pytest.mark.parametrize("tree", ["chain", "tree", "deep", "empty"])
@pytest.mark.parametrize("T", [1, 5, 40])
@pytest.mark.parametrize("rest", [0, 1, 90, 125, 126, 127])
def test_no_page_before_the_windows_is_needed(iq, rest, T, tree):
    """ctx - window leaves `rest` in a block of 128 rows. tree: tokens name themselves and ancestors; deep: every token names at least
    three (positions start behind the context's end); empty: one token names nothing, its window reaches a row further."""
    window, sinks = 256, 4
    ctx = 640 + rest + window
    c = Case(iq, 31 + rest, B=2, T=T, ctx=[ctx, ctx + 384], window=window, sinks=sinks, H=8, hk=2, page_rows=128, tree="chain" if tree == "chain" else "tree")
    if tree == "deep":
        c.see[:, :, :min(3, T)] = True
    if tree == "empty":
        c.see[0, T // 2] = False
    if tree != "chain":
        c.mask = dev(br.mask_words(c.see))
    want = c.expected()
    held = c.visible().reshape(2, -1, 128).any(-1)
    for b in range(2):  # the drafted tokens' own pages are there
        held[b, int(c.ctx[b]) // 128:(int(c.ctx[b]) + T - 1) // 128 + 1] = True
    assert not held.all()
    c.table = np.where(held, c.table, -1).astype(np.int32)
    c.upload()
    out = torch.zeros((2, T, 8, 128), device="cuda")
    c.call(out)
    torch.cuda.synchronize()
    assert c.status.tolist() == [0, 0, 0, 0]
    c.check(out, want=want)


@pytest.mark.parametrize("kw", [dict(ctx=256, window=1), dict(ctx=256, window=1, sinks=5), dict(ctx=256, window=2, T=3), dict(ctx=255, window=1, T=3),
                                dict(ctx=256, window=129, T=2), dict(ctx=128, window=1, t_cap=256, T=2), dict(ctx=384, window=128, t_cap=512, T=4),
                                dict(ctx=384, window=129, t_cap=512, T=4)], ids=lambda k: "-".join(f"{a}{v}" for a, v in k.items()))
@pytest.mark.parametrize("tree", ["chain", "tree", "any"])
def test_windows_at_the_edge_of_a_block_or_of_the_cache(iq, kw, tree):
    """Short windows whose first row, or whose token's own row, begins a block or lies behind the cache (t_cap 256: a token there sees
    what sinks there are, or nothing)."""
    c = Case(iq, 37, **{**dict(T=1, H=4, hk=2, t_cap=256, tree=tree), **kw})
    c.poison()
    c.run()
