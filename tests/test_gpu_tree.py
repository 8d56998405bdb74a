"""iq_tree_attention against its definition in 64 bits (tests/branching.py has the bound): types, head layouts, lengths, masks, windows,
pages, strides, streams and graphs."""
import math

import numpy as np
import pytest

import branching as br

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


def dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda") if dtype is None else torch.tensor(a, dtype=dtype, device="cuda")


class Case:
    """A cache, its drafted tokens and the arguments of a call."""

    def __init__(self, iq, seed, B=1, H=4, hk=1, d=128, bits=3, grid="int8", f16=False, page_rows=0, T=4, ctx=100, tokens=None, window=0, sinks=0,
                 tree="tree", two_sided=False, sm_scale=0.0, q_scale=2.0, t_cap=None):
        rng = np.random.default_rng(seed)
        self.iq, self.rng = iq, rng
        self.B, self.H, self.hk, self.d, self.bits, self.T, self.window, self.sinks, self.page_rows = B, H, hk, d, bits, T, window, sinks, page_rows
        self.ctx = np.asarray([ctx] * B if np.isscalar(ctx) else ctx, np.int32)
        self.tokens = np.asarray([T] * B if tokens is None else tokens, np.int32)
        self.n_tokens = None if tokens is None else dev(self.tokens)
        self.tokens = np.clip(self.tokens, 0, T)
        unit = max(128, page_rows)
        self.t_cap = t_cap or -(-(int(self.ctx.max()) + T) // unit) * unit
        cb = iq.iq_lloyd_max_codebook(d, bits, grid)
        if two_sided:
            v = iq.iq_lloyd_max_codebook(256 if d == 128 else 128, bits, grid)
            cb = cb.with_v(iq.Codebook(tuple(np.float16(1.5 * x) if grid == "fp16" else 1.5 * x for x in v.levels), v.thresholds))
        self.cb = cb
        self.lk = np.array(cb.levels, np.float32)
        self.lv = np.array(cb.v_levels or cb.levels, np.float32)
        self.sm_scale = sm_scale
        self.shape = iq.Shape(B, H, hk, d, self.t_cap, bits, sm_scale)
        if page_rows:
            per = self.t_cap // page_rows
            n = B * per + 3
            self.table = rng.permutation(n)[:B * per].reshape(B, per).astype(np.int32)
            self.rows = br.Rows(rng, n, hk, page_rows, d, bits, f16)
        else:
            self.table = None
            self.rows = br.Rows(rng, B, hk, self.t_cap, d, bits, f16)
        qu = rng.standard_normal((hk, d // 4, 2, 4))
        self.quats = (qu / np.linalg.norm(qu, axis=-1, keepdims=True)).reshape(hk, d // 4, 8).astype(np.float32)
        self.q = (q_scale * rng.standard_normal((B, T, H, d))).astype(np.float16)
        if tree == "chain":
            self.see = np.broadcast_to(np.tril(np.ones((T, T), bool)), (B, T, T)).copy()
        elif tree == "any":
            self.see = rng.random((B, T, T)) < 0.4
        else:
            self.see = np.stack([br.random_tree(rng, T) for _ in range(B)])
        self.mask = None if tree == "chain" else dev(br.mask_words(self.see))

    def visible(self):
        """[B][t_cap]: whether some token sees the row."""
        vis = np.zeros((self.B, self.t_cap), bool)
        for b in range(self.B):
            c, n = min(int(self.ctx[b]), self.t_cap), int(self.tokens[b])
            pos = c + self.see[b][:n, :n].sum(1) - 1
            for t in range(n):
                lo = pos[t] - self.window + 1 if self.window else 0
                r = np.arange(c)
                vis[b, :c] |= (r >= lo) | (r < self.sinks)
                for j in range(min(n, self.t_cap - c)):
                    vis[b, c + j] |= self.see[b, t, j] and (pos[j] >= lo or pos[j] < self.sinks)
        return vis

    def poison(self):
        """NaN and infinite scales, and other codes, wherever no token sees the row."""
        vis = self.visible()
        hidden = np.ones(self.rows.scales[0].shape[0::2], bool)  # [n][rows]
        for b in range(self.B):
            for t in np.nonzero(vis[b])[0]:
                hidden[br.place(self.table, self.page_rows, b, int(t))] = False
        n, r = np.nonzero(hidden)
        for k, x in ((0, np.nan), (1, np.inf)):
            for i, s in enumerate(self.rows.scales):
                sel = (np.arange(len(n)) + i) % 2 == k
                s[n[sel], :, r[sel]] = x

    def upload(self):
        k, ks, v, vs = (dev(a) for a in self.rows.arrays())
        self.cache = self.iq.Cache(k, ks, v, vs, None if self.table is None else dev(self.table), self.page_rows)
        self.rot = dev(self.quats)
        self.ctx_dev = dev(self.ctx)
        self.workspace = torch.full((self.iq.iq_tree_workspace_bytes(self.shape, self.T),), 255, dtype=torch.uint8, device="cuda")  # (NaN)
        self.status = torch.zeros(4, dtype=torch.int32, device="cuda")
        return self

    def call(self, out, lse=None, q=None, stream=None):
        self.iq.iq_tree_attention(self.shape, self.rot, self.cb, dev(self.q) if q is None else q, self.cache, self.ctx_dev, self.mask, self.n_tokens,
                                  self.workspace, out, lse_out=lse, window=self.window, sinks=self.sinks, status_dev=self.status, stream=stream)

    def expected(self):
        return br.attention(self.rows, self.table, self.page_rows, self.quats, self.lk, self.lv, self.q, self.ctx, self.tokens, self.see, self.window,
                            self.sinks, self.t_cap, self.sm_scale)

    def check(self, out, lse=None, want=None):
        o, l, tol, tol_lse = want or self.expected()
        got = out.double().cpu().numpy()
        half = 2.0 ** -11 if out.dtype == torch.float16 else 0.0
        on = np.arange(self.T)[None, :] < self.tokens[:, None]
        o, l, tol, tol_lse, got = o[on], l[on], tol[on], tol_lse[on], got[on]
        err = np.linalg.norm(got - o, axis=-1)
        # (half a step of an output's rounding, and of a subnormal one's)
        lim = tol + half * np.linalg.norm(o, axis=-1) + (2.0 ** -25 * math.sqrt(self.d) if half else 1e-30)
        assert np.all(err <= lim), (float((err / lim).max()), np.argwhere(~(err <= lim))[:4])
        # over all outputs: a lost second term of q~ or of the probabilities, rounded to binary16, would show as 1.4e-4
        if half == 0 and np.linalg.norm(o) > 0:
            assert np.linalg.norm(got - o) <= 1e-4 * np.linalg.norm(o), np.linalg.norm(got - o) / np.linalg.norm(o)
        if lse is not None:
            gl = lse.double().cpu().numpy()[on]
            assert np.array_equal(np.isinf(gl), np.isinf(l))
            f = np.isfinite(l)
            assert np.all(np.abs(gl[f] - l[f]) <= tol_lse[f]), float((np.abs(gl[f] - l[f]) / tol_lse[f]).max())

    def run(self, dtype=torch.float32):
        self.upload()
        out = torch.full((self.B, self.T, self.H, self.d), 7.0, dtype=dtype, device="cuda")
        lse = torch.full((self.B, self.T, self.H), 7.0, dtype=torch.float32, device="cuda")
        self.call(out, lse)
        torch.cuda.synchronize()
        assert self.status.tolist() == [0, 0, 0, 0]
        behind = np.arange(self.T)[None, :] >= self.tokens[:, None]  # left as they were
        assert bool((out.cpu()[torch.from_numpy(behind)] == 7.0).all()) and bool((lse.cpu()[torch.from_numpy(behind)] == 7.0).all())
        self.check(out, lse)
        return out, lse


# the smallest first: what faults, faults in a small call
CASES = [
    dict(T=1, ctx=1),
    dict(T=1, ctx=0),
    dict(T=1, ctx=127, tree="chain"),
    dict(T=3, ctx=126, tree="chain"),                    # the drafted rows cross a block
    dict(T=2, ctx=128, H=1, hk=1),
    dict(T=5, ctx=1000, H=32, hk=8),
    dict(T=7, ctx=300, H=6, hk=2),                       # three heads per KV head
    dict(T=60, ctx=500, H=32, hk=8),
    dict(T=16, ctx=900, H=16, hk=2, tree="any"),
    dict(T=64, ctx=70, H=8, hk=8),
    dict(T=33, ctx=200, H=4, hk=1),
    dict(T=256, ctx=130, H=2, hk=2),
    dict(T=200, ctx=0, H=4, hk=2, tree="chain"),         # a prompt's first chunk
    dict(T=4, ctx=2500, H=20, hk=1, d=256),              # more heads per KV head than a decode item takes
    dict(T=13, ctx=777, H=16, hk=8, d=256, bits=4, grid="fp16", f16=True, page_rows=256),
    dict(T=9, ctx=400, H=8, hk=2, bits=2, two_sided=True),
    dict(T=9, ctx=400, H=8, hk=2, bits=4, two_sided=True, grid="fp16"),
    dict(T=40, ctx=300, H=8, hk=2, d=256, bits=2, grid="fp16"),
    dict(T=12, ctx=260, H=8, hk=1, d=256, bits=3),
    dict(B=3, T=6, ctx=[0, 129, 640], H=8, hk=2, tokens=[6, 0, 3]),
    dict(B=5, T=20, ctx=[1, 0, 300, 128, 1100], H=8, hk=4, tokens=[20, 1, 19, 7, 20], page_rows=128, bits=4),
    dict(B=4, T=1, ctx=[5, 2000, 128, 999], H=64, hk=8, page_rows=512, f16=True),
    dict(B=2, T=70, ctx=[100, 40], H=4, hk=2, tokens=[-3, 999]),   # clamped
    dict(T=6, ctx=250, t_cap=256),                       # the last tokens' rows lie outside the cache
    dict(T=4, ctx=400, t_cap=256),
    dict(T=4, ctx=300, sm_scale=0.3),
    dict(T=1, ctx=200, H=130, hk=1),                     # a token's heads over three passes
    dict(T=3, ctx=1000, H=22, hk=1),                     # 66 pairs: two left for a second pass
]
WINDOWS = [
    dict(T=1, ctx=3000, window=1000, sinks=4, H=8, hk=2),
    dict(T=1, ctx=50, window=1, sinks=0),
    dict(T=1, ctx=600, window=128, sinks=128),
    dict(T=1, ctx=900, window=5, sinks=300, H=8, hk=1),
    dict(T=16, ctx=2000, window=300, sinks=1, H=16, hk=4),
    dict(T=40, ctx=513, window=7, sinks=0, H=4, hk=2),           # ancestors drop out of the window
    dict(T=40, ctx=2, window=3, sinks=5, H=4, hk=2, tree="any"),  # sinks among the drafted tokens
    dict(T=100, ctx=0, window=30, sinks=2, H=4, hk=1, tree="chain"),
    dict(B=4, T=3, ctx=[0, 100, 5000, 1300], window=700, sinks=200, H=8, hk=8, tokens=[3, 2, 3, 1], page_rows=128, d=256, bits=4),
    dict(T=2, ctx=400, window=2147483647, sinks=2147483647),
    dict(B=2, T=1, ctx=[1000, 90], window=256, sinks=0, H=64, hk=8, tree="chain", f16=True),
]


@pytest.mark.parametrize("kw", CASES + WINDOWS, ids=lambda k: "-".join(f"{a}{v}" for a, v in k.items()).replace(" ", ""))
def test_against_the_definition(iq, kw):
    c = Case(iq, 1 + len(str(kw)), **kw)
    c.poison()
    c.run()


@pytest.mark.parametrize("seed", range(12))
def test_random_cases(iq, seed):
    rng = np.random.default_rng(500 + seed)
    H, hk = ((4, 1), (32, 4), (16, 8), (8, 8), (12, 4), (64, 8))[rng.integers(6)]
    B, T = int(rng.integers(1, 5)), int(rng.integers(1, 40))
    kw = dict(B=B, H=H, hk=hk, T=T, d=int(rng.choice([128, 256])), bits=int(rng.integers(2, 5)), grid=str(rng.choice(["int8", "fp16"])),
              f16=bool(rng.integers(2)), page_rows=int(rng.choice([0, 128, 384])), ctx=[int(x) for x in rng.integers(0, 900, B)],
              tokens=[int(x) for x in rng.integers(0, T + 1, B)] if rng.integers(2) else None, tree=str(rng.choice(["tree", "any", "chain"])),
              two_sided=bool(rng.integers(2)))
    if rng.integers(2):
        kw.update(window=int(rng.integers(1, 600)), sinks=int(rng.integers(0, 200)))
    c = Case(iq, 900 + seed, **kw)
    c.poison()
    c.run(torch.float16 if seed % 3 == 0 else torch.float32)


def test_tokens_that_see_nothing(iq):
    c = Case(iq, 3, T=5, ctx=0, H=4, hk=2)
    c.see[:] = False
    c.see[0, 1, 4] = True                     # one token sees one row, behind itself
    c.see[0, 2, 2] = True
    c.mask = dev(br.mask_words(c.see))
    out, lse = c.run()
    assert bool((out[0, [0, 3, 4]] == 0).all()) and bool(torch.isneginf(lse[0, [0, 3, 4]]).all())
    c = Case(iq, 4, T=3, ctx=40, H=4, hk=2)  # no drafted token seen: the context only
    c.see[:] = False
    c.mask = dev(br.mask_words(c.see))
    c.run()


def test_bits_of_tokens_that_are_not_there_are_ignored(iq):
    c = Case(iq, 5, T=6, ctx=200, tokens=[3], H=4, hk=2)
    c.mask = torch.full_like(c.mask, -1)
    c.see[:] = True
    c.run()


@pytest.mark.parametrize("scale", [1e-6, 1.0, 60.0])
def test_magnitudes(iq, scale):
    """Queries from tiny to so long that a softmax is one row, rows of V of very different lengths."""
    c = Case(iq, 6, T=4, ctx=700, H=8, hk=2, q_scale=scale)
    c.rows.scales[1] = (c.rows.scales[1] * np.exp(4 * c.rng.standard_normal(c.rows.scales[1].shape))).astype(np.float32)
    c.q[0, 1] = 0
    c.run()


def test_growing_scores(iq):
    """Every block raises the running maximum."""
    c = Case(iq, 7, T=3, ctx=1500, H=8, hk=2)
    c.rows.scales[0] = (c.rows.scales[0] * np.linspace(0.01, 6, c.t_cap)[None, None, :]).astype(np.float32)
    c.rows.scales[1] = (c.rows.scales[1] * np.geomspace(1e-4, 1e4, c.t_cap)[None, None, :]).astype(np.float32)
    c.run()


def test_non_finite_visible_rows_stay_with_the_tokens_that_see_them(iq):
    c = Case(iq, 8, T=4, ctx=200, H=4, hk=2)
    c.see[0] = np.eye(4, dtype=bool)
    c.mask = dev(br.mask_words(c.see))
    want = c.expected()
    c.rows.scales[1][0, :, 202] = np.inf
    c.upload()
    out = torch.zeros((1, 4, 4, 128), device="cuda")
    c.call(out)
    got = out.cpu()
    assert not bool(torch.isfinite(got[0, 2]).all())
    c.tokens = np.array([2], np.int32)
    c.check(out, want=tuple(w for w in want))


def test_strided_queries_binary16_output_and_repeatability(iq):
    c = Case(iq, 9, B=2, T=5, ctx=[700, 90], H=16, hk=4).upload()
    wide = torch.full((2, 5, 16 + 8, 128), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, :, :16] = dev(c.q)
    outs = [torch.zeros((2, 5, 16, 128), dtype=t, device="cuda") for t in (torch.float16, torch.float32, torch.float16)]
    c.call(outs[0], q=wide[:, :, :16])
    c.call(outs[1])
    c.call(outs[2])
    want = c.expected()
    c.check(outs[0], want=want)
    c.check(outs[1], want=want)
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1].half(), outs[0])


def test_own_stream_and_graph(iq):
    """Captured once, replayed with other lengths, masks, queries and token counts: all are read on the device."""
    a = Case(iq, 10, B=2, T=6, ctx=[300, 40], H=8, hk=2, tokens=[6, 4], t_cap=1024).upload()
    out, lse, q = torch.zeros((2, 6, 8, 128), device="cuda"), torch.zeros((2, 6, 8), device="cuda"), dev(a.q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a.call(out, lse, q=q, stream=s)
    s.synchronize()
    a.check(out, lse)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.call(out, lse, q=q)
    for seed, ctx, tokens in ((11, [1000, 3], [1, 6]), (12, [0, 129], [6, 0]), (10, [300, 40], [6, 4])):
        b = Case(iq, seed, B=2, T=6, ctx=ctx, H=8, hk=2, tokens=tokens, t_cap=1024)
        k, ks, v, vs = (dev(x) for x in b.rows.arrays())
        for x, y in ((a.cache.k_codes, k), (a.cache.k_scales, ks), (a.cache.v_codes, v), (a.cache.v_scales, vs), (a.rot, dev(b.quats)),
                     (a.ctx_dev, dev(b.ctx)), (a.n_tokens, b.n_tokens), (a.mask, b.mask), (q, dev(b.q))):
            x.copy_(y)
        out.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        b.check(out, lse)
        assert bool((out.cpu()[torch.from_numpy(np.arange(6)[None, :] >= b.tokens[:, None])] == 5.0).all())


def test_one_token_is_a_decode_step(iq):
    """A chain of one drafted token over a context of n rows and a decode step over n + 1 rows are the same attention."""
    c = Case(iq, 13, B=3, T=1, ctx=[1, 700, 255], H=32, hk=8, tree="chain").upload()
    out, lse = torch.zeros((3, 1, 32, 128), device="cuda"), torch.zeros((3, 1, 32), device="cuda")
    c.call(out, lse)
    ws = iq.DecodeWorkspace(c.shape, iq.iq_suggest_splits(c.shape, 701))
    iq.decode_step(c.shape, c.rot, c.cb, dev(c.q[:, 0]), c.cache, c.ctx_dev + 1, ws)
    o, l, tol, tol_lse = c.expected()
    # each is within the bound of the definition (the decode step's own arithmetic: 21 bits of q~)
    assert np.all(np.linalg.norm((out[:, 0] - ws.out).double().cpu().numpy(), axis=-1) <= 2 * tol[:, 0] + 1e-3 * np.linalg.norm(o[:, 0], axis=-1))
    assert np.allclose(lse[:, 0].cpu().numpy(), ws.lse.cpu().numpy(), atol=2e-3, rtol=1e-5)


def test_pages_outside_the_window_are_not_needed(iq):
    c = Case(iq, 14, T=2, ctx=3000, window=300, sinks=10, H=8, hk=2, page_rows=128)
    want = c.expected()
    vis = c.visible().reshape(1, -1, 128).any(-1)
    c.table = np.where(vis, c.table, -1).astype(np.int32)
    c.upload()
    out = torch.zeros((1, 2, 8, 128), device="cuda")
    c.call(out)
    torch.cuda.synchronize()
    assert c.status.tolist() == [0, 0, 0, 0]
    c.check(out, want=want)


def test_an_entry_outside_the_pool_is_flagged(iq):
    c = Case(iq, 15, T=2, ctx=300, H=4, hk=2, page_rows=128)
    c.table[0, 1] = 10 ** 6
    c.upload()
    out = torch.zeros((1, 2, 4, 128), device="cuda")
    c.call(out)
    torch.cuda.synchronize()
    assert c.status.tolist()[0] == 4 and bool(torch.isfinite(out).all())


def test_rows_beyond_two_to_the_32_bytes(iq):
    """One sequence of 36 M rows of 128 bytes: the last ones lie more than 2^32 bytes behind the first. Only those in the window are
    made (and read)."""
    d, bits, cap = 256, 4, 36 * 10 ** 6 // 128 * 128
    ctx, window, T = cap - 200, 500, 3
    small = Case(iq, 16, T=T, ctx=ctx % 128 + 1024, H=4, hk=1, d=d, bits=bits, window=window, t_cap=ctx % 128 // 128 * 128 + 1408)
    off = ctx - int(small.ctx[0])
    want = small.expected()
    small.upload()
    k = small.cache
    n = min(small.t_cap, cap - off)
    big = [torch.empty((1, 1, cap) + a.shape[3:], dtype=a.dtype, device="cuda") for a in (k.k_codes, k.k_scales, k.v_codes, k.v_scales)]
    for x, y in zip(big, (k.k_codes, k.k_scales, k.v_codes, k.v_scales)):
        x[:, :, off:off + n] = y[:, :, :n]
    small.cache, small.shape = iq.Cache(*big), iq.Shape(1, 4, 1, d, cap, bits)
    small.ctx_dev = dev([ctx], torch.int32)
    out = torch.zeros((1, T, 4, d), device="cuda")
    small.call(out)
    torch.cuda.synchronize()
    small.check(out, want=want)


@pytest.mark.parametrize("kw", [dict(T=1), dict(T=20, H=8, hk=1), dict(T=40, H=8, hk=2, d=256, bits=4)], ids=["16", "64", "d256"])
def test_a_wait_that_gives_up_ends_the_call_and_says_so(iq, kw):
    """With a limit of 0 the first wait whose copy or product is not there yet gives up; the kernel still ends, flags it, and frees what it
    holds: the next call is right."""
    c = Case(iq, 18, ctx=3000, **kw).upload()
    out = torch.zeros((1, c.T, c.H, c.d), device="cuda")
    iq.iq_selftest_tree_wait(c.shape, c.rot, c.cb, dev(c.q), c.cache, c.ctx_dev, c.mask, c.n_tokens, c.workspace, out, c.status, 0)
    torch.cuda.synchronize()
    assert c.status.tolist() == [2, 0, 0, 0]
    c.status.zero_()
    c.call(out)
    torch.cuda.synchronize()
    assert c.status.tolist() == [0, 0, 0, 0]
    c.check(out)


def test_more_sequences_than_threads(iq):
    rng = np.random.default_rng(17)
    c = Case(iq, 17, B=700, T=2, ctx=[int(x) for x in rng.integers(0, 140, 700)], H=2, hk=1, tokens=[int(x) for x in rng.integers(0, 3, 700)])
    c.run()
