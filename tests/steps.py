"""Steps over requests of any lengths: caches, queries and the attention of new tokens by its definition in 64 bits, for the tests of the
chunk and cross attention calls."""
import math

import numpy as np
import torch

import branching as br
import oracle


def attention(rows, table, page_rows, quats, levels_k, levels_v, q, ctx, tokens, causal, window, sinks, t_cap, sm_scale=0.0):
    """Outputs and lse in 64 bits, and the bounds that the tests hold the kernel to. q: a list of fp16 [n][H][d], one per sequence; ctx [B].
    Returns per sequence (out [n][H][d], lse [n][H], tol on the 2-norm of a head's output, tol_lse).

    The bounds. A score: as in branching.attention, (d / 16 + 2) cuts of a tensor-core sum, twice, of 2^-24 of |q| |k| sm each, and as much
    again for the rounding of q~ (22 bits) and the products with scales. An exponent is the sum of the score, the logarithm of the V scale
    and the reference in 32 bits: three roundings of 2^-24 of its parts' size (log2 units), and the logarithm is
    off by 2^-22 of itself (lg2.approx: four more). exp2, products and sums: (rows / 128 + 64)
    roundings of 2^-22. A weight's rounding to binary16: half a step is 2^-11 of it, independent between rows, so their sum is 2^-11
    sqrt(sum (p |v|)^2 / 3) in the mean; three and a half times that is allowed. What binary16 leaves out below its normal numbers (2^-14): half a step there
    is 2^-25, and the largest weight times value of a row of queries is 1 or more, as a new reference is the largest so far: 2^-25 of it, per row. The tensor core's running sums over the rows: a cut of 2^-23 of the sum so far every 16 rows, by halves."""
    hk, H, d = quats.shape[0], q[0].shape[1], q[0].shape[2]
    G = H // hk
    sm = sm_scale if sm_scale > 0 else 1 / math.sqrt(d)
    rot = [torch.from_numpy(np.asarray(oracle.rotation_matrix(d, quats[g]), np.float64)) for g in range(hk)]
    res = []
    for b in range(len(q)):
        c, n = min(max(int(ctx[b]), 0), t_cap), len(q[b])
        total = min(c + n, t_cap) if causal else c
        out, lse = torch.zeros((n, H, d), dtype=torch.float64), torch.full((n, H), -math.inf, dtype=torch.float64)
        tol, tol_lse = torch.zeros((n, H), dtype=torch.float64), torch.zeros((n, H), dtype=torch.float64)
        res.append((out, lse, tol, tol_lse))
        if total == 0 or n == 0:
            continue
        r = np.arange(total)
        pos = c + np.arange(n)[:, None]
        vis = (r <= pos) if causal else np.ones((n, total), bool)
        if window > 0:
            vis = vis & ((r > pos - window) | (r < sinks))
        used = np.nonzero(vis.any(0))[0]
        at = [br.place(table, page_rows, b, int(x)) for x in used]
        pg, rw = np.array([a[0] for a in at], int), np.array([a[1] for a in at], int)
        on = torch.from_numpy(vis[:, used])
        for g in range(hk):
            k, v = (torch.from_numpy(lv[rows.codes[i][pg, g, rw]].astype(np.float64) * (rows.scales[i][pg, g, rw].astype(np.float64) / math.sqrt(d))[:, None])
                    for i, lv in ((0, levels_k), (1, levels_v)))
            kn, vn = k.norm(dim=1), v.norm(dim=1)
            hs = slice(g * G, (g + 1) * G)
            qr = torch.from_numpy(q[b][:, hs].astype(np.float64)) @ rot[g].T                     # [n][G][d]
            z = torch.where(on[:, None], sm * (qr @ k.T), -math.inf)
            m = z.amax(-1, keepdim=True)
            some = on.any(1)[:, None]
            p = torch.exp(z - torch.where(some[..., None], m, 0.0))
            l = p.sum(-1).clamp(min=1e-300)
            o = (p @ v) / l[..., None] @ rot[g]
            out[:, hs] = torch.where(some[..., None], o, 0.0)
            lse[:, hs] = torch.where(some, m[..., 0] + torch.log(l), -math.inf)
            count = on.sum(1)[:, None].double()
            dz = 4 * (d / 16 + 2) * 2.0 ** -24 * qr.norm(dim=-1) * kn.max() * sm
            size = z.masked_fill(~on[:, None], 0.0).abs().amax(-1) / math.log(2) + abs(np.log2(max(float(vn.max()), 1e-18))) + 64
            dw = dz + 7 * 2.0 ** -24 * size * math.log(2) + (count / 128 + 64) * 2.0 ** -22
            pv = p * vn
            tol[:, hs] = torch.where(some, 2 * dw * torch.where(on[:, None], vn, 0.0).amax(-1) + 3.5 * 2.0 ** -11 * pv.square().sum(-1).div(3).sqrt() / l
                                     + count * 2.0 ** -25 * pv.amax(-1) / l + count / 16 * 2.0 ** -24 * pv.sum(-1) / l, 0.0)
            tol_lse[:, hs] = torch.where(some, dw + 2.0 ** -22 * lse[:, hs].abs().clamp(max=1e30), 0.0)
    return res


class Step:
    """A cache, a step's new tokens and the arguments of a call. tokens: new tokens of every sequence; packed or padded (then `places` per sequence)."""

    def __init__(self, iq, seed, B=1, H=4, hk=1, d=128, bits=3, grid="int8", f16=False, page_rows=0, ctx=100, tokens=8, places=None, packed=False,
                 cross=False, window=0, sinks=0, two_sided=False, sm_scale=0.0, q_scale=2.0, t_cap=None, spare=5):
        rng = np.random.default_rng(seed)
        self.iq, self.rng = iq, rng
        self.B, self.H, self.hk, self.d, self.bits, self.page_rows = B, H, hk, d, bits, page_rows
        self.cross, self.window, self.sinks, self.packed, self.sm_scale = cross, window, sinks, packed, sm_scale
        self.ctx = np.asarray([ctx] * B if np.isscalar(ctx) else ctx, np.int32)
        self.tokens = np.asarray([tokens] * B if np.isscalar(tokens) else tokens, np.int32)
        self.places = int(self.tokens.sum()) + spare if packed else max(1, int(self.tokens.max())) if places is None else places
        unit = max(128, page_rows)
        most = int((self.ctx + (0 if cross else self.tokens)).max())
        self.t_cap = t_cap or max(unit, -(-most // unit) * unit)
        cb = iq.iq_lloyd_max_codebook(d, bits, grid)
        if two_sided:
            v = iq.iq_lloyd_max_codebook(256 if d == 128 else 128, bits, grid)
            cb = cb.with_v(iq.Codebook(tuple(np.float16(1.5 * x) if grid == "fp16" else 1.5 * x for x in v.levels), v.thresholds))
        self.cb = cb
        self.lk, self.lv = np.array(cb.levels, np.float32), np.array(cb.v_levels or cb.levels, np.float32)
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
        self.q = [(q_scale * rng.standard_normal((max(0, n), H, d))).astype(np.float16) for n in self.tokens]

    def visible(self):
        """[B][t_cap]: whether some token sees the row."""
        vis = np.zeros((self.B, self.t_cap), bool)
        r = np.arange(self.t_cap)
        for b in range(self.B):
            c = min(int(self.ctx[b]), self.t_cap)
            for t in range(len(self.q[b])):
                see = (r <= c + t) if not self.cross else r < c
                if self.window:
                    see = see & ((r > c + t - self.window) | (r < self.sinks))
                vis[b] |= see
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
        return self

    def queries(self):
        """The queries as the call takes them; places without a token hold NaN."""
        if self.packed:
            x = np.full((self.places, self.H, self.d), np.nan, np.float16)
            x[:sum(map(len, self.q))] = np.concatenate(self.q)
        else:
            x = np.full((self.B, self.places, self.H, self.d), np.nan, np.float16)
            for b, y in enumerate(self.q):
                x[b, :len(y)] = y
        return torch.from_numpy(x).cuda()

    def upload(self):
        def dev(a):
            return torch.from_numpy(np.ascontiguousarray(a)).cuda()

        k, ks, v, vs = (dev(a) for a in self.rows.arrays())
        self.cache = self.iq.Cache(k, ks, v, vs, None if self.table is None else dev(self.table), self.page_rows)
        self.rot, self.ctx_dev, self.q_dev = dev(self.quats), dev(self.ctx), self.queries()
        self.start = dev(np.concatenate(([0], np.cumsum([len(x) for x in self.q]))).astype(np.int32)) if self.packed else None
        self.count = None if self.packed else dev(self.tokens)
        self.workspace = torch.full((self.iq.iq_chunk_workspace_bytes(self.shape),), 255, dtype=torch.uint8, device="cuda")  # (NaN)
        self.status = torch.zeros(4, dtype=torch.int32, device="cuda")
        return self

    def outputs(self):
        return torch.full_like(self.q_dev, 7.0), torch.full(self.q_dev.shape[:-1], 7.0, dtype=torch.float32, device="cuda")

    def call(self, out, lse=None, q=None, stream=None):
        args = (self.shape, self.rot, self.cb, self.q_dev if q is None else q, self.cache, self.ctx_dev, self.workspace, out)
        kw = dict(token_start=self.start, n_tokens=self.count, lse_out=lse, status_dev=self.status, stream=stream)
        if self.cross:
            self.iq.iq_cross_attention(*args, **kw)
        else:
            self.iq.iq_chunk_attention(*args, window=self.window, sinks=self.sinks, **kw)

    def expected(self):
        return attention(self.rows, self.table, self.page_rows, self.quats, self.lk, self.lv, self.q, self.ctx, self.tokens, not self.cross, self.window,
                         self.sinks, self.t_cap, self.sm_scale)

    def split(self, x):
        """An output of the call as a list, one per sequence, and what lies in places without a token."""
        x = x.cpu()
        n = [len(y) for y in self.q]
        if self.packed:
            return list(x[:sum(n)].split(n)), x[sum(n):]
        return [x[b, :k] for b, k in enumerate(n)], torch.cat([x[b, k:].flatten() for b, k in enumerate(n)])

    def check(self, out, lse=None, want=None):
        got, rest = self.split(out)
        assert bool((rest == 7.0).all()), "places without a token were written"
        lses = None
        if lse is not None:
            lses, rest = self.split(lse)
            assert bool((rest == 7.0).all())
        far = size = 0.0
        for b, (o, l, tol, tol_lse) in enumerate(want or self.expected()):
            e = (got[b].double() - o).norm(dim=-1)
            lim = tol + 2.0 ** -11 * o.norm(dim=-1) + 2.0 ** -25 * math.sqrt(self.d)
            assert bool((e <= lim).all()), (b, float((e / lim).max()), (~(e <= lim)).nonzero()[:4].tolist())
            far, size = far + float(e.square().sum()), size + float(o.square().sum())
            if lses is not None:
                x = lses[b].double()
                assert torch.equal(torch.isinf(x), torch.isinf(l))
                f = torch.isfinite(l)
                assert bool(((x[f] - l[f]).abs() <= tol_lse[f]).all()), float(((x[f] - l[f]).abs() / tol_lse[f]).max())
        # over all outputs: two independent roundings to binary16 (weights, outputs), 2^-11 / sqrt(3) each at most in the mean; half a step
        # of a subnormal output is 2^-25, whatever its size
        subnormal = sum(x.numel() for x in got) * 2.0 ** -50
        assert far <= (4e-4 ** 2) * size + subnormal, math.sqrt(far / max(size, 1e-300))

    def run(self):
        self.upload()
        out, lse = self.outputs()
        self.call(out, lse)
        torch.cuda.synchronize()
        assert self.status.tolist() == [0, 0, 0, 0]
        self.check(out, lse)
        return out
