"""Rows kept, pages copied, sequences forked, pages reserved and released: whole numbers, equal to a plain model of the calls."""
import numpy as np
import pytest

import branching as br

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def ints(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def upload(iq, rows, table=None, page_rows=0):
    k, ks, v, vs = (dev(a) for a in rows.arrays())
    return iq.Cache(k, ks, v, vs, table, page_rows)


def same(cache, rows):
    k, ks, v, vs = rows.arrays()
    for got, want in ((cache.k_codes, k), (cache.v_codes, v), (cache.k_scales, ks), (cache.v_scales, vs)):
        assert np.array_equal(got.cpu().numpy().view(np.uint8), np.ascontiguousarray(want).view(np.uint8).reshape(got.cpu().numpy().view(np.uint8).shape))


# ---------------------------------------------------------------------------------------------------------------------- keep
def keep_model(rows, table, page_rows, t_cap, base, keep, n_keep):
    """Every source read before any destination is written. Returns the rows that were skipped."""
    skipped = 0
    old = [c.copy() for c in rows.codes], [s.copy() for s in rows.scales]
    for b in range(len(base)):
        for i in range(min(max(n_keep[b], 0), keep.shape[1])):
            src, dst = int(base[b]) + int(keep[b, i]), int(base[b]) + i
            if not (0 <= src < t_cap and 0 <= dst < t_cap):
                skipped += 1
                continue
            (ps, rs), (pd, rd) = br.place(table, page_rows, b, src), br.place(table, page_rows, b, dst)
            n = rows.codes[0].shape[0]
            if table is not None and not (0 <= ps < n and 0 <= pd < n):
                skipped += 1
                continue
            for side in range(2):
                rows.codes[side][pd, :, rd] = old[0][side][ps, :, rs]
                rows.scales[side][pd, :, rd] = old[1][side][ps, :, rs]
    return skipped * rows.codes[0].shape[1]


KEEPS = [
    dict(B=1, hk=1, n=1, base=0),
    dict(B=1, hk=2, n=3, base=126),          # over the edge of a block
    dict(B=2, hk=1, n=8, base=120, d=256),
    dict(B=3, hk=2, n=31, base=100, bits=2, page_rows=128),
    dict(B=2, hk=2, n=17, base=300, bits=4, f16=True, page_rows=256),
    dict(B=1, hk=8, n=60, base=95, bits=4, d=256),
    dict(B=2, hk=1, n=256, base=20, reach=300),
]


@pytest.mark.parametrize("order", ["path", "any"])
@pytest.mark.parametrize("kw", KEEPS, ids=lambda k: "-".join(f"{a}{v}" for a, v in k.items()))
def test_keep_rows(iq, kw, order):
    B, hk, n, d, bits = kw["B"], kw["hk"], kw["n"], kw.get("d", 128), kw.get("bits", 3)
    page_rows, f16 = kw.get("page_rows", 0), kw.get("f16", False)
    rng = np.random.default_rng(n)
    reach = kw.get("reach", 2 * n)
    base = np.array([kw["base"] + 7 * b for b in range(B)], np.int32)
    unit = max(page_rows, 128)
    cap = -(-(int(base.max()) + reach) // unit) * unit
    table = None
    if page_rows:
        table = rng.permutation(B * cap // page_rows + 2)[:B * cap // page_rows].reshape(B, -1).astype(np.int32)
        rows = br.Rows(rng, B * cap // page_rows + 2, hk, page_rows, d, bits, f16)
    else:
        rows = br.Rows(rng, B, hk, cap, d, bits, f16)
    if order == "path":
        keep = np.stack([np.sort(rng.choice(reach, n, replace=False)) for _ in range(B)]).astype(np.int32)
    else:  # any order, with repetitions
        keep = rng.integers(0, reach, (B, n)).astype(np.int32)
    n_keep = np.array([n, n // 2, -1][:B], np.int32)
    shape = iq.Shape(B, hk, hk, d, cap, bits)
    cache = upload(iq, rows, None if table is None else dev(table), page_rows)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    iq.iq_keep_rows(shape, cache, dev(base), dev(keep), dev(n_keep), status_dev=status)
    assert keep_model(rows, table, page_rows, cap, base, keep, n_keep) == 0
    same(cache, rows)
    assert status.tolist() == [0, 0, 0, 0]


def test_keep_skips_and_counts_what_it_cannot_place(iq):
    rng = np.random.default_rng(5)
    rows = br.Rows(rng, 4, 2, 128, 128, 3)
    table = np.array([[0, 1], [2, 9]], np.int32)  # the second page of sequence 1 does not exist
    cache = upload(iq, rows, dev(table), 128)
    shape = iq.Shape(2, 2, 2, 128, 256)
    base, keep = np.array([250, 100], np.int32), np.array([[3, 5, -251, 100], [20, 40, 10 ** 9, 5]], np.int32)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    iq.iq_keep_rows(shape, cache, dev(base), dev(keep), None, status_dev=status)
    skipped = keep_model(rows, table, 128, 256, base, keep, [4, 4])
    same(cache, rows)
    assert skipped == 2 * 4 and status.tolist() == [1 | 4, 0, skipped, 0]


# ---------------------------------------------------------------------------------------------------------------------- pool
class Model:
    def __init__(self, n_seqs, per, num_pages, page_rows):
        self.table = np.full((n_seqs, per), -1, np.int64)
        self.ref = np.zeros(num_pages, np.int64)
        self.free = list(range(num_pages - 1, -1, -1))
        self.pr = page_rows
        self.flags = self.count = 0

    def reserve(self, first, end):
        for b in range(len(self.table)):
            f, e = max(0, int(first[b])), min(int(end[b]), self.table.shape[1] * self.pr)
            for j in range(self.table.shape[1]):
                if j * self.pr < e and (j + 1) * self.pr > f and e > f and self.table[b, j] < 0:
                    if self.free:
                        self.table[b, j] = self.free.pop()
                        self.ref[self.table[b, j]] = 1
                    else:
                        self.flags |= 16
                        self.count += 1

    def release(self, first, end):
        gone = []
        for b in range(len(self.table)):
            f, e = max(0, int(first[b])), min(int(end[b]), self.table.shape[1] * self.pr)
            for j in range(self.table.shape[1]):
                p = int(self.table[b, j])
                if j * self.pr >= f and (j + 1) * self.pr <= e and p >= 0:
                    self.table[b, j] = -1
                    if p >= len(self.ref) or self.ref[p] <= 0:
                        self.flags |= 4
                        self.count += 1
                        continue
                    self.ref[p] -= 1
                    if self.ref[p] == 0:
                        gone.append(p)
        self.free += sorted(gone)

    def fork(self, src, dst, rows):
        """Returns the (from page, to page, rows) of the copies."""
        P, copies = self.table.shape[1], []
        ok = []
        for i in range(len(src)):
            good = 0 <= src[i] < len(self.table) and 0 <= dst[i] < len(self.table) and 0 <= rows[i] <= P * self.pr
            good = good and dst[i] not in [s for s in src] and dst[i] not in [dst[k] for k in range(i)]
            ok.append(good)
        for i in range(len(src)):
            if not ok[i]:
                self.flags |= 32
                self.count += 1
                continue
            last, part = divmod(int(rows[i]), self.pr)
            row = np.full(P, -1, np.int64)
            for j in range(last + (part > 0)):
                p = int(self.table[src[i], j])
                inside = 0 <= p < len(self.ref)
                if not inside:
                    self.flags |= 4
                    self.count += 1
                if j < last:
                    if inside:
                        row[j] = p
                        self.ref[p] += 1
                elif self.free:
                    row[j] = self.free.pop()
                    self.ref[row[j]] = 1
                    if inside:
                        copies.append((p, int(row[j]), part))
                else:
                    self.flags |= 16
                    self.count += 1
            self.table[dst[i]] = row
        return copies

    def same(self, pool):
        assert np.array_equal(pool.block_table.cpu().numpy(), self.table)
        assert np.array_equal(pool.ref_count.cpu().numpy(), self.ref)
        n = int(pool.state[0])
        assert n == len(self.free) and pool.free_list[:n].cpu().tolist() == self.free
        assert int(pool.state[1:].abs().sum()) == 0


@pytest.mark.parametrize("n_seqs,per,num_pages,page_rows", [(1, 1, 1, 128), (3, 5, 9, 128), (40, 12, 300, 256), (1500, 3, 4000, 128), (2, 3000, 5000, 128)])
def test_pool_against_a_model(iq, n_seqs, per, num_pages, page_rows):
    """Reserve, release and fork in turn, until pages run out and sequences share many; every number equal after every call."""
    rng = np.random.default_rng(n_seqs)
    pool, m = iq.new_page_pool(n_seqs, per, num_pages, page_rows), Model(n_seqs, per, num_pages, page_rows)
    rows = br.Rows(rng, num_pages, 1, page_rows, 128, 2) if num_pages <= 300 else None
    cache = upload(iq, rows, pool.block_table, page_rows) if rows else None
    shape = iq.Shape(n_seqs, 1, 1, 128, per * page_rows, 2)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    cap = per * page_rows
    for step in range(12):
        lo = rng.integers(-5, cap + 1, n_seqs)
        hi = lo + rng.integers(-3, max(2, cap // (1 + step % 3)), n_seqs)
        if step % 3 == 0:
            lo[:] = 0
        if step % 3 < 2:
            iq.iq_reserve_pages(pool, ints(lo.tolist()), ints(hi.tolist()), status_dev=status)
            m.reserve(lo, hi)
        else:
            iq.iq_release_pages(pool, ints(lo.tolist()), ints(hi.tolist()), status_dev=status)
            m.release(lo, hi)
        m.same(pool)
        if cache is not None and n_seqs > 1:
            n = int(rng.integers(1, min(n_seqs, 9)))
            perm = rng.permutation(n_seqs)
            dst = perm[:n]
            src = rng.choice(perm[n:], n)
            if step % 4 == 3:  # conflicts: a dst twice, one that is a src, numbers out of range
                dst[0] = dst[-1]
                src[-1] = dst[n // 2]
            length = rng.integers(0, cap + 1, n)
            end = np.zeros(n_seqs, np.int64)
            end[dst] = cap
            iq.iq_release_pages(pool, ints([0] * n_seqs), ints(end.tolist()), status_dev=status)
            m.release([0] * n_seqs, end)
            m.same(pool)
            iq.iq_fork_sequences(shape, cache, pool, ints(src.tolist()), ints(dst.tolist()), ints(length.tolist()), status_dev=status)
            for p, q, part in m.fork(src.tolist(), dst.tolist(), length.tolist()):
                k = -(-part // 128) * 128
                for side in range(2):
                    rows.codes[side][q, :, :k] = rows.codes[side][p, :, :k]
                    rows.scales[side][q, :, :k] = rows.scales[side][p, :, :k]
            m.same(pool)
    if cache is not None:
        same(cache, rows)
    assert status.tolist() == [m.flags, 0, m.count, 0]


def test_fork_refusals_are_counted_and_leave_the_pool_alone(iq):
    pool, m = iq.new_page_pool(4, 2, 6, 128), Model(4, 2, 6, 128)
    rows = br.Rows(np.random.default_rng(1), 6, 2, 128, 256, 4)
    cache = upload(iq, rows, pool.block_table, 128)
    shape = iq.Shape(4, 2, 2, 256, 256, 4)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    iq.iq_reserve_pages(pool, ints([0] * 4), ints([256, 0, 0, 0]), status_dev=status)
    m.reserve([0] * 4, [256, 0, 0, 0])
    src, dst, n = [0, -1, 4, 0, 0, 0, 2], [1, 1, 1, 7, 3, 0, 1], [100, 1, 1, 1, 257, 5, 9]
    iq.iq_fork_sequences(shape, cache, pool, ints(src), ints(dst), ints(n), status_dev=status)
    copies = m.fork(src, dst, n)
    m.same(pool)
    assert copies == [(0, 2, 100)] and status.tolist() == [32, 0, 6, 0]


@pytest.mark.parametrize("d,bits,f16", [(128, 3, False), (256, 4, True), (128, 2, True)])
def test_copy_pages(iq, d, bits, f16):
    rng = np.random.default_rng(d + bits)
    rows = br.Rows(rng, 7, 3, 256, d, bits, f16)
    table = ints([[0, 1], [2, 3]])
    cache = upload(iq, rows, table, 256)
    shape = iq.Shape(2, 3, 3, d, 512, bits)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    iq.iq_copy_pages(shape, cache, ints([0, 3, 2, -1, 4]), ints([5, 6, 2, 1, 7]), status_dev=status)
    for side in range(2):
        for s, t in ((0, 5), (3, 6)):
            rows.codes[side][t] = rows.codes[side][s]
            rows.scales[side][t] = rows.scales[side][s]
    same(cache, rows)
    assert status.tolist() == [4, 0, 2, 0]


def test_a_speculative_step_and_a_graph_of_it(iq):
    """The calls as a server makes them, captured once and replayed: pages for the drafted rows, the rows appended, the tree's attention,
    the accepted rows kept, the rest given back. Afterwards the cache holds what appending the accepted rows alone leaves, and a decode
    step over it gives the accepted token's output."""
    B, T, H, hk, d, pr, per = 3, 6, 8, 2, 128, 128, 6
    rng = np.random.default_rng(2)
    cb = iq.iq_int8_codebook(d)
    rot = torch.empty(iq.iq_rotation_floats(d, hk), dtype=torch.float32, device="cuda")
    iq.iq_make_rotation(d, hk, 5, None, rot)
    shape = iq.Shape(B, H, hk, d, per * pr)
    ctx = np.array([250, 3, 511], np.int32)
    accepted = np.array([[0, 2, 5, 0], [0, 1, 0, 0], [1, 3, 4, 5]], np.int32)
    n_acc = np.array([3, 1, 4], np.int32)
    see = np.zeros((B, T, T), bool)
    for b in range(B):
        for t in range(T):
            see[b, t, t] = True
        path = accepted[b, :n_acc[b]]
        for i, t in enumerate(path):
            see[b, t, path[:i]] = True
    new = [torch.from_numpy(rng.standard_normal((B, 600, hk, d)).astype(np.float16)).cuda() for _ in range(2)]
    draft = [torch.from_numpy(rng.standard_normal((B, T, hk, d)).astype(np.float16)).cuda() for _ in range(2)]
    q = torch.from_numpy(rng.standard_normal((B, T, H, d)).astype(np.float16)).cuda()
    zero, lens, mask, keep, n_keep = ints([0] * B), dev(ctx), dev(br.mask_words(see)), dev(accepted), dev(n_acc)
    ends, caps, new_len = lens + T, ints([per * pr] * B), lens + n_keep

    def fresh():
        pool = iq.new_page_pool(B, per, B * per, pr)
        cache = iq.new_paged_cache(shape, B * per, pr, pool.block_table)
        status = torch.zeros(4, dtype=torch.int32, device="cuda")
        iq.iq_reserve_pages(pool, zero, lens, status_dev=status)
        iq.iq_quantize_append(shape, rot, cb, new[0], new[1], zero, lens, 600, cache, status)
        return pool, cache, status

    pool, cache, status = fresh()
    ws = torch.empty(iq.iq_tree_workspace_bytes(shape, T), dtype=torch.uint8, device="cuda")
    out = torch.zeros((B, T, H, d), dtype=torch.float32, device="cuda")

    def step():
        iq.iq_reserve_pages(pool, lens, ends, status_dev=status)
        iq.iq_quantize_append(shape, rot, cb, draft[0], draft[1], lens, None, T, cache, status)
        iq.iq_tree_attention(shape, rot, cb, q, cache, lens, mask, None, ws, out, status_dev=status)
        iq.iq_keep_rows(shape, cache, lens, keep, n_keep, status_dev=status)
        iq.iq_release_pages(pool, new_len, caps, status_dev=status)

    step()
    eager = out.clone()
    table = pool.block_table.clone()
    # the same state, its step captured and replayed (once: a replay is a step)
    pool, cache, status = fresh()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, eager) and torch.equal(pool.block_table, table)
    assert int(status[0]) == 0 and int(status[2]) == 0
    # the accepted rows alone
    pool2, cache2, status2 = fresh()
    iq.iq_reserve_pages(pool2, lens, new_len, status_dev=status2)
    picked = [torch.stack([x[b, accepted[b]] for b in range(B)]) for x in draft]
    iq.iq_quantize_append(shape, rot, cb, picked[0].contiguous(), picked[1].contiguous(), lens, n_keep, 4, cache2, status2)
    ks = [torch.zeros((B, per * pr, hk, d), dtype=torch.float16, device="cuda") for _ in range(4)]
    iq.iq_reconstruct_rows(shape, rot, cb, cache, new_len, ks[0], ks[1])
    iq.iq_reconstruct_rows(shape, rot, cb, cache2, new_len, ks[2], ks[3])
    assert torch.equal(ks[0], ks[2]) and torch.equal(ks[1], ks[3])
    last = torch.stack([q[b, accepted[b, n_acc[b] - 1]] for b in range(B)]).contiguous()
    dws = iq.DecodeWorkspace(shape, iq.iq_suggest_splits(shape, 520))
    iq.decode_step(shape, rot, cb, last, cache, new_len, dws)
    mine = torch.stack([eager[b, accepted[b, n_acc[b] - 1]] for b in range(B)])
    # two kernels of 21 and 22 bits of q~; the framework's bound for an output
    assert bool(((mine - dws.out).abs() <= 2e-3 + 1e-3 * dws.out.abs()).all())
