"""The calls around a step's attention: places of its tokens, rotary positions, packed rows appended; and a run of them together, a server
that takes prompts in pieces."""
import math

import numpy as np
import pytest

import branching as br
import oracle

torch = pytest.importorskip("torch")
from steps import attention  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def iq():
    import paper_2608_08081_b200 as m
    return m


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------------------------------------- places
def plan_model(ctx, n_new, room, t_cap, table, page_rows, num_pages):
    start, pos, seq, slot = [0], np.full(room, -2 ** 31, np.int64), np.full(room, -1), np.full(room, -1, np.int64)
    bad = out = 0
    at = 0
    for b, n in enumerate(np.maximum(n_new, 0)):
        for i in range(n):
            if at < room:
                p = int(ctx[b]) + i
                pos[at], seq[at] = p, b
                if not 0 <= p < t_cap:
                    out += 1
                elif table is None:
                    slot[at] = b * t_cap + p
                else:
                    page = int(table[b, p // page_rows])
                    if 0 <= page < num_pages:
                        slot[at] = page * page_rows + p % page_rows
                    else:
                        bad += 1
            at += 1
        start.append(min(at, room))
    left = max(0, at - room)
    flags = (1 if out + left else 0) | (4 if bad else 0)
    return start, pos, seq, slot, [flags, 0, out + bad + left, 0]


@pytest.mark.parametrize("B,room,page_rows", [(1, 1, 0), (1, 300, 128), (5, 64, 0), (8, 700, 128), (300, 900, 256), (257, 1500, 128), (2000, 4000, 0)])
@pytest.mark.parametrize("kind", ["tokens", "mixed", "odd"])
def test_plan(iq, B, room, page_rows, kind):
    rng = np.random.default_rng(B + room)
    t_cap = 1024
    ctx = rng.integers(0, 900, B)
    n_new = rng.integers(0, max(2, 2 * room // B), B) if kind != "mixed" else np.where(np.arange(B) % 7 == 0, 5, rng.integers(0, 2, B))
    if kind == "odd":
        ctx[::3], n_new[1::4] = rng.integers(-5, 1100, len(ctx[::3])), -3
    table, num_pages = None, 0
    if page_rows:
        per = t_cap // page_rows
        num_pages = B * per
        table = rng.permutation(num_pages).reshape(B, per)
        if kind == "odd":
            table[rng.random(table.shape) < 0.2] = -1
            table[0, -1] = num_pages
    shape = iq.Shape(B, 4, 1, 128, t_cap)
    start, pos, seq = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (B + 1, room, room))
    slot = torch.full((room,), 77, dtype=torch.int64, device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    kw = dict(block_table=None if table is None else ints(table), page_rows=page_rows, num_pages=num_pages)
    iq.iq_plan_tokens(shape, ints(ctx), ints(n_new), start, pos, seq, slot, status_dev=status, **kw)
    w = plan_model(ctx, n_new, room, t_cap, table, page_rows, num_pages)
    assert start.tolist() == w[0]
    assert pos.tolist() == w[1].tolist() and seq.tolist() == w[2].tolist() and slot.tolist() == w[3].tolist()
    assert status.tolist() == w[4]
    # outputs that are not asked for
    start2 = torch.full_like(start, 77)
    iq.iq_plan_tokens(shape, ints(ctx), ints(n_new), start2, n_tokens_max=room, **kw)
    assert torch.equal(start, start2)


def test_plan_without_sequences(iq):
    start, pos = torch.full((1,), 7, dtype=torch.int32, device="cuda"), torch.full((9,), 7, dtype=torch.int32, device="cuda")
    iq.iq_plan_tokens(iq.Shape(0, 4, 1, 128, 128), ints([]), ints([]), start, pos)
    assert start.tolist() == [0] and pos.tolist() == [iq.IQ_NO_POSITION] * 9


# ------------------------------------------------------------------------------------------------------------ rotary
def rotary_model(x, positions, freq, magnitude, r, interleaved):
    """x fp16 [n][H][d] -> 64 bits; complex numbers turned by their angles."""
    y = x.astype(np.float64)
    i = np.arange(r // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
    w = magnitude * np.exp(1j * (np.asarray(positions, np.float64)[:, None] * freq))[:, None]
    u = (y[..., a] + 1j * y[..., b]) * w
    y[..., a], y[..., b] = u.real, u.imag
    return y


def near(got, want, x, magnitude, r):
    """An element is off by the angle (2^-24 of half a turn, and the sine's 2^-23) and three roundings of 2^-24, times the pair's size; then half a
    step of binary16."""
    pair = np.abs(x.astype(np.float64)).max(-1, keepdims=True) * math.sqrt(2) * magnitude
    lim = pair * (math.pi * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -11 * np.abs(want) + 2.0 ** -25
    e = np.abs(got.double().cpu().numpy() - want)
    assert np.all(e <= lim), float((e / lim).max())
    assert np.array_equal(got.cpu().numpy()[..., r:], x[..., r:])


FREQS = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0, base=500000.0),
         dict(scaling="parts", factor=16.0, original_len=4096), dict(scaling="parts", factor=2.5, original_len=100, beta_fast=8.0, beta_slow=2.0)]


def frequencies(r, base=10000.0, scaling="none", factor=1.0, original_len=1, beta_fast=32.0, beta_slow=1.0):
    if scaling == "base":
        base = base * factor ** (r / (r - 2))
    f = base ** (-2.0 * np.arange(r // 2) / r)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "parts":
        def pair(t):
            return r * math.log(original_len / (2 * math.pi * t)) / (2 * math.log(base))

        low, high = max(math.floor(pair(beta_fast)), 0), min(math.ceil(pair(beta_slow)), r - 1)
        k = np.clip((np.arange(r // 2) - low) / max(high - low, 0.001), 0, 1)
        return f / factor * k + f * (1 - k), 0.1 * math.log(factor) + 1
    return f, 1.0


@pytest.mark.parametrize("d,r", [(128, 128), (128, 16), (128, 96), (256, 256), (256, 64)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kw", FREQS)
def test_rotary(iq, d, r, interleaved, kw):
    rng = np.random.default_rng(d + r)
    n, H, hk = 37, 6, 2
    x = [(3 * rng.standard_normal((n, h, d))).astype(np.float16) for h in (H, hk)]
    positions = rng.integers(0, 1 << 20, n)
    positions[:3] = 0, 1, 131072
    f, m = frequencies(r, **kw)
    rot = iq.iq_make_rotary(r, interleaved=interleaved, **kw)
    assert abs(rot.magnitude - m) <= 2.0 ** -24 * m
    q, k = (torch.from_numpy(a).cuda() for a in x)
    shape = iq.Shape(1, H, hk, d, 128)
    yq, yk = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    iq.iq_apply_rotary(shape, rot, q, k, ints(positions), yq, yk)
    # (the model's own angle in 64 bits is off by 2^-53 of it: 1e-10 at position 2^20)
    near(yq, rotary_model(x[0], positions, f, m, r, interleaved), x[0], m, r)
    near(yk, rotary_model(x[1], positions, f, m, r, interleaved), x[1], m, r)
    iq.iq_apply_rotary(shape, rot, q, k, ints(positions))  # in place
    assert torch.equal(q, yq) and torch.equal(k, yk)


@pytest.mark.parametrize("n,H,hk", [(1, 32, 8), (1, 1, 1), (17, 4, 1), (300, 64, 8), (1000, 1, 1)])
@pytest.mark.parametrize("d", [128, 256])
def test_rotary_sizes_and_strides(iq, n, H, hk, d):
    rng = np.random.default_rng(n)
    qkv = torch.from_numpy(rng.standard_normal((n, H + 2 * hk, d)).astype(np.float16)).cuda()
    before = qkv.clone()
    positions = rng.integers(0, 5000, n)
    rot, shape = iq.iq_make_rotary(d // 2), iq.Shape(1, H, hk, d, 128)
    f, _ = frequencies(d // 2)
    iq.iq_apply_rotary(shape, rot, qkv[:, :H], qkv[:, H:H + hk], ints(positions))
    assert torch.equal(qkv[:, H + hk:], before[:, H + hk:])
    x = before.cpu().numpy()
    near(qkv[:, :H + hk], rotary_model(x[:, :H + hk], positions, f, 1.0, d // 2, False), x[:, :H + hk], 1.0, d // 2)
    # the keys alone, of tokens in a batch, heads before tokens
    k = before[:, H:H + hk].transpose(0, 1).contiguous().transpose(0, 1)[None]
    out = torch.zeros((1, n, hk, d), dtype=torch.float16, device="cuda")
    iq.iq_apply_rotary(shape, rot, None, k, ints(positions), None, out)
    assert torch.equal(out[0], qkv[:, H:H + hk])


def test_rotary_positions(iq):
    """Negative positions turn back; far ones are exact; places without a token are left as they are."""
    shape = iq.Shape(1, 1, 1, 128, 128)
    x = np.random.default_rng(1).standard_normal((5, 1, 128)).astype(np.float16)
    q = torch.from_numpy(x).cuda()
    f = np.array([2 * math.pi * (0.25 + 1 / 3 * i) for i in range(64)])
    rot = iq.iq_make_rotary(128, inv_freq=f)
    positions = [-1, 2 ** 31 - 1, iq.IQ_NO_POSITION, -(2 ** 31) + 1, 3]
    y = torch.full_like(q, 7.0)
    iq.iq_apply_rotary(shape, rot, q, None, ints(positions), y)
    # the turns as whole numbers of 2^-64, in python's integers
    from fractions import Fraction
    for t, p in enumerate(positions):
        if p == iq.IQ_NO_POSITION:
            assert bool((y[t] == 7.0).all())
            continue
        turn = np.array([float(Fraction((p * w) % 2 ** 64, 2 ** 64)) for w in rot.turns])
        u = (x[t, :, :64].astype(np.float64) + 1j * x[t, :, 64:]) * np.exp(2j * np.pi * turn)
        near(y[t:t + 1], np.concatenate((u.real, u.imag), -1)[None], x[t:t + 1], 1.0, 128)
    z = iq.iq_make_rotary(64, inv_freq=[0.0] * 32, magnitude=0.5)
    iq.iq_apply_rotary(shape, z, q, None, ints([1, 2, 3, 4, 5]), y)
    assert torch.equal(y[..., :64], q[..., :64] * 0.5) and torch.equal(y[..., 64:], q[..., 64:])


def test_rotary_in_a_graph(iq):
    shape, rot = iq.Shape(1, 4, 2, 128, 128), iq.iq_make_rotary(128, base=500000.0)
    q, k = torch.randn((9, 4, 128), device="cuda").half(), torch.randn((9, 2, 128), device="cuda").half()
    pos, yq, yk = ints(np.arange(9)), torch.zeros_like(q), torch.zeros_like(k)
    iq.iq_apply_rotary(shape, rot, q, k, pos, yq, yk)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        iq.iq_apply_rotary(shape, rot, q, k, pos, yq, yk)
    pos += 1000
    g.replay()
    got = yq.clone()
    iq.iq_apply_rotary(shape, rot, q, k, pos, yq, yk)
    assert torch.equal(got, yq)


# ------------------------------------------------------------------------------------------------------ packed append
@pytest.mark.parametrize("d,bits", [(128, 3), (128, 4), (256, 3), (256, 2)])
@pytest.mark.parametrize("lens", [[1, 1, 1], [3, 0, 130], [0, 1, 7], [300, 129, 1]])
@pytest.mark.parametrize("page_rows", [0, 128])
def test_packed_append(iq, d, bits, lens, page_rows):
    """The same bytes as the padded call's."""
    rng = np.random.default_rng(sum(lens))
    B, hk, t_cap = len(lens), 2, 512
    shape, cb = iq.Shape(B, 4, hk, d, t_cap, bits), iq.iq_lloyd_max_codebook(d, bits)
    rot = torch.empty(iq.iq_rotation_floats(d, hk), dtype=torch.float32, device="cuda")
    iq.iq_make_rotation(d, hk, 5, None, rot)
    N, T = sum(lens) + 3, max(lens)
    k, v = (torch.from_numpy(rng.standard_normal((N, hk, d)).astype(np.float16)).cuda() for _ in range(2))
    start = ints(np.concatenate(([0], np.cumsum(lens))))
    pos = ints([5, 200, 120])
    table = ints(np.arange(B * 4).reshape(B, 4)[:, ::-1].copy()) if page_rows else None

    def cache():
        return iq.new_paged_cache(shape, B * 4, page_rows, table) if page_rows else iq.new_cache(shape)

    a, b, status = cache(), cache(), torch.zeros(4, dtype=torch.int32, device="cuda")
    iq.iq_quantize_append_packed(shape, rot, cb, k, v, pos, start, T, a, status)
    pk, pv = (torch.zeros((B, max(1, T), hk, d), dtype=torch.float16, device="cuda") for _ in range(2))
    at = 0
    for i, n in enumerate(lens):
        pk[i, :n], pv[i, :n] = k[at:at + n], v[at:at + n]
        at += n
    iq.iq_quantize_append(shape, rot, cb, pk, pv, pos, ints(lens), T, b)
    assert status.tolist()[0] == 0
    for x, y in ((a.k_codes, b.k_codes), (a.v_codes, b.v_codes), (a.k_scales, b.k_scales), (a.v_scales, b.v_scales)):
        assert torch.equal(x, y)


# ------------------------------------------------------------------------------------------------- a run of the calls
@pytest.mark.parametrize("d,H,hk,window", [(128, 8, 2, 0), (256, 4, 2, 0), (128, 8, 2, 200)])
def test_a_server_that_takes_prompts_in_pieces(iq, d, H, hk, window):
    """Requests come and go through a pool of pages: each step plans its tokens, reserves pages, turns queries and keys, appends and attends.
    Every output is checked against the definition over the rows that the cache then holds, and those rows against the prompts appended at once."""
    rng = np.random.default_rng(d)
    B, t_cap, bits, sinks = 3, 1024, 3, 4
    shape, cb = iq.Shape(B, H, hk, d, t_cap, bits), iq.iq_lloyd_max_codebook(d, bits)
    levels = np.array(cb.levels, np.float32)
    qu = rng.standard_normal((hk, d // 4, 2, 4))
    quats = (qu / np.linalg.norm(qu, axis=-1, keepdims=True)).reshape(hk, d // 4, 8).astype(np.float32)
    rot = torch.from_numpy(quats).cuda()
    rotary = iq.iq_make_rotary(d // 2, scaling="parts", factor=4.0, original_len=256)
    pool = iq.new_page_pool(B, t_cap // 128, 20, 128)
    cache = iq.new_paged_cache(shape, 20, 128, pool.block_table)
    ws = torch.empty(iq.iq_chunk_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    total = [700, 130, 1]
    x = [(rng.standard_normal((n + 4, H + 2 * hk, d))).astype(np.float16) for n in total]  # prompts and four tokens after them
    done = [0, 0, 0]
    start, places = torch.zeros(B + 1, dtype=torch.int32, device="cuda"), 450
    positions, sequences = (torch.zeros(places, dtype=torch.int32, device="cuda") for _ in range(2))
    slots = torch.zeros(places, dtype=torch.int64, device="cuda")
    while any(a < n + 4 for a, n in zip(done, total)):
        new = [min(300 if a < n else 1, (n if a < n else n + 4) - a) for a, n in zip(done, total)]
        ctx, n_new, end = ints(done), ints(new), ints([a + n for a, n in zip(done, new)])
        qkv = torch.zeros((places, H + 2 * hk, d), dtype=torch.float16, device="cuda")
        qkv[:sum(new)] = torch.from_numpy(np.concatenate([x[b][done[b]:done[b] + new[b]] for b in range(B)])).cuda()
        q, k, v = qkv[:, :H], qkv[:, H:H + hk], qkv[:, H + hk:]
        iq.iq_reserve_pages(pool, ctx, end, status)
        iq.iq_plan_tokens(shape, ctx, n_new, start, positions, sequences, slots, block_table=pool.block_table, page_rows=128, num_pages=20, status_dev=status)
        iq.iq_apply_rotary(shape, rotary, q, k, positions)
        iq.iq_quantize_append_packed(shape, rot, cb, k, v, ctx, start, max(new), cache, status)
        out = torch.full((places, H, d), 7.0, dtype=torch.float16, device="cuda")
        iq.iq_chunk_attention(shape, rot, cb, q, cache, ctx, ws, out, token_start=start, window=window, sinks=sinks, status_dev=status)
        assert status.tolist()[0] == 0
        # the rows that the plan names hold the tokens' norms
        norms = v[:sum(new)].double().norm(dim=-1).float()
        held = cache.v_scales.transpose(1, 2).reshape(-1, hk)[slots[:sum(new)]]
        assert bool(((held - norms).abs() <= 2.0 ** -23 * norms).all())
        rows = br.Rows.__new__(br.Rows)
        rows.codes = br.Rows.codes_of(cache.k_codes.cpu().numpy(), cache.v_codes.cpu().numpy(), d, bits)
        rows.scales = [cache.k_scales.cpu().numpy(), cache.v_scales.cpu().numpy()]
        qs = np.split(q[:sum(new)].cpu().numpy(), np.cumsum(new)[:-1])
        want = attention(rows, pool.block_table.cpu().numpy(), 128, quats, levels, levels, qs, done, new, True, window, sinks, t_cap)
        at = 0
        for b in range(B):
            o, _, tol, _ = want[b]
            e = (out[at:at + new[b]].double().cpu() - o).norm(dim=-1)
            assert bool((e <= tol + 2.0 ** -11 * o.norm(dim=-1) + 2.0 ** -20).all())
            at += new[b]
        assert bool((out[at:] == 7.0).all())
        done = [a + n for a, n in zip(done, new)]
    # the prompts at once, padded: the same rows
    again = iq.new_cache(shape)
    T = max(total) + 4
    kv = [torch.zeros((B, T, hk, d), dtype=torch.float16, device="cuda") for _ in range(2)]
    for b, y in enumerate(x):
        kv[0][b, :len(y)], kv[1][b, :len(y)] = (torch.from_numpy(y[:, H + i * hk:H + (i + 1) * hk]).cuda() for i in range(2))
    iq.iq_apply_rotary(shape, rotary, None, kv[0], torch.arange(T, dtype=torch.int32, device="cuda").repeat(B))
    iq.iq_quantize_append(shape, rot, cb, kv[0], kv[1], ints([0] * B), ints([len(y) for y in x]), T, again)
    table = pool.block_table.long().cpu()
    for b, y in enumerate(x):
        r = torch.arange(len(y))
        assert torch.equal(cache.k_codes.cpu()[table[b, r // 128], :, r % 128], again.k_codes.cpu()[b][:, r].transpose(0, 1))
        assert torch.equal(cache.v_scales.cpu()[table[b, r // 128], :, r % 128], again.v_scales.cpu()[b][:, r].transpose(0, 1))


def test_one_token_is_a_decode_step(iq):
    """A step of one token per sequence: what iq_decode_attention and iq_combine_splits give, within the two calls' roundings."""
    from steps import Step
    c = Step(iq, 31, B=3, H=8, hk=2, ctx=[600, 0, 129], tokens=1).upload()
    out, lse = c.outputs()
    c.call(out, lse)
    w = iq.DecodeWorkspace(c.shape, 8)
    iq.decode_step(c.shape, c.rot, c.cb, c.q_dev[:, 0].contiguous(), c.cache, c.ctx_dev + 1, w)
    want = c.expected()
    for b in range(3):
        o, _, tol, _ = want[b]
        e = (out[b].double() - w.out[b].double()).norm(dim=-1).cpu()
        assert bool((e <= tol + 2.0 ** -11 * o.norm(dim=-1) + 2e-5 * o.norm(dim=-1)).all())
    assert bool(((lse[:, 0] - w.lse).abs() < 1e-4).all())
