"""Branching generation over the packed cache, as cases that can be timed and compared.

Four kinds of call:

  tree    attention for a tree of drafted tokens: every drafted token of a sequence attends to the cached context and to its own
          ancestors in the tree, whose rows were appended behind the context (speculative decoding's verification; a chain of
          tokens is a chunk of a prompt). With ``window``: the context that is further back than the window is left out, but for
          the first ``sinks`` rows; with one token that is a decode step of a sliding-window layer.
  keep    after verification: the rows of the accepted drafted tokens are moved together behind the context
  fork    sequences that branch off others in a paged cache: whole pages are shared, the last, partly filled one is copied; the
          branches that lost the step before give their pages back first
  pages   a step of a paged server: the pages that the last step did not need are released, those that the next one may write
          are reserved

Head counts, head sizes, contexts and batches are those of this repository's configurations (query heads / KV heads 4/1, 32/4,
16/8, 32/8, 64/8; head_dim 128 and 256; contexts up to 32 K rows, batches up to 32) and odd sizes between them; sliding windows
and page tables go further, where only what is visible is held.

The plain form of an operator is written with elementary torch operations; it takes the same packed cache, whose format it
reads on its own.
"""
import math
import random

import torch

own = False

HEADS = ((4, 1), (32, 4), (16, 8), (32, 8), (64, 8))
MAX_ROWS = 32 * 32768 * 8    # rows x KV heads of the largest cache
# Max's levels for a unit Gaussian with 4, 8 and 16 cells, upper halves
GAUSS = {2: (0.4528, 1.510), 3: (0.2451, 0.7560, 1.344, 2.152),
         4: (0.1284, 0.3881, 0.6568, 0.9424, 1.256, 1.618, 2.069, 2.733)}


# ---------------------------------------------------------------------------------------------------------------- cases
def _case(kind, **kw):
    case = dict(kind=kind, batch=1, heads=32, kv_heads=8, head_dim=128, ctx=4096, bits=3, grid="int8", scales="fp32", page_rows=0,
                tokens=8, ragged=False, window=0, sinks=0)
    case.update(kw)
    return case


def listed():
    def c(name, kind, **kw):
        return dict(_case(kind, **kw), name=name)

    return [
        # five drafted tokens of one short chat: latency
        c("tree_one_1k", "tree", ctx=1000, tokens=5),
        # a wide tree over a long context, one sequence: as many drafted tokens as drafters make
        c("tree_one_32k_60", "tree", ctx=32700, tokens=60),
        # a batched server at long, ragged contexts, four drafted tokens each: the largest cache
        c("tree_batch32_32k", "tree", batch=32, heads=64, ctx=32760, tokens=4, ragged=True),
        # wide heads, 4-bit codes of binary16 levels in pages with binary16 scales, trees of different sizes
        c("tree_d256_4bit_paged", "tree", batch=4, heads=16, head_dim=256, ctx=16000, bits=4, grid="fp16", scales="fp16", page_rows=256,
          tokens=13, ragged=True),
        # a decode step of a sliding-window layer, one sequence
        c("window_one", "tree", ctx=32767, tokens=1, window=4096, sinks=4),
        # the same for a batch far beyond the window, whose pages outside it have been given back
        c("window_batch64_paged", "tree", batch=64, heads=64, ctx=131000, page_rows=128, tokens=1, window=1024, sinks=64, ragged=True),
        # three of five drafted tokens accepted
        c("keep_one", "keep", ctx=1000, tokens=5),
        # a batch of wide trees, up to a quarter accepted
        c("keep_batch64", "keep", batch=64, heads=64, ctx=1500, tokens=60, page_rows=256, ragged=True),
        # one prompt branches into four
        c("fork_four", "fork", batch=1, ctx=1000, page_rows=128, tokens=4),
        # every sequence of a batch branches in two, pages of 512 rows
        c("fork_batch64", "fork", batch=64, heads=64, ctx=8000, page_rows=512, tokens=1, ragged=True),
        # a small server's page table
        c("pages_batch8", "pages", batch=8, ctx=8000, page_rows=128, tokens=60, ragged=True),
        # a large one's
        c("pages_batch512", "pages", batch=512, ctx=32000, page_rows=128, tokens=200, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(("tree", "window", "keep", "fork", "pages"), (5, 2, 1, 1, 1))[0]
    heads, kv_heads = rng.choice(HEADS)
    head_dim = rng.choice((128, 128, 256))
    bits = rng.choices((3, 2, 4), (3, 1, 1))[0]
    grid = rng.choice(("int8", "int8", "fp16"))
    scales = rng.choice(("fp32", "fp32", "fp16"))
    page_rows = rng.choice((0, 0, 128, 512))
    ragged = rng.random() < 0.7
    common = dict(heads=heads, kv_heads=kv_heads, head_dim=head_dim, bits=bits, grid=grid, scales=scales, ragged=ragged)
    if kind == "tree":
        ctx = _log_int(rng, 1, 32000)
        rows = MAX_ROWS * 128 // head_dim
        batch = _log_int(rng, 1, max(1, min(32, rows // (ctx * kv_heads))))
        tokens = _log_int(rng, 1, 64)
        # the work of the largest listed case: 32 sequences, mean context 24 K, 64 heads, 4 tokens, d = 128
        most = 32 * 24000 * 64 * 4 * 128 // max(1, batch * ctx * heads * head_dim)
        return _case("tree", batch=batch, ctx=ctx, tokens=max(1, min(tokens, most)), page_rows=page_rows, **common)
    if kind == "window":
        window, sinks = _log_int(rng, 1, 8192), rng.choice((0, 1, 4, 64, 200))
        return _case("tree", batch=_log_int(rng, 1, 64), ctx=_log_int(rng, 1, 130000), tokens=rng.choice((1, 1, 3, 16)), window=window,
                     sinks=sinks, page_rows=rng.choice((128, 512)), **common)
    if kind == "keep":
        return _case("keep", batch=_log_int(rng, 1, 64), ctx=_log_int(rng, 1, 2000), tokens=_log_int(rng, 1, 64), page_rows=page_rows, **common)
    if kind == "fork":
        return _case("fork", batch=_log_int(rng, 1, 64), ctx=_log_int(rng, 1, 8000), tokens=1, page_rows=rng.choice((128, 256, 512)), **common)
    return _case("pages", batch=_log_int(rng, 1, 512), ctx=_log_int(rng, 100, 32000), tokens=_log_int(rng, 1, 400),
                 page_rows=rng.choice((128, 256, 512)), ragged=ragged)


def _context(c):
    """Context rows of every sequence: the same for every seed, so that the work is the case's."""
    return [max(1, int(c["ctx"] * (0.5 + 0.5 * ((i * 0.6180339887 + 0.37) % 1.0)))) if c["ragged"] else c["ctx"] for i in range(c["batch"])]


def _tokens(c):
    """Drafted tokens of every sequence, at most c["tokens"]."""
    n = c["tokens"]
    return [max(1, n - (i * 5) % 3 * (n // 4)) if c["ragged"] else n for i in range(c["batch"])]


def _accepted(c):
    return [max(1, min(n, (n + 3) // 4 + (i % 3))) for i, n in enumerate(_tokens(c))]


def _cap(c, more):
    unit = max(128, c["page_rows"])
    return -(-(c["ctx"] + more) // unit) * unit


def _visible(c, ctx, j):
    """Context rows that a drafted token at depth j (0: the first) sees."""
    if c["window"] <= 0:
        return ctx
    first = max(0, ctx + j - c["window"] + 1)
    return min(ctx, c["sinks"] + max(0, ctx - max(first, c["sinks"])))


# --------------------------------------------------------------------------------------------------------------- inputs
def _levels(bits, grid):
    """Levels and thresholds of a Lloyd-Max codebook: levels on an 8-bit grid, or exact binary16 values."""
    up = GAUSS[bits]
    if grid == "int8":
        delta = float(torch.tensor(up[-1] / 127.0, dtype=torch.float32))
        up = [float(torch.tensor(round(x / delta) * delta, dtype=torch.float32)) for x in up]
    else:
        up = [float(torch.tensor(x).half()) for x in up]
    lv = [-x for x in reversed(up)] + list(up)
    return lv, [0.5 * (a + b) for a, b in zip(lv, lv[1:])]


def _pack(codes, bits):
    """Codes (int32, a multiple of 32 along the last axis) -> the packed 32-bit words of the run."""
    sh = 4 * torch.arange(8, device=codes.device, dtype=torch.int32)
    if bits == 4:
        return (codes.unflatten(-1, (-1, 8)) << sh).sum(-1, dtype=torch.int32)
    if bits == 2:
        g = codes.unflatten(-1, (-1, 2, 8))
        return ((g[..., 0, :] << sh) + (g[..., 1, :] << (sh + 2))).sum(-1, dtype=torch.int32)
    g = codes.unflatten(-1, (-1, 4, 8))
    k = torch.arange(3, device=codes.device, dtype=torch.int32)[:, None]
    return ((g[..., :3, :] << sh) + (((g[..., 3:, :] >> k) & 1) << (sh + 3))).sum(-1, dtype=torch.int32).flatten(-2)


def _cache(c, gen, rows_shape):
    """A packed cache of rows whose rotated coordinates are Gaussian: arrays [n][kv_heads][rows][...], a few heads at a time."""
    n, hk, rows = rows_shape
    d, bits = c["head_dim"], c["bits"]
    _, th = _levels(bits, c["grid"])
    dev = gen.device
    th = torch.tensor(th, device=dev)
    P = bits * d // 8
    sdt = torch.float16 if c["scales"] == "fp16" else torch.float32
    k = torch.empty((n * hk, rows, P // 4), dtype=torch.int32, device=dev)
    v = torch.empty((n * hk, rows // 128, d, 4 * bits), dtype=torch.int32, device=dev)
    step = max(1, (1 << 27) // (rows * d))
    for i in range(0, n * hk, step):
        m = min(step, n * hk - i)
        k[i:i + m] = _pack(torch.bucketize(torch.randn((m, rows, d), generator=gen, device=dev), th, out_int32=True), bits)
        v[i:i + m] = _pack(torch.bucketize(torch.randn((m, rows // 128, d, 128), generator=gen, device=dev), th, out_int32=True), bits)

    def scales():
        return (math.sqrt(d) * torch.exp(0.3 * torch.randn((n, hk, rows), generator=gen, device=dev))).to(sdt)

    return dict(k_codes=k.view(n, hk, rows, P // 4).view(torch.uint8), v_codes=v.view(n, hk, rows, P // 4).view(torch.uint8),
                k_scales=scales(), v_scales=scales())


def _tree(rng, batch, tokens):
    """Parents drawn among the tokens before: bit j of a token's mask says that it attends to drafted token j. int32 words."""
    words = (tokens + 31) // 32
    out = []
    for _ in range(batch):
        masks = []
        for t in range(tokens):
            p = rng.randint(max(-1, t - 6), t - 1)
            masks.append((masks[p] if p >= 0 else 0) | 1 << t)
        out.append([[((m >> (32 * w)) & 0xFFFFFFFF) for w in range(words)] for m in masks])
    return torch.tensor(out, dtype=torch.int64).to(torch.int32)


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed * 7919 + 11)
    rng = random.Random(seed)
    s = dict(case=c)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    B, hk, d, pr = c["batch"], c["kv_heads"], c["head_dim"], c["page_rows"]
    if c["kind"] in ("tree", "keep"):
        cap = _cap(c, c["tokens"])
        ctx, tok = _context(c), _tokens(c)
        s["ctx"], s["n_tokens"] = ints(ctx), ints(tok) if c["ragged"] else None
        if pr:
            # pages that a step can reach; those between the sinks and the window have been given back (-1)
            held = []
            for b in range(B):
                first = max(0, ctx[b] - c["window"]) // pr if c["window"] > 0 else 0
                held.append([j for j in range(cap // pr) if (j * pr < c["sinks"] or j >= first) and j * pr < ctx[b] + tok[b]])
            n = sum(map(len, held))
            pages = list(range(n))
            rng.shuffle(pages)
            table = [[-1] * (cap // pr) for _ in range(B)]
            at = 0
            for b in range(B):
                for j in held[b]:
                    table[b][j] = pages[at]
                    at += 1
            s["table"] = ints(table)
            s["cache"] = _cache(c, gen, (n, hk, pr))
        else:
            s["table"] = None
            s["cache"] = _cache(c, gen, (B, hk, cap))
    if c["kind"] == "tree":
        q = torch.randn((hk, d // 4, 2, 4), generator=gen, device=dev, dtype=torch.float64)
        s["quats"] = (q / q.norm(dim=-1, keepdim=True)).float().reshape(hk, d // 4, 8).contiguous()
        s["q"] = (2 * torch.randn((B, c["tokens"], c["heads"], d), generator=gen, device=dev)).half()
        s["mask"] = _tree(rng, B, c["tokens"]).to(dev)
        s["rot"] = s["quats"]  # (unit quaternion pairs: the rotation as the library keeps it)
    if c["kind"] == "keep":
        acc = _accepted(c)
        s["n_keep"] = ints(acc)
        s["keep"] = ints([sorted(rng.sample(range(n), k)) + [0] * (max(acc) - k) for n, k in zip(tok, acc)])
    if c["kind"] == "fork":
        ctx, per = _context(c), c["tokens"]
        cap = _cap(c, 128)
        P = cap // pr
        need = [-(-x // pr) for x in ctx]
        n = sum(need) + B * per + 7
        pages = list(range(n))
        rng.shuffle(pages)
        at, table, ref = 0, [], [0] * n
        for b in range(B):
            table.append(pages[at:at + need[b]] + [-1] * (P - need[b]))
            at += need[b]
        for b in [b for b in range(B) for _ in range(per)]:  # the branches of the last step, which a pass gives back first
            row = table[b][:ctx[b] // pr] + pages[at:at + need[b] - ctx[b] // pr]
            at += need[b] - ctx[b] // pr
            table.append(row + [-1] * (P - need[b]))
        for p in [p for row in table for p in row if p >= 0]:
            ref[p] += 1
        s["table"], s["ref"] = ints(table), ints(ref)
        s["free"] = ints(pages[at:] + [0] * at)
        # the pool's state: the number of free pages, then words that are zero between calls (the library's)
        s["state"] = ints([n - at] + [0] * (3 + (n + 31) // 32))
        s["n_free"] = s["state"][:1]
        s["cache"] = _cache(c, gen, (n, hk, pr))
        s["src"] = ints([b for b in range(B) for _ in range(per)])
        s["dst"] = ints(list(range(B, B + B * per)))
        s["rows"] = ints([ctx[b] for b in range(B) for _ in range(per)])
        s["first"], s["end"] = ints([0] * (B + B * per)), ints([0] * B + [cap] * (B * per))
    if c["kind"] == "pages":
        ctx = _context(c)
        cap = _cap(c, c["tokens"])
        P = cap // pr
        most = [-(-(x + c["tokens"]) // pr) for x in ctx]
        n = sum(most) + 13
        pages = list(range(n))
        rng.shuffle(pages)
        at, table, ref = 0, [], [0] * n
        for b in range(B):  # every third sequence shares the whole pages of the one before (a common prompt)
            shared = table[b - 1][:min(ctx[b - 1], ctx[b]) // pr] if b % 3 == 1 else []
            row = shared + pages[at:at + most[b] - len(shared)]  # with the rows that the last step reserved
            at += most[b] - len(shared)
            for p in row:
                ref[p] += 1
            table.append(row + [-1] * (P - most[b]))
        s["table"], s["ref"] = ints(table), ints(ref)
        s["free"] = ints(pages[at:] + [0] * at)
        # the pool's state: the number of free pages, then words that are zero between calls (the library's)
        s["state"] = ints([n - at] + [0] * (3 + (n + 31) // 32))
        s["n_free"] = s["state"][:1]
        s["rows"], s["first"], s["end"] = ints([x + c["tokens"] for x in ctx]), ints(ctx), ints([cap] * B)
    if own:  # the descriptors and the workspace that a program keeps beside its cache
        import paper_2608_08081_b200 as iq

        s["iq"] = iq
        s["status"] = torch.zeros(4, dtype=torch.int32, device=dev)
        if "cache" in s:
            k = s["cache"]
            n_seqs = s["table"].shape[0] if s["table"] is not None else B
            s["shape"] = iq.Shape(n_seqs, c["heads"], hk, d, cap, c["bits"])
            s["handle"] = iq.Cache(k["k_codes"], k["k_scales"], k["v_codes"], k["v_scales"], s["table"], pr)
        if "ref" in s:
            s["pool"] = iq.PagePool(s["table"], s["ref"], s["free"], s["state"], pr)
        if c["kind"] == "tree":
            lv, th = _levels(c["bits"], c["grid"])
            s["codebook"] = iq.Codebook(tuple(lv), tuple(th))
            s["workspace"] = torch.empty(iq.iq_tree_workspace_bytes(s["shape"], c["tokens"]), dtype=torch.uint8, device=dev)
            s["out"] = torch.zeros((B, c["tokens"], c["heads"], d), dtype=torch.float16, device=dev)
    return s


# ---------------------------------------------------------------------------------------------------------- plain forms
def _unpack(words, bits):
    """Packed words (int32, along the last axis) -> codes, int32."""
    sh = 4 * torch.arange(8, device=words.device, dtype=torch.int32)
    if bits == 4:
        return ((words.unsqueeze(-1) >> sh) & 15).flatten(-2)
    if bits == 2:
        return torch.stack(((words.unsqueeze(-1) >> sh) & 3, (words.unsqueeze(-1) >> (sh + 2)) & 3), -2).flatten(-3)
    w = words.unflatten(-1, (-1, 3)).unsqueeze(-1)
    top = (w >> (sh + 3)) & 1
    return torch.cat(((w >> sh) & 7, (top[..., 0, :] | top[..., 1, :] << 1 | top[..., 2, :] << 2).unsqueeze(-2)), -2).flatten(-3)


def _rotation(quats):
    """[kv_heads][d][d] fp32: the SO(4) blocks after the normalised Walsh-Hadamard transform."""
    q = quats.double()
    a, b, c, d, e, f, g, h = (q / torch.cat((q[..., :4].norm(dim=-1, keepdim=True).expand_as(q[..., :4]),
                                             q[..., 4:].norm(dim=-1, keepdim=True).expand_as(q[..., 4:])), -1)).unbind(-1)
    left = torch.stack((a, -b, -c, -d, b, a, -d, c, c, d, a, -b, d, -c, b, a), -1).unflatten(-1, (4, 4))
    right = torch.stack((e, f, g, h, -f, e, -h, g, -g, h, e, -f, -h, -g, f, e), -1).unflatten(-1, (4, 4))
    n = 4 * quats.shape[1]
    i = torch.arange(n, device=quats.device)
    x = i[:, None] & i
    x = x ^ (x >> 4)
    x = x ^ (x >> 2)
    x = (x ^ (x >> 1)) & 1
    x = x ^ (((i[:, None] & i) >> 8) & 1)
    had = (1.0 - 2.0 * x.double()) / math.sqrt(n)
    return (left @ right @ had.unflatten(0, (-1, 4))).flatten(1, 2).float()


def _blocks(s):
    """The 128-row blocks that the sequences see: their numbers [B][n] (past the end: any), and where each lies, [B][n] as a page
    (or sequence) and a block in it."""
    c, ctx = s["case"], s["ctx"].long()
    total = _cap(c, c["tokens"]) // 128
    if c["window"] > 0:
        ns = min(total, -(-c["sinks"] // 128))
        nw = min(total, (c["window"] + 127) // 128 + 1 + (c["tokens"] + 127) // 128)
        first = ((ctx - c["window"]).clamp(min=0) // 128).clamp(min=ns)
        no = torch.cat((torch.arange(ns, device=ctx.device).expand(len(ctx), ns), first[:, None] + torch.arange(nw, device=ctx.device)), 1)
    else:
        no = torch.arange(total, device=ctx.device).expand(len(ctx), total)
    at = no.clamp(max=total - 1)
    if s["table"] is None:
        return no, torch.arange(len(ctx), device=ctx.device)[:, None].expand_as(at), at
    per = c["page_rows"] // 128
    return no, s["table"].long().gather(1, at // per).clamp(min=0), at % per


def _plain_tree(s):
    c, ctx = s["case"], s["ctx"].long()
    B, T, hq, hk, d, bits = c["batch"], c["tokens"], c["heads"], c["kv_heads"], c["head_dim"], c["bits"]
    lv = torch.tensor(_levels(bits, c["grid"])[0], device="cuda")
    no, page, blk = _blocks(s)
    nb = no.shape[1]
    # packed rows of the blocks, [B][nb][hk][...]
    k = s["cache"]["k_codes"].view(torch.int32).unflatten(2, (-1, 128))[page, :, blk]
    v = s["cache"]["v_codes"].view(torch.int32).unflatten(2, (-1, 128)).flatten(3).unflatten(3, (d, 4 * bits))[page, :, blk]
    ks = s["cache"]["k_scales"].unflatten(2, (-1, 128))[page, :, blk].float() / math.sqrt(d)
    vs = s["cache"]["v_scales"].unflatten(2, (-1, 128))[page, :, blk].float() / math.sqrt(d)
    k = lv[_unpack(k, bits)].transpose(1, 2).flatten(2, 3)                                          # [B][hk][rows][d]
    v = lv[_unpack(v, bits)].permute(0, 2, 1, 4, 3).flatten(2, 3)
    ks, vs = ks.transpose(1, 2).flatten(2), vs.transpose(1, 2).flatten(2)                           # [B][hk][rows]
    rot = _rotation(s["quats"])
    q = s["q"].float().unflatten(2, (hk, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3) @ rot.transpose(1, 2)  # [B][hk][T G][d]
    z = (q @ k.transpose(2, 3)) * ks[:, :, None] / math.sqrt(d)
    # what each drafted token sees: the context (less what lies before its window), and its ancestors
    bit = torch.arange(T, device="cuda")
    anc = ((s["mask"][:, :, bit // 32] >> (bit % 32).int()) & 1).bool()                              # [B][T][T]
    pos = ctx[:, None] + anc.sum(-1) - 1                                                           # [B][T]
    lo = pos - c["window"] + 1 if c["window"] > 0 else torch.zeros_like(pos)
    anc = anc & ((pos[:, None, :] >= lo[..., None]) | (pos[:, None, :] < c["sinks"]))
    row = (no[:, :, None] * 128 + torch.arange(128, device="cuda")).flatten(1)[:, None]              # [B][1][rows]
    old = (row < ctx[:, None, None]) & ((row >= lo[..., None]) | (row < c["sinks"]))
    j = row - ctx[:, None, None]
    new = anc.gather(2, j.clamp(0, T - 1).expand(-1, T, -1)) & (j >= 0) & (j < T)
    see = (old | new).repeat_interleave(hq // hk, 1)[:, None]                                      # [B][1][T G][rows]
    z = torch.where(see, z, -math.inf)
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(m > -math.inf, m, 0.0))
    l = p.sum(-1, keepdim=True)
    o = torch.where(l > 0, (p * vs[:, :, None]) @ v / l, 0.0) @ rot
    o = o.unflatten(2, (T, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3).half()                          # [B][T][hq][d]
    if s["n_tokens"] is not None:
        o = torch.where((torch.arange(T, device="cuda") < s["n_tokens"][:, None])[..., None, None], o, 0.0)
    return o


def _arrays(s):
    return [s["cache"][n] for n in ("k_codes", "k_scales", "v_codes", "v_scales")]


def _plain_keep(s):
    c, cache = s["case"], s["cache"]
    d, bits = c["head_dim"], c["bits"]
    i = torch.arange(s["keep"].shape[1], device="cuda")
    on = i < s["n_keep"][:, None]
    b = torch.arange(c["batch"], device="cuda")[:, None].expand_as(on)[on]
    src, dst = (s["ctx"][:, None] + s["keep"]).long()[on], (s["ctx"][:, None] + i).long()[on]

    def place(t):
        return (b, t) if s["table"] is None else (s["table"].long()[b, t // c["page_rows"]], t % c["page_rows"])

    (ps, rs), (pd, rd) = place(src), place(dst)
    k, ks, v, vs = _arrays(s)
    k[pd, :, rd] = k[ps, :, rs]
    ks[pd, :, rd] = ks[ps, :, rs]
    vs[pd, :, rd] = vs[ps, :, rs]
    # V codes: the bits of the row inside the records of its block, [n][hk][block][d][words]
    w = v.view(torch.int32).unflatten(2, (-1, 128)).flatten(3).unflatten(3, (d, 4 * bits))
    blocks = torch.unique(torch.stack((torch.cat((ps, pd)), torch.cat((rs, rd)) // 128)), dim=1)  # the blocks that are touched, once each
    codes = _unpack(w[blocks[0], :, blocks[1]], bits)                                              # [blocks][hk][d][128]
    index = torch.zeros((w.shape[0], w.shape[2]), dtype=torch.long, device="cuda")
    index[blocks[0], blocks[1]] = torch.arange(blocks.shape[1], device="cuda")
    codes[index[pd, rd // 128], :, :, rd % 128] = codes[index[ps, rs // 128], :, :, rs % 128]
    w[blocks[0], :, blocks[1]] = _pack(codes, bits)


def _plain_reserve(s, first, end):
    table, ref, free, n_free = s["table"], s["ref"], s["free"], s["n_free"]
    pr = s["case"]["page_rows"]
    start = torch.arange(table.shape[1], device="cuda") * pr
    want = (start + pr > first[:, None]) & (start < end[:, None]) & (table < 0)
    k = want.flatten().cumsum(0).view_as(want) - 1
    got = want & (k < n_free)
    page = free.gather(0, (n_free - 1 - k).clamp(min=0).flatten()).view_as(table)
    table.copy_(torch.where(got, page, table))
    ref.index_add_(0, table.clamp(min=0).flatten(), got.flatten().int())
    n_free.sub_(got.sum().int())


def _plain_release(s, first, end):
    table, ref, free, n_free = s["table"], s["ref"], s["free"], s["n_free"]
    pr = s["case"]["page_rows"]
    start = torch.arange(table.shape[1], device="cuda") * pr
    drop = (table >= 0) & (start >= first[:, None]) & (start + pr <= end[:, None])
    was = ref.clone()
    ref.index_add_(0, table.clamp(min=0).flatten(), -drop.flatten().int())
    table.masked_fill_(drop, -1)
    gone = (was > 0) & (ref == 0)
    at = n_free + gone.cumsum(0) - 1
    page = torch.arange(len(ref), device="cuda", dtype=torch.int32)
    spare = torch.cat((free, free[:1]))  # (a place behind the end for the pages that stay)
    spare.scatter_(0, torch.where(gone, at, len(free)), page)
    free.copy_(spare[:-1])
    n_free.add_(gone.sum().int())


def _plain_fork(s):
    table, ref, free, n_free = s["table"], s["ref"], s["free"], s["n_free"]
    pr = s["case"]["page_rows"]
    src, dst, rows = s["src"].long(), s["dst"].long(), s["rows"].long()
    part = rows % pr != 0
    k = part.cumsum(0) - 1
    last = rows // pr
    fresh = free[(n_free - 1 - k).clamp(min=0)]
    j = torch.arange(table.shape[1], device="cuda")
    whole = j < last[:, None]
    old = table[src]
    ref.index_add_(0, old.clamp(min=0).flatten(), whole.flatten().int())
    ref.index_add_(0, fresh, part.int())
    table[dst] = torch.where(whole, old, torch.where(part[:, None] & (j == last[:, None]), fresh[:, None], -1)).int()
    n_free.sub_(part.sum().int())
    a, b = old.gather(1, last.clamp(max=table.shape[1] - 1)[:, None])[part, 0].long(), fresh[part].long()
    # the 128-row blocks of the page that hold rows
    on = (torch.arange(pr // 128, device="cuda") * 128 < (rows % pr)[part][:, None])
    i, blk = on.nonzero(as_tuple=True)
    k_, ks, v, vs = (x.unflatten(2, (-1, 128)) for x in _arrays(s))
    k_[b[i], :, blk], ks[b[i], :, blk], v[b[i], :, blk], vs[b[i], :, blk] = k_[a[i], :, blk], ks[a[i], :, blk], v[a[i], :, blk], vs[a[i], :, blk]


def run(state):
    s, c = state, state["case"]
    if c["kind"] == "tree":
        if not own:
            return _plain_tree(s)
        s["iq"].iq_tree_attention(s["shape"], s["rot"], s["codebook"], s["q"], s["handle"], s["ctx"], s["mask"], s["n_tokens"], s["workspace"],
                                  s["out"], window=c["window"], sinks=c["sinks"], status_dev=s["status"])
        return s["out"]
    if c["kind"] == "keep":
        if own:
            s["iq"].iq_keep_rows(s["shape"], s["handle"], s["ctx"], s["keep"], s["n_keep"], status_dev=s["status"])
        else:
            _plain_keep(s)
        return s["cache"]
    # what the last step left over is given back, and the next one takes its own: the pool is updated in place
    pool = dict(table=s["table"], ref=s["ref"], free=s["free"], n_free=s["n_free"])
    if own:
        s["iq"].iq_release_pages(s["pool"], s["first"], s["end"], status_dev=s["status"])
    else:
        _plain_release(s, s["first"], s["end"])
    if c["kind"] == "fork":
        if own:
            s["iq"].iq_fork_sequences(s["shape"], s["handle"], s["pool"], s["src"], s["dst"], s["rows"], status_dev=s["status"])
        else:
            _plain_fork(s)
        return dict(s["cache"], **pool)
    if own:
        s["iq"].iq_reserve_pages(s["pool"], s["first"], s["rows"], status_dev=s["status"])
    else:
        _plain_reserve(s, s["first"], s["rows"])
    return pool


# ------------------------------------------------------------------------------------------------------------ the work
def work(case):
    c = case
    d, hk, hq, pr = c["head_dim"], c["kv_heads"], c["heads"], c["page_rows"]
    row = c["bits"] * d // 8 + (2 if c["scales"] == "fp16" else 4)  # bytes of a packed row, a side
    if c["kind"] == "tree":
        ctx, tok = _context(c), _tokens(c)
        # rows that some token of the sequence sees (read once), and rows seen by its tokens (a chain's: what a tree's come near to)
        rows = sum(max(_visible(c, x, 0), 0) + t for x, t in zip(ctx, tok))
        seen = sum(t * _visible(c, x, 0) + t * min(t, 4) for x, t in zip(ctx, tok))
        qo = 4 * sum(tok) * hq * d
        return dict(bytes=2 * rows * hk * row + qo + hk * d * 8, flops=4 * d * seen * hq)
    if c["kind"] == "keep":
        return dict(bytes=4 * sum(_accepted(c)) * hk * row, flops=0)
    if c["kind"] == "fork":
        ctx = _context(c)
        pages = sum(-(-x // pr) for x in ctx)
        return dict(bytes=c["tokens"] * (4 * sum(x % pr for x in ctx) * hk * row + 24 * pages), flops=0)
    ctx = _context(c)
    # the entries of the pages that are given back and taken, each in the table, the counts and the list
    moved = sum(-(-(x + c["tokens"]) // pr) - -(-x // pr) for x in ctx)
    return dict(bytes=12 * len(ctx) + 48 * moved + 4, flops=0)


# ------------------------------------------------------------------------------------------------- the definition, fp64
def _exact_code(byte_rows, entry, bits):
    """Codes of the given entries of packed runs (bytes along the last axis), bit by bit as the format has them."""
    code = torch.zeros((*byte_rows.shape[:-1], len(entry)), dtype=torch.int64, device=byte_rows.device)
    for k in range(bits):
        if bits == 4:
            at = 4 * entry + k
        elif bits == 2:
            e = entry % 16
            at = 32 * (entry // 16) + 4 * (e % 8) + 2 * (e // 8) + k
        else:
            e, unit = entry % 32, 96 * (entry // 32)
            at = unit + torch.where(e < 24, 32 * (e // 8) + 4 * (e % 8) + k, 32 * k + 4 * (e - 24) + 3)
        code += ((byte_rows[..., at // 8].long() >> (at % 8)) & 1) << k
    return code


def _exact_rotation(pairs, d):
    """R = blockdiag(v -> q_L v conj(q_R)) H, column by column from the quaternion products."""
    def times(x, y):
        a, b, c, e = x
        f, g, h, i = y
        return (a * f - b * g - c * h - e * i, a * g + b * f + c * i - e * h, a * h - b * i + c * f + e * g, a * i + b * h - c * g + e * f)

    had = torch.ones((1, 1), dtype=torch.float64, device=pairs.device)
    while had.shape[0] < d:
        had = torch.cat((torch.cat((had, had), 1), torch.cat((had, -had), 1)), 0)
    had /= math.sqrt(d)
    p = pairs.double().view(-1, 2, 4)
    p = p / p.norm(dim=-1, keepdim=True)
    ql, qr = [x[:, None] for x in p[:, 0].unbind(-1)], [x[:, None] for x in p[:, 1].unbind(-1)]
    v = had.view(d // 4, 4, d).unbind(1)
    return torch.stack(times(times(ql, v), (qr[0], -qr[1], -qr[2], -qr[3])), 1).reshape(d, d)


def exact(case, seed):
    """The attention by its definition, in 64 bits: the cached rows are taken back to the original space, a sequence and a KV head at a
    time, and each drafted token's softmax runs over the rows that it sees. The other operators move whole values."""
    c = case
    if c["kind"] != "tree":
        return None
    if 4 * c["head_dim"] * sum(_context(c)) * c["tokens"] * c["heads"] > 4e12:
        return None
    s = prepare(c, seed)
    B, T, hq, hk, d, bits = c["batch"], c["tokens"], c["heads"], c["kv_heads"], c["head_dim"], c["bits"]
    dev = s["q"].device
    lv = torch.tensor(_levels(bits, c["grid"])[0], device=dev).double()
    out = torch.zeros((B, T, hq, d), dtype=torch.float64, device=dev)
    ctx, tok, mask = _context(c), _tokens(c), s["mask"].cpu().tolist()
    rots = [_exact_rotation(s["quats"][g], d) for g in range(hk)]
    entry_k, entry_v = torch.arange(d, device=dev), torch.arange(128, device=dev)
    pr = c["page_rows"]
    for b in range(B):
        n = ctx[b] + tok[b]
        anc = [[j for j in range(T) if (mask[b][t][j // 32] >> (j % 32)) & 1] for t in range(T)]
        place = [ctx[b] + len(a) - 1 for a in anc]
        see = torch.zeros((T, n), dtype=torch.bool)
        for t in range(tok[b]):
            lo = place[t] - c["window"] + 1 if c["window"] > 0 else 0
            see[t, max(lo, 0):ctx[b]] = True
            see[t, :min(c["sinks"], ctx[b])] = True
            for j in anc[t]:
                if place[j] >= lo or place[j] < c["sinks"]:
                    see[t, ctx[b] + j] = True
        used = see.any(0).view(-1).to(dev)
        blocks = torch.unique(used.nonzero().view(-1) // 128)
        see = see.to(dev)
        if s["table"] is None:
            at = torch.full_like(blocks, b), blocks * 128
        else:
            at = s["table"][b].long()[blocks * 128 // pr], blocks * 128 % pr
        r = blocks[:, None] * 128 + entry_v
        inside = (r < n).view(-1)
        seen = see[:, r.view(-1)[inside]]
        for g in range(hk):
            rows = at[1][:, None] + entry_v
            kb = s["cache"]["k_codes"][at[0][:, None], g, rows]                       # [blocks][128][P]
            vb = s["cache"]["v_codes"][at[0][:, None], g, rows].reshape(len(blocks), d, 16 * bits)
            ks = s["cache"]["k_scales"][at[0][:, None], g, rows].double()
            vs = s["cache"]["v_scales"][at[0][:, None], g, rows].double()
            k = lv[_exact_code(kb, entry_k, bits)] * ks[..., None] / math.sqrt(d)
            v = lv[_exact_code(vb, entry_v, bits)].transpose(1, 2) * vs[..., None] / math.sqrt(d)
            k, v = (x.reshape(-1, d)[inside] @ rots[g] for x in (k, v))
            G = hq // hk
            q = s["q"][b, :, g * G:(g + 1) * G].double().reshape(T * G, d)
            z = (q @ k.T / math.sqrt(d)).view(T, G, -1)
            z = torch.where(seen[:, None], z, -math.inf)
            top = z.amax(-1, keepdim=True)
            p = torch.exp(z - torch.where(torch.isfinite(top), top, 0.0))
            w = p.sum(-1, keepdim=True)
            o = torch.where(w > 0, (p.view(T * G, -1) @ v).view(T, G, d) / w, 0.0)
            out[b, :tok[b], g * G:(g + 1) * G] = o[:tok[b]]
    return out
