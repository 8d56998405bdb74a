"""A step over a batch of requests of any lengths (prompts, pieces of prompts, single tokens) on the packed cache, as cases that can
be timed and compared.

Four kinds of call:

  plan    from the requests' lengths: where each one's new tokens start among the step's tokens, and for every token its position, its
          sequence and the cache row that will hold it (by the block table)
  rotary  rotary positions applied to the queries and keys of the step's tokens: pairs in halves or interleaved, the whole head or
          its first part, frequencies as they are or scaled for longer contexts
  chunk   attention of new tokens over the cache, whose rows the tokens' own follow: a prompt, a piece of one, a step that mixes pieces
          and single tokens; with ``window``: the rows that are further back are left out, but for the first ``sinks``
  cross   attention of a decoder's tokens to an encoder's states of another length, kept as a packed cache: every token sees all rows

Tokens come padded, [batch][tokens], or packed one request after the other, [all tokens]. Head counts, head sizes, contexts and batches
are those of this repository's configurations (query heads / KV heads 4/1, 32/4, 16/8, 32/8, 64/8; head_dim 128 and 256; contexts up to
32 K rows, batches up to 32) and odd sizes between them; page tables and positions go further.

The plain form of an operator is written with elementary torch operations; it takes the same packed cache, whose format it
reads on its own.
"""
import math
import random

import torch

own = False

HEADS = ((4, 1), (32, 4), (16, 8), (32, 8), (64, 8))
MAX_ROWS = 32 * 32768 * 8    # rows x KV heads of the largest cache
MAX_FLOPS = 4.0e12           # of an attention: the largest listed case's
SLAB = 1 << 28               # scores that a plain form holds at a time
NO_POSITION = -(1 << 31)     # position of the places behind the last token
# Max's levels for a unit Gaussian with 4, 8 and 16 cells, upper halves
GAUSS = {2: (0.4528, 1.510), 3: (0.2451, 0.7560, 1.344, 2.152),
         4: (0.1284, 0.3881, 0.6568, 0.9424, 1.256, 1.618, 2.069, 2.733)}


# ---------------------------------------------------------------------------------------------------------------- cases
def _case(kind, **kw):
    case = dict(kind=kind, batch=1, heads=32, kv_heads=8, head_dim=128, ctx=4096, bits=3, grid="int8", scales="fp32", page_rows=0,
                tokens=128, ragged=False, mixed=False, packed=False, window=0, sinks=0, rotary_dim=128, interleaved=False, scaling="none",
                factor=1.0)
    case.update(kw)
    return case


def listed():
    def c(name, kind, **kw):
        return dict(_case(kind, **kw), name=name)

    return [
        # a turn of a chat: 64 new tokens behind 1000 rows, one sequence: latency
        c("chunk_one_64", "chunk", ctx=1000, tokens=64),
        # a prompt from its beginning, into pages
        c("chunk_prompt_2k", "chunk", ctx=0, tokens=2047, page_rows=128, packed=True),
        # the last piece of a long prompt, many heads: the largest products
        c("chunk_long_4k", "chunk", heads=64, ctx=28000, tokens=4096),
        # a server's step: every eighth sequence brings a piece of its prompt, the others one token each
        c("chunk_mixed_batch32", "chunk", batch=32, ctx=16000, tokens=500, page_rows=128, ragged=True, mixed=True, packed=True),
        # wide heads, 4-bit codes of binary16 levels in pages with binary16 scales, a sliding-window layer
        c("chunk_d256_4bit_window", "chunk", batch=2, heads=16, head_dim=256, ctx=12000, bits=4, grid="fp16", scales="fp16", page_rows=256,
          tokens=1000, window=4096, sinks=4, ragged=True),
        # a decoder's first tokens over one encoded input
        c("cross_one", "cross", heads=16, ctx=1500, tokens=5),
        # a batch of decoders' prompts over encoded inputs of different lengths
        c("cross_batch16", "cross", batch=16, heads=16, ctx=1500, tokens=448, ragged=True, packed=True),
        # one token of one sequence, far in its context
        c("rotary_one", "rotary", ctx=100000, tokens=1),
        # a prompt's tokens, frequencies scaled for a context eight times as long as the trained one
        c("rotary_prompt_8k", "rotary", heads=64, ctx=120000, tokens=8192, scaling="parts", factor=8.0),
        # a quarter of wide heads, interleaved pairs
        c("rotary_part_d256", "rotary", batch=7, heads=16, head_dim=256, ctx=5000, tokens=301, rotary_dim=64, interleaved=True, scaling="linear",
          factor=4.0, ragged=True),
        # a small server's step
        c("plan_batch8", "plan", batch=8, ctx=8000, tokens=60, page_rows=128, ragged=True, packed=True),
        # a large one's
        c("plan_batch512", "plan", batch=512, ctx=32000, tokens=400, page_rows=128, ragged=True, mixed=True, packed=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(("chunk", "window", "cross", "rotary", "plan"), (4, 1, 2, 2, 1))[0]
    heads, kv_heads = rng.choice(HEADS)
    head_dim = rng.choice((128, 128, 256))
    bits = rng.choices((3, 2, 4), (3, 1, 1))[0]
    grid = rng.choice(("int8", "int8", "fp16"))
    scales = rng.choice(("fp32", "fp32", "fp16"))
    page_rows = rng.choice((0, 128, 512))
    ragged = rng.random() < 0.7
    packed = rng.random() < 0.5
    mixed = packed and rng.random() < 0.4
    common = dict(heads=heads, kv_heads=kv_heads, head_dim=head_dim, bits=bits, grid=grid, scales=scales, page_rows=page_rows, ragged=ragged,
                  packed=packed, mixed=mixed)
    if kind == "rotary":
        rotary_dim = rng.choice((head_dim, head_dim, head_dim // 2, head_dim // 4, 96, 16))
        scaling = rng.choice(("none", "linear", "base", "parts"))
        tokens = _log_int(rng, 1, 8192)
        return _case("rotary", heads=heads, kv_heads=kv_heads, head_dim=head_dim, ragged=ragged, batch=_log_int(rng, 1, max(1, min(32, 8192 // tokens))),
                     ctx=_log_int(rng, 1, 1000000), tokens=tokens, rotary_dim=rotary_dim, interleaved=rng.random() < 0.5, scaling=scaling,
                     factor=1.0 if scaling == "none" else rng.choice((1.5, 2.0, 8.0, 32.0)))
    if kind == "plan":
        return _case("plan", batch=_log_int(rng, 1, 512), ctx=_log_int(rng, 1, 32000), tokens=_log_int(rng, 1, 400), page_rows=rng.choice((0, 128, 512)),
                     ragged=ragged, mixed=mixed, packed=True)
    ctx = _log_int(rng, 1, 1500 if kind == "cross" else 32000)
    if kind == "chunk" and rng.random() < 0.15:
        ctx = 0
    c = _case("cross" if kind == "cross" else "chunk", ctx=ctx, tokens=_log_int(rng, 1, 4096), **common)
    if kind == "window":
        c.update(window=_log_int(rng, 1, 8192), sinks=rng.choice((0, 1, 4, 64, 200)))
    rows = MAX_ROWS * 128 // head_dim // kv_heads
    c["batch"] = _log_int(rng, 1, max(1, min(32, rows // (c["ctx"] + c["tokens"]))))
    while work(c)["flops"] > MAX_FLOPS:
        c["tokens"] = max(1, c["tokens"] // 2)
        c["batch"] = max(1, c["batch"] * 2 // 3)
    return c


def _context(c):
    """Rows of every sequence before the step: the same for every seed, so that the work is the case's."""
    return [max(min(1, c["ctx"]), int(c["ctx"] * (0.5 + 0.5 * ((i * 0.6180339887 + 0.37) % 1.0)))) if c["ragged"] else c["ctx"] for i in range(c["batch"])]


def _tokens(c):
    """New tokens of every sequence, at most c["tokens"]."""
    n = c["tokens"]
    if c["mixed"]:
        return [n - (i * 5) % 3 * (n // 4) if i % 8 == 0 else 1 for i in range(c["batch"])]
    return [max(1, n - (i * 5) % 3 * (n // 4)) if c["ragged"] else n for i in range(c["batch"])]


def _starts(c):
    at = [0]
    for n in _tokens(c):
        at.append(at[-1] + n)
    return at


def _room(c):
    """Places for the tokens of a packed step: a multiple of 64, as a server allocates them."""
    return -(-_starts(c)[-1] // 64) * 64


def _end(c):
    """Rows of every sequence that its last token sees."""
    return [x + (n if c["kind"] != "cross" else 0) for x, n in zip(_context(c), _tokens(c))]


def _cap(c):
    unit = max(128, c["page_rows"])
    return -(-(c["ctx"] + (c["tokens"] if c["kind"] != "cross" else 0)) // unit) * unit


def _inv_freq(c):
    """Radians per position of each pair, and the factor of the results, by the formulas."""
    r, base, s = c["rotary_dim"], 10000.0, c["factor"]
    if c["scaling"] == "base":
        base *= s ** (r / (r - 2))
    f = [base ** (-2.0 * i / r) for i in range(r // 2)]
    if c["scaling"] == "linear":
        f = [x / s for x in f]
    if c["scaling"] == "parts":
        def turns(beta):  # the pair that turns beta times over the trained context
            return r * math.log(4096 / (2 * math.pi * beta)) / (2 * math.log(base))

        low, high = max(math.floor(turns(32.0)), 0), min(math.ceil(turns(1.0)), r - 1)
        ramp = [min(1.0, max(0.0, (i - low) / max(high - low, 0.001))) for i in range(r // 2)]
        return [x / s * k + x * (1 - k) for x, k in zip(f, ramp)], 0.1 * math.log(s) + 1
    return f, 1.0


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


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed * 7919 + 13)
    rng = random.Random(seed)
    s = dict(case=c)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    B, T, hq, hk, d, pr = c["batch"], c["tokens"], c["heads"], c["kv_heads"], c["head_dim"], c["page_rows"]
    if c["kind"] == "rotary":
        # positions a little different for every seed, all tokens of a sequence one after the other; the queries and keys lie in the
        # output of one projection, beside the values
        first = [x - rng.randrange(0, min(x, 50) + 1) for x in _context(c)]
        s["positions"] = torch.cat([torch.arange(x, x + n, dtype=torch.int32, device=dev) for x, n in zip(first, _tokens(c))])
        n = len(s["positions"])
        qkv = torch.randn((n, hq + 2 * hk, d), generator=gen, device=dev).half()
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hk]
        s["inv_freq"] = torch.tensor(_inv_freq(c)[0], dtype=torch.float64, device=dev)
    else:
        cap = _cap(c)
        ctx, tok, end = _context(c), _tokens(c), _end(c)
        s["ctx"], s["n_tokens"] = ints(ctx), ints(tok)
        if c["kind"] == "plan":  # lengths a little different for every seed, within the rows that the pages below hold
            s["ctx"] = ints([x - rng.randrange(0, min(x, 50) + 1) for x in ctx])
            s["n_tokens"] = ints([n - rng.randrange(0, min(n, 9)) for n in tok])
        if pr:
            # the pages that a sequence holds, in any order of the pool; those between the sinks and the windows have been given back (-1)
            held = []
            for b in range(B):
                first = max(0, ctx[b] - c["window"]) // pr if c["window"] > 0 else 0
                held.append([j for j in range(cap // pr) if (j * pr < c["sinks"] or j >= first) and j * pr < end[b]])
            n = max(1, sum(map(len, held)))
            pages = list(range(n))
            rng.shuffle(pages)
            table = [[-1] * (cap // pr) for _ in range(B)]
            at = 0
            for b in range(B):
                for j in held[b]:
                    table[b][j] = pages[at]
                    at += 1
            s["table"], rows_shape = ints(table), (n, hk, pr)
        else:
            s["table"], rows_shape = None, (B, hk, cap)
        s["n_pages"] = rows_shape[0]
        if c["packed"]:
            s["start"] = ints(_starts(c))
        if c["kind"] != "plan":
            s["cache"] = _cache(c, gen, rows_shape)
            q = torch.randn((hk, d // 4, 2, 4), generator=gen, device=dev, dtype=torch.float64)
            s["quats"] = (q / q.norm(dim=-1, keepdim=True)).float().reshape(hk, d // 4, 8).contiguous()
            s["q"] = (2 * torch.randn((_room(c), hq, d) if c["packed"] else (B, T, hq, d), generator=gen, device=dev)).half()
    if own:  # the descriptors, outputs and the workspace that a program keeps beside its cache
        import paper_2608_08081_b200 as iq

        s["iq"] = iq
        s["status"] = torch.zeros(4, dtype=torch.int32, device=dev)
        if c["kind"] == "rotary":
            s["shape"] = iq.Shape(B, hq, hk, d, 128)
            s["rotary"] = iq.iq_make_rotary(c["rotary_dim"], interleaved=c["interleaved"], scaling=c["scaling"], factor=c["factor"], original_len=4096)
            s["q_out"] = torch.empty((n, hq, d), dtype=torch.float16, device=dev)
            s["k_out"] = torch.empty((n, hk, d), dtype=torch.float16, device=dev)
            return s
        s["shape"] = iq.Shape(B, hq, hk, d, cap, c["bits"])
        if c["kind"] == "plan":
            room = _room(c)
            s["starts_out"] = torch.empty(B + 1, dtype=torch.int32, device=dev)
            s["positions_out"], s["sequences_out"] = (torch.empty(room, dtype=torch.int32, device=dev) for _ in range(2))
            s["slots_out"] = torch.empty(room, dtype=torch.int64, device=dev)
            return s
        k = s["cache"]
        s["handle"] = iq.Cache(k["k_codes"], k["k_scales"], k["v_codes"], k["v_scales"], s["table"], pr)
        s["rot"] = s["quats"]  # (unit quaternion pairs: the rotation as the library keeps it)
        lv, th = _levels(c["bits"], c["grid"])
        s["codebook"] = iq.Codebook(tuple(lv), tuple(th))
        s["workspace"] = torch.empty(iq.iq_chunk_workspace_bytes(s["shape"]), dtype=torch.uint8, device=dev)
        s["out"] = torch.zeros_like(s["q"])
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


def _plain_attention(s):
    """A sequence at a time, as many tokens at a time as the scores have room for (most cases: all of them)."""
    c = s["case"]
    hq, hk, d, bits = c["heads"], c["kv_heads"], c["head_dim"], c["bits"]
    G = hq // hk
    lv = torch.tensor(_levels(bits, c["grid"])[0], device="cuda")
    rot = _rotation(s["quats"])
    out = torch.zeros_like(s["q"])
    cache = s["cache"]
    kw = cache["k_codes"].view(torch.int32).unflatten(2, (-1, 128))
    vw = cache["v_codes"].view(torch.int32).unflatten(2, (-1, 128)).flatten(3).unflatten(3, (d, 4 * bits))
    causal = c["kind"] == "chunk"
    for b, (x, n, end, at) in enumerate(zip(_context(c), _tokens(c), _end(c), _starts(c))):
        # the blocks of 128 rows that the sequence's tokens see: the sinks', and those from the first window on
        first = max(0, x - c["window"] + 1) // 128 if c["window"] > 0 else 0
        no = torch.arange(first, -(-end // 128), device="cuda")
        no = torch.cat((torch.arange(min(first, -(-c["sinks"] // 128)), device="cuda"), no))
        if s["table"] is None:
            page, blk = torch.full_like(no, b), no
        else:
            per = c["page_rows"] // 128
            page, blk = s["table"][b].long()[no // per], no % per
        k = lv[_unpack(kw[page, :, blk], bits)].transpose(0, 1).flatten(1, 2)                      # [hk][rows][d]
        v = lv[_unpack(vw[page, :, blk], bits)].permute(1, 0, 3, 2).flatten(1, 2)
        ks, vs = (cache[name].unflatten(2, (-1, 128))[page, :, blk].float().transpose(0, 1).flatten(1)[:, None] / math.sqrt(d)
                  for name in ("k_scales", "v_scales"))                                           # [hk][1][rows]
        row = (no[:, None] * 128 + torch.arange(128, device="cuda")).flatten()
        tokens, mine = (s["q"][at:at + n], out[at:at + n]) if c["packed"] else (s["q"][b, :n], out[b, :n])
        slab = max(1, SLAB // max(1, hq * len(row)))
        for t in range(0, n, slab):
            q = tokens[t:t + slab].float().unflatten(1, (hk, G)).permute(1, 0, 2, 3).flatten(1, 2) @ rot.transpose(1, 2)  # [hk][tokens G][d]
            pos = x + torch.arange(t, min(n, t + slab), device="cuda")[:, None]
            see = (row <= pos) & (row < end) if causal else (row < end).expand(len(pos), -1)
            if c["window"] > 0:
                see = see & ((row > pos - c["window"]) | (row < c["sinks"]))
            z = torch.where(see.repeat_interleave(G, 0), (q @ k.transpose(1, 2)) * ks / math.sqrt(d), -math.inf)
            m = z.amax(-1, keepdim=True) if len(row) else z.new_full((hk, z.shape[1], 1), -math.inf)
            p = torch.exp(z - torch.where(m > -math.inf, m, 0.0))
            w = p.sum(-1, keepdim=True)
            o = torch.where(w > 0, (p * vs) @ v / w, 0.0) @ rot
            mine[t:t + slab] = o.unflatten(1, (-1, G)).permute(1, 0, 2, 3).flatten(1, 2).half()
    return out


def _plain_rotary(s):
    c = s["case"]
    r, factor = c["rotary_dim"], _inv_freq(c)[1]
    angle = s["positions"].double()[:, None] * s["inv_freq"]
    cos, sin = ((f(angle) * factor).float()[:, None] for f in (torch.cos, torch.sin))             # [tokens][1][pairs]

    def turned(x):
        x = x.float()
        a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
        y = (a * cos - b * sin, a * sin + b * cos)
        y = torch.stack(y, -1).flatten(-2) if c["interleaved"] else torch.cat(y, -1)
        return torch.cat((y, x[..., r:]), -1).half()

    return turned(s["q"]), turned(s["k"])


def _plain_plan(s):
    c, ctx = s["case"], s["ctx"]
    n = s["n_tokens"].clamp(min=0)
    start = torch.cat((n.new_zeros(1), n.cumsum(0, dtype=torch.int32)))
    t = torch.arange(_room(c), dtype=torch.int32, device="cuda")
    b = torch.searchsorted(start[1:], t, right=True).clamp(max=c["batch"] - 1)
    on = t < start[-1]
    pos = ctx[b] + t - start[b]
    cap, pr = _cap(c), c["page_rows"]
    at = pos.clamp(max=cap - 1).long()
    if s["table"] is None:
        slot = b * cap + at
        good = on & (pos < cap)
    else:
        page = s["table"][b, at // pr].long()
        slot = page * pr + at % pr
        good = on & (pos < cap) & (page >= 0) & (page < s["n_pages"])
    return dict(starts=start, positions=torch.where(on, pos, NO_POSITION), sequences=torch.where(on, b.int(), -1), slots=torch.where(good, slot, -1))


def run(state):
    s, c = state, state["case"]
    if not own:
        return _plain_rotary(s) if c["kind"] == "rotary" else _plain_plan(s) if c["kind"] == "plan" else _plain_attention(s)
    iq = s["iq"]
    if c["kind"] == "rotary":
        iq.iq_apply_rotary(s["shape"], s["rotary"], s["q"], s["k"], s["positions"], s["q_out"], s["k_out"])
        return s["q_out"], s["k_out"]
    if c["kind"] == "plan":
        iq.iq_plan_tokens(s["shape"], s["ctx"], s["n_tokens"], s["starts_out"], s["positions_out"], s["sequences_out"], s["slots_out"],
                          block_table=s["table"], page_rows=c["page_rows"], num_pages=s["n_pages"], status_dev=s["status"])
        return dict(starts=s["starts_out"], positions=s["positions_out"], sequences=s["sequences_out"], slots=s["slots_out"])
    layout = dict(token_start=s["start"]) if c["packed"] else dict(n_tokens=s["n_tokens"])
    if c["kind"] == "cross":
        iq.iq_cross_attention(s["shape"], s["rot"], s["codebook"], s["q"], s["handle"], s["ctx"], s["workspace"], s["out"], status_dev=s["status"], **layout)
    else:
        iq.iq_chunk_attention(s["shape"], s["rot"], s["codebook"], s["q"], s["handle"], s["ctx"], s["workspace"], s["out"], window=c["window"],
                              sinks=c["sinks"], status_dev=s["status"], **layout)
    return s["out"]


# ------------------------------------------------------------------------------------------------------------ the work
def _seen(c, x, n):
    """Rows seen by all tokens of a sequence with x rows before its n tokens, and rows seen by some token."""
    if c["kind"] == "cross":
        return n * x, x
    if c["window"] <= 0:
        return n * x + n * (n + 1) // 2, x + n
    total = 0
    for p in range(x, x + n):
        first = max(0, p - c["window"] + 1)
        total += p + 1 - first + min(c["sinks"], first)
    first = max(0, x - c["window"] + 1)
    return total, x + n - first + min(c["sinks"], first)


def work(case):
    c = case
    d, hk, hq = c["head_dim"], c["kv_heads"], c["heads"]
    tok = _tokens(c)
    if c["kind"] == "rotary":
        return dict(bytes=sum(tok) * (4 * (hq + hk) * d + 4), flops=3 * sum(tok) * (hq + hk) * c["rotary_dim"])
    if c["kind"] == "plan":
        pages = sum(-(-(x + n) // c["page_rows"]) - x // c["page_rows"] for x, n in zip(_context(c), tok)) if c["page_rows"] else 0
        return dict(bytes=16 * _room(c) + 12 * c["batch"] + 4 * pages, flops=0)
    row = c["bits"] * d // 8 + (2 if c["scales"] == "fp16" else 4)  # bytes of a packed row, a side
    seen = [_seen(c, x, n) for x, n in zip(_context(c), tok)]
    return dict(bytes=2 * sum(r for _, r in seen) * hk * row + 4 * sum(tok) * hq * d + hk * d * 8, flops=4 * d * hq * sum(p for p, _ in seen))


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


def _exact_rotary(c, s):
    """Every pair as a complex number, turned by its angle."""
    pairs, factor = _inv_freq(c)
    w = torch.polar(torch.full((1, 1), factor, dtype=torch.float64, device="cuda"),
                    s["positions"].double()[:, None] * torch.tensor(pairs, dtype=torch.float64, device="cuda"))[:, None]
    r, res = c["rotary_dim"], []
    for x in (s["q"], s["k"]):
        y = x.double().clone()
        i = torch.arange(r // 2, device="cuda")
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + r // 2)
        u = torch.complex(y[..., a], y[..., b]) * w
        y[..., a], y[..., b] = u.real, u.imag
        res.append(y)
    return tuple(res)


def exact(case, seed):
    """The attention by its definition, in 64 bits: the cached rows are taken back to the original space, a sequence and a KV head at a
    time, and each token's softmax runs over the rows that it sees. A plan is whole numbers."""
    c = case
    if c["kind"] == "plan":
        return None
    s = prepare(c, seed)
    if c["kind"] == "rotary":
        return _exact_rotary(c, s)
    hq, hk, d, bits, pr = c["heads"], c["kv_heads"], c["head_dim"], c["bits"], c["page_rows"]
    G, dev = hq // hk, s["q"].device
    lv = torch.tensor(_levels(bits, c["grid"])[0], device=dev).double()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    rots = [_exact_rotation(s["quats"][g], d) for g in range(hk)]
    entry_k, entry_v = torch.arange(d, device=dev), torch.arange(128, device=dev)
    at = 0
    for b, (x, n) in enumerate(zip(_context(c), _tokens(c))):
        rows = x if c["kind"] == "cross" else x + n
        q, mine = (s["q"][at:at + n], out[at:at + n]) if c["packed"] else (s["q"][b, :n], out[b, :n])
        at += n
        r = torch.arange(rows, device=dev)
        lo = x - c["window"] + 1 if c["window"] > 0 else 0
        r = r[(r >= lo) | (r < c["sinks"])]  # (what a later token does not see is left out below)
        if rows == 0:
            continue
        blocks = torch.unique(r // 128)
        where = (torch.full_like(blocks, b), blocks * 128) if s["table"] is None else (s["table"][b].long()[blocks * 128 // pr], blocks * 128 % pr)
        number = (blocks[:, None] * 128 + entry_v).view(-1)
        inside = torch.isin(number, r)
        number = number[inside]
        for g in range(hk):
            i = where[1][:, None] + entry_v
            kb = s["cache"]["k_codes"][where[0][:, None], g, i]                                    # [blocks][128][P]
            vb = s["cache"]["v_codes"][where[0][:, None], g, i].reshape(len(blocks), d, 16 * bits)
            ks = s["cache"]["k_scales"][where[0][:, None], g, i].double()
            vs = s["cache"]["v_scales"][where[0][:, None], g, i].double()
            k = lv[_exact_code(kb, entry_k, bits)] * ks[..., None] / math.sqrt(d)
            v = lv[_exact_code(vb, entry_v, bits)].transpose(1, 2) * vs[..., None] / math.sqrt(d)
            k, v = (y.reshape(-1, d)[inside] @ rots[g] for y in (k, v))
            step = max(1, (1 << 26) // (G * len(number)))
            for t in range(0, n, step):
                m = min(step, n - t)
                z = (q[t:t + m, g * G:(g + 1) * G].double().reshape(m * G, d) @ k.T / math.sqrt(d)).view(m, G, -1)
                if c["kind"] == "chunk":
                    p = x + torch.arange(t, t + m, device=dev)[:, None]
                    see = number <= p
                    if c["window"] > 0:
                        see &= (number > p - c["window"]) | (number < c["sinks"])
                    z = torch.where(see[:, None], z, -math.inf)
                mine[t:t + m, g * G:(g + 1) * G] = (torch.softmax(z, -1).view(m * G, -1) @ v).view(m, G, d)
    return out
