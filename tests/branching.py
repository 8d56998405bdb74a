"""Packed caches made from codes, and the drafted tokens' attention by its definition in 64 bits, for the tests of the branching calls."""
import math

import numpy as np

import oracle


def pack(codes, bits):
    """uint8 codes [..., 32 n] -> bytes of the packed run, entry by entry as docs/FORMAT.md places them."""
    codes = np.asarray(codes, np.uint32)
    lead, n = codes.shape[:-1], codes.shape[-1]
    words = np.zeros(lead + (n * bits // 32,), np.uint32)
    for e in range(n):
        c = codes[..., e]
        if bits == 4:
            words[..., e // 8] |= c << np.uint32(4 * (e % 8))
        elif bits == 2:
            j = e % 16
            words[..., e // 16] |= c << np.uint32(4 * j if j < 8 else 4 * (j - 8) + 2)
        else:
            u, j = 3 * (e // 32), e % 32
            if j < 24:
                words[..., u + j // 8] |= c << np.uint32(4 * (j % 8))
            else:
                for k in range(3):
                    words[..., u + k] |= ((c >> np.uint32(k)) & np.uint32(1)) << np.uint32(4 * (j - 24) + 3)
    return words.view(np.uint8)


def unpack(data, bits):
    """The inverse of pack."""
    words = np.ascontiguousarray(data).view(np.uint32)
    n = words.shape[-1] * 32 // bits
    out = np.zeros(words.shape[:-1] + (n,), np.uint8)
    for e in range(n):
        if bits == 4:
            out[..., e] = (words[..., e // 8] >> np.uint32(4 * (e % 8))) & 15
        elif bits == 2:
            j = e % 16
            out[..., e] = (words[..., e // 16] >> np.uint32(4 * j if j < 8 else 4 * (j - 8) + 2)) & 3
        else:
            u, j = 3 * (e // 32), e % 32
            if j < 24:
                out[..., e] = (words[..., u + j // 8] >> np.uint32(4 * (j % 8))) & 7
            else:
                for k in range(3):
                    out[..., e] |= (((words[..., u + k] >> np.uint32(4 * (j - 24) + 3)) & 1) << k).astype(np.uint8)
    return out


class Rows:
    """Codes and scales of a cache, [n][kv_heads][rows][d] and [n][kv_heads][rows] (n: sequences or pages), and its packed arrays."""

    def __init__(self, rng, n, kv_heads, rows, d, bits, f16=False):
        self.d, self.bits = d, bits
        levels = 1 << bits
        self.codes = [np.clip(np.rint((levels - 1) / 2 + levels / 6 * rng.standard_normal((n, kv_heads, rows, d))), 0, levels - 1).astype(np.uint8)
                      for _ in range(2)]
        sdt = np.float16 if f16 else np.float32
        self.scales = [(math.sqrt(d) * np.exp(0.3 * rng.standard_normal((n, kv_heads, rows)))).astype(sdt) for _ in range(2)]

    def arrays(self):
        n, h, rows, d = self.codes[0].shape
        k = pack(self.codes[0], self.bits)
        v = pack(np.swapaxes(self.codes[1].reshape(n, h, rows // 128, 128, d), 3, 4), self.bits).reshape(k.shape)
        return k, self.scales[0], v, self.scales[1]

    @staticmethod
    def codes_of(k_codes, v_codes, d, bits):
        n, h, rows, _ = k_codes.shape
        v = unpack(np.ascontiguousarray(v_codes).reshape(n, h, rows // 128, d, 16 * bits), bits)
        return unpack(k_codes, bits), np.swapaxes(v, 3, 4).reshape(n, h, rows, d)


def place(table, page_rows, b, t):
    """(sequence or page, row in it) of row t of sequence b."""
    return (b, t) if table is None else (int(table[b, t // page_rows]), t % page_rows)


def random_tree(rng, tokens, reach=5):
    """[tokens][tokens] truth values: the ancestors of each token, itself included."""
    see = np.zeros((tokens, tokens), bool)
    for t in range(tokens):
        parent = int(rng.integers(max(-1, t - reach), t)) if t else -1
        if parent >= 0:
            see[t] = see[parent]
        see[t, t] = True
    return see


def mask_words(see):
    """[..][T][T] truth values -> uint32 words [..][T][ceil(T / 32)] as int32."""
    T = see.shape[-1]
    out = np.zeros(see.shape[:-1] + ((T + 31) // 32,), np.uint32)
    for j in range(T):
        out[..., j // 32] |= see[..., j].astype(np.uint32) << np.uint32(j % 32)
    return out.view(np.int32)


def attention(rows, table, page_rows, quats, levels_k, levels_v, q, ctx, tokens, see, window, sinks, t_cap, sm_scale=0.0):
    """Outputs and lse in 64 bits, and the bound that the tests hold a kernel to. q fp16 [B][T][H][d]; see [B][T][T]; ctx, tokens [B].
    Returns out [B][T][H][d], lse [B][T][H], tol (on the 2-norm of a head's output), tol_lse; tokens from tokens[b] on are NaN.

    The bound: a kernel that keeps 22 bits of q~ and of the probabilities and sums in 32 bits is off in a score by at most
    (d / 16 + 2) cuts of a tensor-core sum, twice (two terms of q~), of 2^-24 of |q| |k| sm_scale each, and as much again for the
    rounding of q~ and the two products with scales; in a weight by that and 64 roundings of 2^-22 (exp2, products, the terms of
    p), in a sum over n rows by n / 128 partial sums of 2^-22. An output is off by at most twice the weights' error times the
    longest value."""
    B, T, H, d = q.shape
    hk = quats.shape[0]
    G = H // hk
    sm = sm_scale if sm_scale > 0 else 1 / math.sqrt(d)
    out, lse = np.full((B, T, H, d), np.nan), np.full((B, T, H), np.nan)
    tol, tol_lse = np.zeros((B, T, H)), np.zeros((B, T, H))
    rot = [oracle.rotation_matrix(d, quats[g]) for g in range(hk)]
    for b in range(B):
        c = min(max(int(ctx[b]), 0), t_cap)
        n = min(max(int(tokens[b]), 0), T)
        total = min(c + n, t_cap)
        sees = see[b][:n, :n]
        pos = c + sees.sum(1) - 1
        vis = np.zeros((n, total), bool)
        for t in range(n):
            lo = pos[t] - window + 1 if window > 0 else 0
            r = np.arange(min(c, total))
            vis[t, :len(r)] = (r >= lo) | (r < sinks)
            for j in range(total - c):
                vis[t, c + j] = sees[t, j] and (pos[j] >= lo or pos[j] < sinks)
        used = np.nonzero(vis.any(0))[0]
        at = [place(table, page_rows, b, int(r)) for r in used]
        pg, rw = np.array([a[0] for a in at], int), np.array([a[1] for a in at], int)
        for g in range(hk):
            k = levels_k[rows.codes[0][pg, g, rw]].astype(np.float64) * (rows.scales[0][pg, g, rw].astype(np.float64) / math.sqrt(d))[:, None]
            v = levels_v[rows.codes[1][pg, g, rw]].astype(np.float64) * (rows.scales[1][pg, g, rw].astype(np.float64) / math.sqrt(d))[:, None]
            for h in range(g * G, (g + 1) * G):
                qr = q[b, :n, h].astype(np.float64) @ rot[g].T
                z = sm * (qr @ k.T)
                for t in range(n):
                    on = vis[t][used]
                    if not on.any():
                        out[b, t, h], lse[b, t, h] = 0.0, -np.inf
                        continue
                    zt = z[t][on]
                    m = zt.max()
                    w = np.exp(zt - m)
                    out[b, t, h] = (w @ v[on]) / w.sum() @ rot[g]
                    lse[b, t, h] = m + math.log(w.sum())
                    dz = 4 * (d / 16 + 2) * 2.0 ** -24 * np.linalg.norm(qr[t]) * np.linalg.norm(k[on], axis=1).max() * sm
                    dw = dz + (on.sum() / 128 + 64) * 2.0 ** -22
                    tol[b, t, h] = 2 * dw * np.linalg.norm(v[on], axis=1).max()
                    tol_lse[b, t, h] = dw + 2.0 ** -22 * abs(lse[b, t, h])
    return out, lse, tol, tol_lse
