"""Oracle: the long-context cache operators (float64 and whole numbers).

Test infrastructure only (see the package docstring). The paper's decode
attention reads the whole growing cache (section 1); these operators rotate
what enters the cache and restrict what is read of it, which the paper does not
define. Definitions (readings of this library):

rotation of channels (a, b) at position p, c and s from the caller's table:
    a' = a c - b s,  b' = b c + a s
    pairs (i, i + R/2), or (2i, 2i + 1) when interleaved; channels >= R copied.

summary of a full block's keys k [16, D] (one kv head), all finite:
    e   = least whole number >= -100 with |k| < 2^e everywhere
    S_d = sum_t rne(k_td 2^(14 - e)),  r = max(0, bits(max |S|) - 7)
    code_d = clamp(rne(S_d 2^-r), -127, 127),  exponent e - 18 + r
    (a non-finite key: codes 0, exponent 127)

choice of N = min(top, n) of a sequence's n blocks for kv head g: the first
`sink`, the last `recent`, and the others of the highest
    score_j = fp32( max_h 2^(e_h - 7 + exponent_j) <c_h, code_j> )
with the query codes c_h, e_h made like a summary's (non-finite channels 0);
+inf for exponent 127, last for a bad block id, the lower index first among
equals; ascending, -1 behind them.

sparse attention: softmax over the tokens of the listed blocks; an entry that
does not exceed the one before it, or is no block of the sequence, or has a
bad pool id, contributes nothing; no token at all gives 0.
"""
from __future__ import annotations

import math

import torch

LEAST_EXP, ALWAYS = -100, 127


def rotate(x, angles, interleaved: bool):
    """x [T, H, D] in float64, turned by angles [T, R] (cosines, then sines)."""
    x, angles = x.to(torch.float64).clone(), angles.to(torch.float64)
    R = angles.shape[-1]
    i = torch.arange(R // 2)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    c, s = angles[:, None, :R // 2], angles[:, None, R // 2:]
    a, b = x[..., ia], x[..., ib]
    x[..., ia], x[..., ib] = a * c - b * s, b * c + a * s
    return x


def exponent_above(x):
    """Least e >= LEAST_EXP with |x| < 2^e for the finite elements of x."""
    x = x.to(torch.float64)
    big = float(torch.where(torch.isfinite(x), x, 0.0).abs().max())
    return max(math.frexp(big)[1], LEAST_EXP) if big > 0 else LEAST_EXP


def summarise(k):
    """Codes int8 [D] and exponent of one block's keys k [16, D]."""
    k = k.to(torch.float64)
    if not bool(torch.isfinite(k).all()):
        return torch.zeros(k.shape[1], dtype=torch.int8), ALWAYS
    e = exponent_above(k)
    total = torch.round(k * 2.0 ** (14 - e)).sum(0)
    r = max(0, int(total.abs().max()).bit_length() - 7)
    return torch.round(total / 2.0 ** r).clamp(-127, 127).to(torch.int8), e - 18 + r


def block_summary(k_cache, block_table, context_lens, keys, exp):
    """keys and exp with every full block's summary in place (new tensors)."""
    keys, exp = keys.clone(), exp.clone()
    N, Hkv = k_cache.shape[:2]
    for b in range(block_table.shape[0]):
        for j in range(int(context_lens[b]) // 16):
            blk = int(block_table[b, j])
            if 0 <= blk < N:
                for g in range(Hkv):
                    keys[blk, g], exp[blk, g] = summarise(k_cache[blk, g])
    return keys, exp


def select(q, keys, exp, block_table, context_lens, top: int, sink: int, recent: int):
    """int32 [B, Hkv, top]: the chosen blocks of each (sequence, kv head)."""
    B, Hq, D = q.shape
    N, Hkv = keys.shape[:2]
    G = Hq // Hkv
    out = torch.full((B, Hkv, top), -1, dtype=torch.int32)
    x = q.to(torch.float64)
    x = torch.where(torch.isfinite(x), x, 0.0)
    for b in range(B):
        n = -(-max(int(context_lens[b]), 0) // 16)
        ids = block_table[b, :n].long()
        good = (ids >= 0) & (ids < N)
        ids = torch.where(good, ids, 0)
        for g in range(Hkv):
            score = torch.full((n,), -math.inf, dtype=torch.float64)
            ex = exp[ids, g].to(torch.float64)
            for h in range(g * G, (g + 1) * G):
                e = exponent_above(x[b, h])
                c = torch.round(x[b, h] * 2.0 ** (7 - e)).clamp(-127, 127)
                score = torch.maximum(score, (keys[ids, g].to(torch.float64) @ c) * 2.0 ** (ex + (e - 7)))
            score = score.to(torch.float32)
            score[ex == ALWAYS] = math.inf
            rank = [(2 if j < sink or j >= n - recent else 1 if good[j] else 0, float(score[j]), -j) for j in range(n)]
            took = sorted(sorted(range(n), key=lambda j: rank[j], reverse=True)[:min(top, n)])
            out[b, g, :len(took)] = torch.tensor(took, dtype=torch.int32)
    return out


def attention_sparse(q, k_cache, v_cache, block_table, context_lens, selected, scale=None):
    """(out [B, Hq, D], sum_j p_j |v_j| [B, Hq, D]) in float64; the second bounds rounding errors."""
    B, Hq, D = q.shape
    N, Hkv = k_cache.shape[:2]
    G = Hq // Hkv
    scale = scale or 1.0 / math.sqrt(D)
    out = torch.zeros(B, Hq, D, dtype=torch.float64)
    mag = torch.zeros_like(out)
    for b in range(B):
        ctx = int(context_lens[b])
        n = -(-ctx // 16)
        for g in range(Hkv):
            ks, vs, prev = [], [], -1
            for j in selected[b, g, :min(n, selected.shape[2])].tolist():
                ok, prev = prev < j < n and j >= 0, j
                blk = int(block_table[b, j]) if ok else -1
                if 0 <= blk < N:
                    m = min(16, ctx - 16 * j)
                    ks.append(k_cache[blk, g, :m])
                    vs.append(v_cache[blk, g, :, :m].t())
            if not ks:
                continue
            k, v = torch.cat(ks).to(torch.float64), torch.cat(vs).to(torch.float64)
            p = torch.softmax(q[b, g * G:(g + 1) * G].to(torch.float64) @ k.t() * scale, -1)
            out[b, g * G:(g + 1) * G] = p @ v
            mag[b, g * G:(g + 1) * G] = p @ v.abs()
    return out, mag
