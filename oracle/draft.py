"""Oracle: the 8-bit cache and drafted tokens (float64).

Test infrastructure only (see the package docstring). The paper's decode
attention reads the whole cache for one new token per sequence (section 1);
these operators hold the cache in 8 bits and attend several new tokens at once,
which the paper does not define. Definitions (readings of this library):

a row x [D] in 8 bits: e = least whole number >= -100 with |x_d| <= 448 2^e for
all finite x_d; c_d = x_d 2^-e rounded to e4m3 (to nearest, ties to even), NaN
for a non-finite x_d. It stands for c 2^e. e4m3: 3 mantissa bits, exponents down
to 2^-6, below that steps of 2^-9.

drafts: the newest n_b tokens of a context are the sequence's rows; row i sees the
places before them and, of them, place s_b + j where bit j of its mask is set
(no masks: j <= i). Nothing to see gives 0.

accepted drafts: the leading entries that ascend strictly within [0, n_b), at
most the count, move to places s_b, s_b + 1, ...
"""
from __future__ import annotations

import math

import torch

LEAST_ROW_EXP = -100


def round_e4m3(y):
    """float64 values of magnitude up to 448, rounded to e4m3."""
    y = y.to(torch.float64)
    power = torch.frexp(y.abs()).exponent.clamp(min=-5)  # |y| < 2^power
    step = torch.ldexp(torch.ones_like(y), power - 4)
    return torch.round(y / step) * step


def encode(x):
    """(codes' values, exponents) of rows x [.., D]."""
    x = x.to(torch.float64)
    fine = torch.isfinite(x)
    m = torch.where(fine, x, 0.0).abs().amax(-1)
    e = torch.full(m.shape, LEAST_ROW_EXP, dtype=torch.int64)
    for _ in range(256):
        e = torch.where(m > torch.ldexp(torch.full_like(m, 448.0), e), e + 1, e)
    c = round_e4m3(torch.ldexp(torch.where(fine, x, 0.0), -e[..., None]))
    return torch.where(fine, c, math.nan), e


def held(pool, exp):
    """What an 8-bit pool's rows stand for: pool [.., D] or any codes, exp broadcast to them."""
    return torch.ldexp(pool.to(torch.float64), exp.to(torch.int64))


def held_pools(k_cache, v_cache, kv_exp):
    """(K [N, Hkv, 16, D], V [N, Hkv, D, 16]) in float64; kv_exp None: bf16 pools."""
    if kv_exp is None:
        return k_cache.to(torch.float64), v_cache.to(torch.float64)
    return held(k_cache, kv_exp[:, :, 0, :, None]), held(v_cache, kv_exp[:, :, 1, None, :])


def write(k_cache, v_cache, kv_exp, block_table, context_lens, cu, k, v):
    """Pools (codes' values, exponents) after rows k, v [T, Hkv, D] were written as the newest tokens."""
    kc, vc, ex = k_cache.to(torch.float64), v_cache.to(torch.float64), kv_exp.clone()
    cap = block_table.shape[1] * 16
    (kq, ke), (vq, ve) = encode(k), encode(v)
    for b in range(len(context_lens)):
        ctx = int(context_lens[b])
        if not 1 <= ctx <= cap:
            continue
        for r in range(cu[b], cu[b + 1]):
            pos = ctx - cu[b + 1] + r
            blk = int(block_table[b, pos // 16]) if pos >= 0 else -1
            if not 0 <= blk < kc.shape[0]:
                continue
            kc[blk, :, pos % 16], vc[blk, :, :, pos % 16] = kq[r], vq[r]
            ex[blk, :, 0, pos % 16], ex[blk, :, 1, pos % 16] = ke[r].to(torch.int8), ve[r].to(torch.int8)
    return kc, vc, ex


def attention_tree(q, k_cache, v_cache, kv_exp, block_table, context_lens, cu, masks=None, scale=None):
    """out [T, Hq, D] and what bounds its rounding errors, in float64: sum_j p_j |v_j| [T, Hq, D]; the largest
    sum_d |q_d k_jd| scale over the seen j [T, Hq]; for an 8-bit cache max_j (p_j 2^e_j) sum_j |c_j| [T, Hq, D], e_j
    and c_j the exponent and codes of v_j (else zeros)."""
    T, Hq, D = q.shape
    N, Hkv = k_cache.shape[:2]
    G = Hq // Hkv
    scale = scale or 1.0 / math.sqrt(D)
    kp, vp = held_pools(k_cache, v_cache, kv_exp)
    out, mag = torch.zeros(T, Hq, D, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64)
    size, small = torch.zeros(T, Hq, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64)
    for b in range(len(context_lens)):
        ctx, n = max(int(context_lens[b]), 0), cu[b + 1] - cu[b]
        start = ctx - n
        pos = torch.arange(ctx)
        blk = block_table[b, :-(-ctx // 16)].long().repeat_interleave(16)[:ctx]
        good = (blk >= 0) & (blk < N)
        for i in range(n):
            mask = (2 << i) - 1 if masks is None else int(masks[cu[b] + i])
            bits = torch.tensor([mask >> j & 1 == 1 for j in range(n)], dtype=torch.bool)
            see = good & ((pos < start) | bits[(pos - start).clamp(min=0)]) if n and ctx else good
            at = see.nonzero()[:, 0]
            if len(at) == 0:
                continue
            for g in range(Hkv):
                k, v = kp[blk[at], g, at % 16], vp[blk[at], g, :, at % 16]
                h = slice(g * G, (g + 1) * G)
                x = q[cu[b] + i, h].to(torch.float64)
                p = torch.softmax(x @ k.t() * scale, -1)
                out[cu[b] + i, h], mag[cu[b] + i, h] = p @ v, p @ v.abs()
                size[cu[b] + i, h] = (x.abs() @ k.abs().t()).amax(-1) * scale
                if kv_exp is not None:
                    e = kv_exp[blk[at], g, 1, at % 16].to(torch.int64)
                    codes = v_cache[blk[at], g, :, at % 16].to(torch.float64).abs().sum(0)
                    small[cu[b] + i, h] = torch.ldexp(p, e).amax(-1, keepdim=True) * codes
    return out, mag, size, small


def accept(k_cache, v_cache, kv_exp, block_table, context_lens, cu, accepted, counts):
    """(pools after the move, new context lengths); pools as given, copied."""
    kc, vc = k_cache.clone(), v_cache.clone()
    ex = None if kv_exp is None else kv_exp.clone()
    N, cap = kc.shape[0], block_table.shape[1] * 16
    new = context_lens.clone()
    for b in range(len(context_lens)):
        ctx, n = int(context_lens[b]), int(cu[b + 1] - cu[b])
        if not 1 <= ctx <= cap or not 0 <= n <= ctx:
            continue
        start, took = ctx - n, []
        for a in accepted[b, :max(int(counts[b]), 0)].tolist():
            if not (took[-1] if took else -1) < a < n:
                break
            took.append(a)
        new[b] = start + len(took)
        for i, a in enumerate(took):
            s, d = int(block_table[b, (start + a) // 16]), int(block_table[b, (start + i) // 16])
            if not (0 <= s < N and 0 <= d < N):
                continue
            o0, o1 = (start + a) % 16, (start + i) % 16
            kc[d, :, o1], vc[d, :, :, o1] = k_cache[s, :, o0], v_cache[s, :, :, o0]
            if ex is not None:
                ex[d, :, :, o1] = kv_exp[s, :, :, o0]
    return kc, vc, ex, new
