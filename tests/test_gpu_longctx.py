"""HIP long-context operators (rotation and cache write, block summaries, choice
of blocks, attention over chosen blocks) against the oracle.

Tolerances. Rotation: a c - b s in fp32, three roundings of at most 2^-24 of
|a c| + |b s| <= |a| + |b| each, then bf16, half a step 2^-8 of the result:
|y - r| <= 2^-8 |r| (1 + 2^-7) + 2^-22 (|a| + |b|). Attention: out is rounded to
bf16 (2^-8 |out|); softmax weights are rounded to bf16 before the products and
summed as rounded, so the quotient is off by at most 2 * 2^-8 sum p|v|; scores
carry fp32 sums of at most 128 products, of which exp2 makes less than 2^-10 of
the weights at these magnitudes (|score| < 64: 64 * 128 * 2^-24 = 2^-11 before
the exponential). Copies, summaries and choices are compared for equality.
"""
import threading

import numpy as np
import pytest
import torch

from oracle import longctx as lc
from paper_2608_01891_amd import aflex, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CACHE = ("k_cache", "v_cache")


def _bf(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).bfloat16()


def _tokens(seed, T, heads, strided):
    Hq, Hkv, D = heads
    x = _bf(seed, T, Hq + 2 * Hkv, D)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if strided:
        y = x.to(DEV)
        return (q, k, v), (y[:, :Hq], y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:])
    return (q, k, v), tuple(t.contiguous().to(DEV) for t in (q, k, v))


def _check_rotation(got, x, angles, inter, what):
    ref = lc.rotate(x, angles, inter)
    most = 2 * x.double().abs().amax(-1, keepdim=True)  # no less than |a| + |b|
    bound = ref.abs() * 2.0 ** -8 * (1 + 2.0 ** -7) + 2.0 ** -22 * most
    bad = (got.double() - ref).abs() > bound
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} values"
    R = angles.shape[1]
    assert torch.equal(got[..., R:], x[..., R:]), f"{what}: channels that are not rotated"


def _expect_write(a, k, v, cu, kq):
    """Pools after the write of k, v (rows cu) with the rotated keys kq, and the blocks that it fills."""
    kc, vc, full = a.k_cache.clone(), a.v_cache.clone(), []
    for b in range(a.B):
        ctx, n = int(a.context_lens[b]), cu[b + 1] - cu[b]
        if ctx <= 0 or ctx > a.max_blocks * 16:
            continue
        for i in range(n):
            pos = ctx - n + i
            if pos < 0:
                continue
            blk = int(a.block_table[b, pos // 16])
            if not 0 <= blk < a.num_blocks:
                continue
            kc[blk, :, pos % 16] = kq[cu[b] + i]
            vc[blk, :, :, pos % 16] = v[cu[b] + i]
            if pos % 16 == 15:
                full.append(blk)
    return kc, vc, full


def _summary_bytes(a, seed=5):
    g = torch.Generator().manual_seed(seed)
    return aflex.BlockSummary(torch.randint(-9, 9, (a.num_blocks, a.Hkv, a.D), generator=g).to(torch.int8),
                              torch.randint(-9, 9, (a.num_blocks, a.Hkv), generator=g).to(torch.int8))


def _check_written(a, ad, s, sd, k, v, cu, angles, inter, left=()):
    """The pools and summaries on the GPU after a write, rows `left` left alone."""
    got = ad.k_cache.cpu()
    kq = lc.rotate(k, angles, inter).bfloat16() if angles is not None else k.clone()
    kc, vc, full = _expect_write(a, k, v, cu, kq)
    # rotated keys: to a rounding; their bits as held go on
    slots = (kc != a.k_cache).any(-1)
    assert torch.equal(got[~slots], kc[~slots]), "key slots that are not written"
    if angles is None:
        assert torch.equal(got, kc)
    else:
        d, ref = (got[slots].double() - kc[slots].double()).abs(), kc[slots].double().abs()
        # both sides are rounded: two half steps, and the fp32 part
        assert bool((d <= 2 * 2.0 ** -8 * ref * (1 + 2.0 ** -7) + 2.0 ** -20 * 8).all())
    assert torch.equal(ad.v_cache.cpu(), vc), "values"
    keys, exp = s.keys.clone(), s.exp.clone()
    for blk in full:
        for g in range(a.Hkv):
            keys[blk, g], exp[blk, g] = lc.summarise(got[blk, g])
    assert torch.equal(sd.keys.cpu(), keys) and torch.equal(sd.exp.cpu(), exp), "summaries"


HEADS = [(8, 2, 64), (64, 8, 128), (5, 5, 64), (28, 4, 128), (48, 3, 128), (3, 1, 128)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("rot,inter,strided", [(1.0, False, True), (1.0, True, False), (0.5, False, False),
                                               (0.25, True, True), (0.0, False, True)])
def test_append(gpu_lib, heads, rot, inter, strided):
    ctx = [1, 16, 17, 31, 32, 33, 48, 100, 160, 5]
    Hq, Hkv, D = heads
    R = int(rot * D)
    a = synth.custom_attention(11, len(ctx), Hq, Hkv, D, ctx, ctx_hi=160)
    s = _summary_bytes(a)
    (q, k, v), dev = _tokens(12, a.B, heads, strided)
    rope = aflex.rope_table(160, R, 1000.0) if R else None
    ad, sd = a.to(DEV), aflex.BlockSummary(s.keys.to(DEV), s.exp.to(DEV))
    out = aflex.rope_append(ad, *dev, None if rope is None else rope.to(DEV), interleaved=inter, summary=sd)
    ang = rope[torch.tensor(ctx) - 1] if R else None
    if R:
        _check_rotation(out.cpu(), q, ang, inter, "queries")
    else:
        assert torch.equal(out.cpu(), q)
    _check_written(a, ad, s, sd, k, v, list(range(a.B + 1)), ang, inter)


def test_append_rotates_like_fp32_operations(gpu_lib):
    """The bits are those of the formula with each fp32 operation rounded."""
    a = synth.custom_attention(13, 6, 16, 4, 128, [40, 1, 7, 99, 16, 64], ctx_hi=112)
    (q, k, v), dev = _tokens(14, 6, (16, 4, 128), False)
    rope = aflex.rope_table(112, 128)
    out = aflex.rope_append(a.to(DEV), *dev, rope.to(DEV)).cpu()
    t = rope[a.context_lens.long() - 1]
    c, s, x, y = t[:, None, :64], t[:, None, 64:], q[..., :64].float(), q[..., 64:].float()
    assert torch.equal(out, torch.cat([x * c - y * s, y * c + x * s], -1).bfloat16())


def test_append_leaves_alone_what_has_no_place(gpu_lib):
    """Empty and over-long contexts, positions outside the table, bad block ids."""
    heads = (8, 2, 128)
    a = synth.custom_attention(15, 7, *heads, [20, 40, 33, 16, 50, 48, 8], ctx_hi=64)
    a.context_lens = torch.tensor([0, -3, 33, 16, 65, 48, 8], dtype=torch.int32)  # capacity 64
    a.block_table[3, 0], a.block_table[6, 0] = -1, a.num_blocks
    s = _summary_bytes(a)
    (q, k, v), dev = _tokens(16, 7, heads, True)
    rope = aflex.rope_table(70, 128)
    positions = torch.tensor([1, 1, 70, 3, 4, -1, 60], dtype=torch.int32)
    for pos in (None, positions):
        ad, sd = a.to(DEV), aflex.BlockSummary(s.keys.to(DEV), s.exp.to(DEV))
        out = torch.full((7, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        aflex.rope_append(ad, *dev, rope.to(DEV), summary=sd, q_out=out,
                          positions=None if pos is None else pos.to(DEV))
        at = a.context_lens.long() - 1 if pos is None else pos.long()
        live = [2, 3, 5, 6] if pos is None else [3, 6]
        for b in range(7):
            if b in live:
                _check_rotation(out[b:b + 1].cpu(), q[b:b + 1], rope[at[b]:at[b] + 1], False, f"row {b}")
            else:
                assert bool((out[b] == 7).all())
        c = synth.AttnInputs(**a.__dict__)
        c.context_lens = torch.where(torch.tensor([b in live for b in range(7)]), a.context_lens, 0)
        _check_written(c, ad, s, sd, k, v, list(range(8)), rope[at.clamp(0, 69)], False)


def test_append_at_far_positions(gpu_lib):
    heads = (4, 1, 128)
    a = synth.custom_attention(17, 3, *heads, [20, 33, 8], ctx_hi=48)
    (q, k, v), dev = _tokens(18, 3, heads, False)
    rope = aflex.rope_table(1 << 20, 128, 500000.0)
    pos = torch.tensor([(1 << 20) - 1, 999999, 524288], dtype=torch.int32)
    out = aflex.rope_append(a.to(DEV), *dev, rope.to(DEV), positions=pos.to(DEV))
    _check_rotation(out.cpu(), q, rope[pos.long()], False, "far")


WRITES = [([1], [0]), ([15, 16, 17, 0, 1, 33], [0] * 6), ([5, 0, 27, 16, 1, 40], [3, 9, 5, 16, 15, 31]),
          ([130, 2], [7, 30]), ([0, 0, 3], [1, 20, 13])]


@pytest.mark.parametrize("lens,past", WRITES)
@pytest.mark.parametrize("heads,R,inter,strided", [((8, 2, 64), 64, False, True), ((64, 8, 128), 128, False, False),
                                                   ((28, 4, 128), 96, True, True), ((20, 20, 64), 16, True, False),
                                                   ((17, 17, 128), 0, False, True), ((48, 3, 128), 48, False, True)])
def test_write(gpu_lib, lens, past, heads, R, inter, strided):
    Hq, Hkv, D = heads
    ctx = [n + p for n, p in zip(lens, past)]
    a = synth.custom_attention(21, len(ctx), Hq, Hkv, D, ctx, ctx_hi=max(max(ctx), 1) + 5)
    s = _summary_bytes(a)
    T = sum(lens)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    (q, k, v), dev = _tokens(22, T, heads, strided)
    rope = aflex.rope_table(200, R, 100.0) if R else None
    ad, sd = a.to(DEV), aflex.BlockSummary(s.keys.to(DEV), s.exp.to(DEV))
    out = aflex.rope_write(ad, *dev, torch.tensor(cu, dtype=torch.int32, device=DEV),
                           None if rope is None else rope.to(DEV), interleaved=inter, summary=sd)
    pos = torch.tensor([p + i for n, p in zip(lens, past) for i in range(n)])
    ang = rope[pos] if R else None
    if R:
        _check_rotation(out.cpu(), q, ang, inter, "queries")
    else:
        assert torch.equal(out.cpu(), q)
    _check_written(a, ad, s, sd, k, v, cu, ang, inter)


def test_write_longer_than_the_cache_and_out_of_range(gpu_lib):
    """New tokens before place 0, contexts over the capacity, bad ids, positions outside the table."""
    heads = (8, 2, 64)
    a = synth.custom_attention(23, 4, *heads, [40, 40, 64, 20], ctx_hi=64)
    a.context_lens = torch.tensor([30, 70, 64, 20], dtype=torch.int32)
    a.block_table[2, 1] = a.num_blocks + 5
    lens = [40, 10, 50, 20]
    cu = [0, 40, 50, 100, 120]
    s = _summary_bytes(a)
    (q, k, v), dev = _tokens(24, 120, heads, True)
    rope = aflex.rope_table(60, 64)
    ad, sd = a.to(DEV), aflex.BlockSummary(s.keys.to(DEV), s.exp.to(DEV))
    out = torch.full((120, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    aflex.rope_write(ad, *dev, torch.tensor(cu, dtype=torch.int32, device=DEV), rope.to(DEV), summary=sd, q_out=out)
    out, got = out.cpu(), ad.k_cache.cpu()
    kc, vc = a.k_cache.clone(), a.v_cache.clone()
    for b, n in enumerate(lens):
        for i in range(n):
            r, pos = cu[b] + i, int(a.context_lens[b]) - n + i
            if b == 1 or pos < 0 or pos >= 60:
                assert bool((out[r] == 7).all())
                continue
            _check_rotation(out[r:r + 1], q[r:r + 1], rope[pos:pos + 1], False, f"row {r}")
            blk = int(a.block_table[b, pos // 16])
            if blk < a.num_blocks:
                _check_rotation(got[blk, :, pos % 16][None], k[r:r + 1], rope[pos:pos + 1], False, f"key {r}")
                kc[blk, :, pos % 16] = got[blk, :, pos % 16]
                vc[blk, :, :, pos % 16] = v[r]
    assert torch.equal(got, kc) and torch.equal(ad.v_cache.cpu(), vc)
    # (block 3 of sequence 2 is not filled: its place 63 is left alone)
    full = [int(a.block_table[b, j]) for b, j in ((0, 0), (2, 0), (2, 2), (3, 0))]
    keys, exp = s.keys.clone(), s.exp.clone()
    for blk in full:
        for g in range(2):
            keys[blk, g], exp[blk, g] = lc.summarise(got[blk, g])
    assert torch.equal(sd.keys.cpu(), keys) and torch.equal(sd.exp.cpu(), exp)


def test_write_of_nothing(gpu_lib):
    a = synth.custom_attention(19, 2, 8, 2, 64, [20, 33], ctx_hi=48).to(DEV)
    before = a.k_cache.clone()
    e = torch.empty(0, 8, 64, dtype=torch.bfloat16, device=DEV)
    out = aflex.rope_write(a, e, e[:, :2], e[:, :2], torch.zeros(3, dtype=torch.int32, device=DEV),
                           aflex.rope_table(48, 64).to(DEV))
    assert out.shape == (0, 8, 64) and torch.equal(a.k_cache, before)


def test_write_of_single_tokens_is_append(gpu_lib):
    heads = (28, 4, 128)
    a = synth.custom_attention(25, 9, *heads, [1, 16, 17, 32, 64, 65, 7, 48, 50], ctx_hi=80)
    _, dev = _tokens(26, 9, heads, True)
    rope = aflex.rope_table(80, 128).to(DEV)
    one, two = a.to(DEV), a.to(DEV)
    s1, s2 = aflex.BlockSummary.of(one), aflex.BlockSummary.of(two)
    o1 = aflex.rope_append(one, *dev, rope, summary=s1)
    o2 = aflex.rope_write(two, *dev, torch.arange(10, dtype=torch.int32, device=DEV), rope, max_seqlen=1, summary=s2)
    for x, y in [(o1, o2), (one.k_cache, two.k_cache), (one.v_cache, two.v_cache), (s1.keys, s2.keys), (s1.exp, s2.exp)]:
        assert torch.equal(x, y)


# ------------------------------------------------------------------ summaries
def _odd_keys(seed, a):
    """Pools with large and small blocks, zeros, subnormals and non-finite keys."""
    g = torch.Generator().manual_seed(seed)
    a.k_cache = (a.k_cache.float() * torch.exp2(torch.randint(-30, 30, (a.num_blocks, a.Hkv, 1, 1), generator=g))
                 ).bfloat16()
    a.k_cache[0], a.k_cache[1, 0] = 0.0, 1e-39
    a.k_cache[2, 0, 3, 5], a.k_cache[3, a.Hkv - 1, 15, a.D - 1] = float("nan"), -float("inf")
    a.k_cache[4, 0], a.k_cache[5, 0] = 3.3e38, -3.3e38
    return a


@pytest.mark.parametrize("heads", HEADS)
def test_block_summary(gpu_lib, heads):
    a = _odd_keys(31, synth.custom_attention(31, 6, *heads, [150, 0, 15, 16, 47, 160], ctx_hi=176))
    a.block_table[5, 2], a.block_table[0, 3] = -7, a.num_blocks
    s = _summary_bytes(a)
    sd = aflex.block_summary(a.to(DEV), aflex.BlockSummary(s.keys.to(DEV), s.exp.to(DEV)))
    keys, exp = lc.block_summary(a.k_cache, a.block_table, a.context_lens, s.keys, s.exp)
    assert torch.equal(sd.keys.cpu(), keys) and torch.equal(sd.exp.cpu(), exp)


def test_block_summary_more_tiles_than_work_groups(gpu_lib):
    """2100 sequences leave each 16 work-groups, 128 tiles a pass: 200 and 136 tiles take two."""
    ctx = [0, 16, 15] * 700
    ctx[0], ctx[1], ctx[2099] = 405, 256, 272
    heads = (8, 8, 64)
    a = _odd_keys(32, synth.custom_attention(32, len(ctx), *heads, ctx, ctx_hi=416))
    s = _summary_bytes(a)
    sd = aflex.block_summary(a.to(DEV), aflex.BlockSummary(s.keys.to(DEV), s.exp.to(DEV)))
    keys, exp = lc.block_summary(a.k_cache, a.block_table, a.context_lens, s.keys, s.exp)
    assert torch.equal(sd.keys.cpu(), keys) and torch.equal(sd.exp.cpu(), exp)


# ------------------------------------------------------------------ the choice
def _choice(seed, ctx, heads, top, sink, recent, edit=None):
    Hq, Hkv, D = heads
    table, n = synth.paged_block_table(np.random.default_rng(seed), np.array(ctx, dtype=np.int32),
                                       -(-max(max(ctx), 1) // 16))
    a = synth.AttnInputs(q=_bf(seed, len(ctx), Hq, D), k_cache=torch.empty(0), v_cache=torch.empty(0),
                         block_table=torch.from_numpy(table), context_lens=torch.tensor(ctx, dtype=torch.int32),
                         B=len(ctx), Hq=Hq, Hkv=Hkv, D=D, block_size=16, max_blocks=table.shape[1], num_blocks=n,
                         max_context_len=16 * table.shape[1])
    g = torch.Generator().manual_seed(seed)
    s = aflex.BlockSummary(torch.randint(-127, 128, (n, Hkv, D), generator=g).to(torch.int8),
                           torch.randint(-9, -5, (n, Hkv), generator=g).to(torch.int8))
    if edit:
        edit(a, s)
    got = aflex.block_select(a.to(DEV), a.q.to(DEV), aflex.BlockSummary(s.keys.to(DEV), s.exp.to(DEV)), top, sink,
                             recent)
    ref = lc.select(a.q, s.keys, s.exp, a.block_table, a.context_lens, top, sink, recent)
    assert torch.equal(got.cpu(), ref)


@pytest.mark.parametrize("heads", HEADS + [(16, 1, 64), (32, 2, 128)])
@pytest.mark.parametrize("top,sink,recent", [(8, 1, 1), (5, 2, 3), (17, 0, 4), (64, 1, 2), (1, 0, 1)])
def test_block_select(gpu_lib, heads, top, sink, recent):
    _choice(41, [1, 16, 129, 700, 1000, 0, 1024, 333], heads, top, sink, recent)


@pytest.mark.parametrize("ctx,top", [([16400, 40000], 128), ([17000], 1000), ([33000, 5, 16384, 16385], 1024),
                                     ([540000], 300), ([300000, 280000], 4096)])
def test_block_select_long(gpu_lib, ctx, top):
    _choice(42, ctx, (8, 1, 64), top, 4, 8)


def test_block_select_ties_and_odd_values(gpu_lib):
    heads = (8, 2, 128)

    def equal(a, s):
        s.keys.fill_(1), s.exp.fill_(-7)

    def few(a, s):  # a handful of distinct scores
        s.keys.copy_((s.keys > 0).to(torch.int8) * (torch.arange(128) == 3).to(torch.int8))
        s.exp.fill_(-4)

    def odd(a, s):
        s.exp[::3] = 127
        s.exp[1::7] = 120
        s.exp[2::7] = -118
        a.q[0, 0, 5], a.q[0, 3, 6], a.q[1, 1] = float("nan"), float("inf"), float("nan")
        a.q[1, 4:], a.q[2, :4] = 0.0, 1e-39
        a.q[2, 4:] = 3e38
        a.block_table[0, 3:9] = -1
        a.block_table[2, 10:40] = a.num_blocks

    for seed, edit in enumerate((equal, few, odd)):
        for top in (4, 9, 40):
            _choice(43 + seed, [900, 640, 1500], heads, top, 2, 2, edit=edit)


@pytest.mark.parametrize("heads", HEADS + [(16, 1, 64), (32, 2, 128), (18, 9, 64)])
@pytest.mark.parametrize("top,sink,recent", [(9, 1, 2), (200, 0, 1)])
def test_block_select_ragged_with_one_long(gpu_lib, heads, top, sink, recent):
    _choice(48, [17000, 300, 0, 16400, 1, 3300, 63, 4096], heads, top, sink, recent)


@pytest.mark.parametrize("n", [1100, 5000, 33000])
@pytest.mark.parametrize("top", [64, 1500])
def test_block_select_long_with_equal_scores(gpu_lib, n, top):
    """More equal scores than the short lists hold, and a few that stand out at the ends."""
    def equal(a, s):
        s.keys.fill_(1), s.exp.fill_(-7)

    def two(a, s):
        equal(a, s)
        s.exp[a.block_table[0, 5::7].long()] = -6
        s.exp[a.block_table[0, n - 3].long()] = -8

    for edit in (equal, two):
        _choice(49, [16 * n - 5], (4, 1, 64), top, 1, 1, edit=edit)


def test_block_select_long_sequences_among_many_short(gpu_lib):
    ctx = [5] * 200
    ctx[3], ctx[70], ctx[199] = 17000, 2100, 18000
    _choice(53, ctx, (4, 2, 64), 20, 1, 1)


def test_block_select_many_units_under_a_long_bound(gpu_lib):
    """1024 units, most of them short: long and short ones are chosen by launches of their own."""
    ctx = [16 * (i % 40) + i % 17 for i in range(128)]
    ctx[5], ctx[77], ctx[100] = 70000, 66000, 30000
    _choice(55, ctx, (8, 8, 64), 20, 1, 1)


def test_block_select_scores_too_small_for_fp32(gpu_lib):
    """Scores of both signs that round to zero are equal."""
    def tiny(a, s):
        a.q *= 2.0 ** -100
        s.exp.fill_(-118)
        s.exp[a.block_table[0, 30:33].long()] = 0

    for ctx in (900, 17000):
        _choice(54, [ctx], (8, 2, 128), 12, 1, 1, edit=tiny)


def test_block_select_heads_far_apart_in_size(gpu_lib):
    """Heads of one group whose scales differ by more than fp32's range, both with whole codes."""
    def far(a, s):
        a.q[:, 0], a.q[:, 1] = a.q[:, 0] * 1e30, a.q[:, 1].abs() * -1e-25
        a.q[0, 2:4] *= 1e-20
        s.exp[::2] = -118
        s.exp[1::5] = 100
        s.keys[::3] = 0

    for ctx in ([900, 640], [17000, 400]):
        _choice(50, ctx, (8, 2, 128), 12, 1, 1, edit=far)


def test_block_select_takes_no_more_than_the_host_bound(gpu_lib):
    """Device contexts over max_context_len are cut to it, negative ones are empty."""
    a = synth.custom_attention(47, 3, 8, 2, 64, [320, 100, 300], ctx_hi=320)
    s = aflex.block_summary(a.to(DEV))
    a.max_context_len = 200
    a.context_lens[1] = -4
    sel = aflex.block_select(a.to(DEV), a.q.to(DEV), s, 6, 1, 1).cpu()
    b = synth.AttnInputs(**a.__dict__)
    b.context_lens = a.context_lens.clamp(0, 200)
    assert torch.equal(sel, lc.select(a.q, s.keys.cpu(), s.exp.cpu(), a.block_table, b.context_lens, 6, 1, 1))


# ------------------------------------------------------------------- attention
def _attend(a, sel, **kw):
    got = aflex.attn_sparse_decode(a.to(DEV), sel.to(DEV), **kw).cpu()
    again = aflex.attn_sparse_decode(a.to(DEV), sel.to(DEV), **kw).cpu()
    assert torch.equal(got, again)
    ref, mag = lc.attention_sparse(a.q, a.k_cache, a.v_cache, a.block_table, a.context_lens, sel, kw.get("scale"))
    bound = 2.0 ** -8 * ref.abs() + (2.0 ** -7 + 2.0 ** -10) * mag
    bad = (got.double() - ref).abs() > bound
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} values"
    return got


def _lists(seed, a, top):
    g = torch.Generator().manual_seed(seed)
    sel = torch.full((a.B, a.Hkv, top), -1, dtype=torch.int32)
    for b, ctx in enumerate(a.context_lens.tolist()):
        n = -(-max(ctx, 0) // 16)
        for h in range(a.Hkv):
            row = torch.randperm(n, generator=g)[:min(n, top)].sort().values
            if n:
                row[-1] = n - 1
            sel[b, h, :len(row)] = row.int()
    return sel


@pytest.mark.parametrize("heads", HEADS + [(16, 1, 64), (32, 2, 128)])
@pytest.mark.parametrize("top", [1, 7, 33, 70])
def test_attention(gpu_lib, heads, top):
    a = synth.custom_attention(51, 7, *heads, [1, 16, 150, 0, 700, 1111, 33], ctx_hi=1120)
    _attend(a, _lists(52, a, top))


def test_attention_of_many_units(gpu_lib):
    """1024 and more (sequence, kv head) pairs: a work-group each; and lists too long for that."""
    ctx = [1 + 37 * i % 700 for i in range(64)]
    a = synth.custom_attention(62, 64, 16, 16, 64, ctx, ctx_hi=720)
    a.context_lens[::9] = 0
    for top in (5, 20, 45):
        _attend(a, _lists(63 + top, a, top))
    b = synth.custom_attention(64, 128, 8, 8, 128, [50 + 17 * i % 300 for i in range(127)] + [3000])
    _attend(b, _lists(65, b, 150))


def test_attention_split_over_many_work_groups(gpu_lib):
    a = synth.custom_attention(53, 1, 16, 2, 128, [9000])
    _attend(a, _lists(54, a, 500))
    a = synth.custom_attention(55, 40, 8, 8, 64, [600 + 13 * i for i in range(40)])
    _attend(a, _lists(56, a, 60), scale=0.3)


def test_attention_ignores_what_is_no_ascending_block(gpu_lib):
    a = synth.custom_attention(57, 4, 8, 2, 128, [800, 650, 30, 300], ctx_hi=800)
    a.block_table[1, 4:9] = torch.tensor([-1, a.num_blocks, -5, 1 << 30, a.num_blocks + 1], dtype=torch.int32)
    sel = _lists(58, a, 40)
    sel[0, 0, 5], sel[0, 1, 7:9], sel[0, 0, 30:] = sel[0, 0, 4], -1, 1 << 30
    sel[1, 0, 3], sel[1, 1, 0], sel[1, 1, 6] = 99, -9, 0
    sel[2] = -1          # nothing is left of this sequence
    sel[3, 1, 0:19] = -1  # nor of this head
    got = _attend(a, sel)
    assert not got[2].any() and not got[3, 4:].any()


def test_attention_masks_what_is_behind_the_context(gpu_lib):
    """NaN and infinities in the unused slots of the last block and in blocks that are not listed."""
    a = synth.custom_attention(59, 3, 8, 2, 64, [70, 641, 16], ctx_hi=656)
    sel = _lists(60, a, 12)
    used = torch.zeros(a.num_blocks, 2, 16, dtype=torch.bool)
    for b, ctx in enumerate(a.context_lens.tolist()):
        for g in range(2):
            for j in sel[b, g].tolist():
                if j >= 0:
                    used[a.block_table[b, j], g, :min(16, ctx - 16 * j)] = True
    a.k_cache[~used] = float("nan")
    a.v_cache.transpose(2, 3)[~used] = float("inf")
    _attend(a, sel)


def test_all_blocks_give_dense_attention(gpu_lib):
    for top in (50, 64):
        a = synth.custom_attention(61, 5, 32, 4, 128, [790, 1, 0, 512, 333], ctx_hi=800)
        ad = a.to(DEV)
        sel = aflex.block_select(ad, ad.q, aflex.block_summary(ad), top)
        assert torch.equal(sel.cpu()[0, 0, :50], torch.arange(50, dtype=torch.int32))
        _attend(a, sel.cpu())
        dense, sparse = aflex.attn_decode(ad).float(), aflex.attn_sparse_decode(ad, sel).float()
        # the same weights and values, split otherwise: both are within the bound of the exact result
        _, mag = lc.attention_sparse(a.q, a.k_cache, a.v_cache, a.block_table, a.context_lens, sel.cpu())
        bound = 2 * (2.0 ** -8 * dense.cpu().double().abs() + (2.0 ** -7 + 2.0 ** -10) * mag)
        assert bool(((dense - sparse).cpu().double().abs() <= bound).all())


# ---------------------------------------------------------------- all together
def _step(a, dev, rope, s, top, **kw):
    q = aflex.rope_append(a, *dev, rope, summary=s, **{k: v for k, v in kw.items() if k == "stream"})
    sel = aflex.block_select(a, q, s, top, 1, 2, **kw)
    return q, sel, aflex.attn_sparse_decode(a, sel, q=q, **kw)


def test_decode_step(gpu_lib):
    """A prompt written in two chunks, then decode steps over block borders: the cache, the summaries that the
    writes keep, the choice and the attention, each step against the oracle on the cache as it is held."""
    heads = (16, 2, 128)
    lens = [300, 45, 16, 129]
    a = synth.custom_attention(71, 4, *heads, [n + 40 for n in lens], ctx_hi=352)
    a.k_cache.zero_(), a.v_cache.zero_()
    ad = a.to(DEV)
    s = aflex.BlockSummary.of(ad)
    rope = aflex.rope_table(352, 128).to(DEV)
    for part in (0, 1):
        n = [l // 3 if part == 0 else l - l // 3 for l in lens]
        ad.context_lens.copy_(torch.tensor([l // 3 if part == 0 else l for l in lens]))
        cu = torch.tensor([0] + n).cumsum(0).int()
        aflex.rope_write(ad, *_tokens(72 + part, sum(n), heads, True)[1], cu.to(DEV), rope, summary=s)
    for t in range(20):
        ad.context_lens += 1
        _, dev = _tokens(80 + t, 4, heads, True)
        q, sel, out = _step(ad, dev, rope, s, 6)
        if t % 3 == 0:
            h = synth.AttnInputs(**{**ad.__dict__, "q": q}).to("cpu")
            keys, exp = lc.block_summary(h.k_cache, h.block_table, h.context_lens, *(x.cpu() for x in (s.keys, s.exp)))
            assert torch.equal(s.keys.cpu(), keys) and torch.equal(s.exp.cpu(), exp)
            assert torch.equal(sel.cpu(), lc.select(h.q, keys, exp, h.block_table, h.context_lens, 6, 1, 2))
            ref, mag = lc.attention_sparse(h.q, h.k_cache, h.v_cache, h.block_table, h.context_lens, sel.cpu())
            assert bool(((out.cpu().double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -7 + 2.0 ** -10) * mag).all())


def test_captured_and_replayed(gpu_lib):
    """Two captured steps of different sizes, replayed in turn with eager work between."""
    steps = []
    for seed, ctx, heads, top in [(91, [900, 77, 640], (8, 2, 64), 9), (92, [3000] * 5, (32, 8, 128), 40)]:
        a = synth.custom_attention(seed, len(ctx), *heads, ctx).to(DEV)
        rope = aflex.rope_table(3008, heads[2]).to(DEV)
        s = aflex.block_summary(a)
        dev = _tokens(seed, a.B, heads, True)[1]
        eager = [x.clone() for x in _step(a, dev, rope, s, top)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs = _step(a, dev, rope, s, top)
        steps.append((g, outs, eager, a, dev, rope, s, top))
    for _ in range(3):
        for g, outs, eager, *_ in steps:
            for x in outs:
                x.zero_()
            g.replay()
        for g, outs, eager, a, dev, rope, s, top in steps:
            again = _step(a, dev, rope, s, top)
            torch.cuda.synchronize()
            for x, y, z in zip(outs, eager, again):
                assert torch.equal(x, y) and torch.equal(z, y)


def test_two_streams_at_once(gpu_lib):
    work = []
    for seed in (95, 96):
        a = synth.custom_attention(seed, 4, 32, 8, 128, [2000, 1500, 1000, 1700], ctx_hi=2000).to(DEV)
        s = aflex.block_summary(a)
        dev = _tokens(seed, 4, (32, 8, 128), False)[1]
        rope = aflex.rope_table(2000, 128).to(DEV)
        work.append((a, dev, rope, s, 20, [x.clone() for x in _step(a, dev, rope, s, 20)], torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[] for _ in work]
    for _ in range(5):
        for i, (*args, _ref, stream) in enumerate(work):
            got[i].append(_step(*args, stream=stream))
    torch.cuda.synchronize()
    for i, w in enumerate(work):
        for outs in got[i]:
            for x, y in zip(outs, w[5]):
                assert torch.equal(x, y)


def test_pools_of_more_than_2_to_the_31_elements(gpu_lib):
    """Blocks at the far end of pools whose offsets pass 32 bits."""
    Hq, Hkv, D, n = 8, 8, 128, 140000  # 2.3e9 elements a pool
    a = synth.custom_attention(97, 2, Hq, Hkv, D, [100, 64], ctx_hi=112)
    small = a.to(DEV)
    move = torch.tensor([n - 1 - 3 * i for i in range(a.num_blocks)], device=DEV)
    big = synth.AttnInputs(**small.__dict__)
    big.num_blocks = n
    big.k_cache = torch.zeros(n, Hkv, 16, D, dtype=torch.bfloat16, device=DEV)
    big.v_cache = torch.zeros(n, Hkv, D, 16, dtype=torch.bfloat16, device=DEV)
    big.k_cache[move], big.v_cache[move] = small.k_cache, small.v_cache
    big.block_table = torch.where(small.block_table >= 0, move[small.block_table.clamp(min=0).long()].int(), -1).int()
    rope = aflex.rope_table(112, 128).to(DEV)
    dev = _tokens(98, 2, (Hq, Hkv, D), False)[1]
    res = []
    for c in (small, big):
        s = aflex.block_summary(c)
        res.append((*_step(c, dev, rope, s, 4), s))
    for x, y in zip(res[0][:3], res[1][:3]):
        assert torch.equal(x, y)
    assert torch.equal(res[0][3].keys, res[1][3].keys[move]) and torch.equal(res[0][3].exp, res[1][3].exp[move])
    assert torch.equal(small.k_cache, big.k_cache[move]) and torch.equal(small.v_cache, big.v_cache[move])


@pytest.mark.parametrize("op", ["attn_sparse_decode", "attn_decode"])
def test_workspace_grown_while_another_stream_reads_it(gpu_lib, op):
    """A caller's workspace used on a busy stream, then grown on the one it is from: its
    memory is not handed out before the busy stream is done."""
    small, large = [(a.to(DEV), _lists(101, a, 70).to(DEV)) for a in (
        synth.custom_attention(99, 2, 8, 2, 128, [2000, 1500]), synth.custom_attention(100, 64, 8, 2, 128, [600] * 64))]

    def run(x, ws):
        return aflex.attn_decode(x[0], ws=ws) if op == "attn_decode" else aflex.attn_sparse_decode(*x, ws=ws)

    want = run(small, None)
    ws, side = aflex.Workspace(), torch.cuda.Stream()
    run(small, ws)
    torch.cuda.synchronize()
    at, size = ws.buf.data_ptr(), ws.buf.numel()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
        got = run(small, ws)
    run(large, ws)
    assert not side.query()  # still asleep
    assert ws.buf.numel() > size
    other = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(4)]
    assert all(not t.data_ptr() <= at < t.data_ptr() + size for t in other)
    for t in other:
        t.fill_(255)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("heads", [(8, 2, 64), (64, 8, 128), (28, 4, 128)])
@pytest.mark.parametrize("top", [7, 70])
def test_attention_carries_one_rounding(gpu_lib, heads, top):
    """Scores that are exact (one channel of the keys, its query 1): what is left is the output's rounding,
    2^-8 |out|, the weights' as two bf16 values, 2^-16 each above and below the line, exponents of at most 2^-19,
    and the sums: a wave adds at most 36 pairs of blocks, of 70, in steps of 32 products twice, so 64 roundings
    of 2^-23 for each of the 9 pairs that it has, 2^-13.8. In all less than 2^-13 sum p|v|."""
    a = synth.custom_attention(111, 6, *heads, [1, 150, 0, 700, 1111, 33], ctx_hi=1120)
    a.k_cache[..., 1:] = 0
    a.k_cache[..., 0] = (a.k_cache[..., 0].float() * 2).clamp(-4, 4).bfloat16()
    a.q[..., 0] = 1
    sel = _lists(112, a, top)
    got = aflex.attn_sparse_decode(a.to(DEV), sel.to(DEV), scale=1.0).cpu().double()
    ref, mag = lc.attention_sparse(a.q, a.k_cache, a.v_cache, a.block_table, a.context_lens, sel, 1.0)
    bad = (got - ref).abs() > 2.0 ** -8 * ref.abs() + 2.0 ** -13 * mag
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} values"


@pytest.mark.parametrize("B,heads,blocks,top", [(128, (8, 8, 64), (110, 130), 100), (128, (32, 8, 128), (66, 90), 128),
                                                (64, (8, 8, 64), (140, 200), 128), (64, (32, 8, 128), (140, 200), 128),
                                                (3, (4, 2, 128), (400, 600), 300), (40, (8, 8, 64), (60, 100), 90)])
def test_attention_of_long_lists_shows_every_block(gpu_lib, B, heads, blocks, top):
    """Keys of zero, so every weight is 1, and values of whole numbers in one channel per block: a result is
    sum / count, rounded to bf16 once, and shows each block that is lost, doubled or strange. Lists longer than
    the 64 entries that a wave holds at a time, a work-group per list and split ones, with entries around the
    64th that contribute nothing."""
    Hq, Hkv, D = heads
    g = torch.Generator().manual_seed(120 + B)
    n = blocks[1]
    nblk = torch.randint(blocks[0], n + 1, (B,), generator=g)
    ctx = (nblk * 16 - torch.randint(0, 16, (B,), generator=g)).int()
    table = torch.stack([torch.randperm(n, generator=g) for _ in range(B)]).int()
    head = torch.arange(Hkv)
    v = torch.zeros(n, Hkv, D, 16)
    for blk in range(n):
        v[blk, head, (blk + head) % D] = 1 + blk // D
    sel = torch.full((B, Hkv, top), -1, dtype=torch.int32)
    for b in range(B):
        for h in range(Hkv):
            row = torch.randperm(int(nblk[b]), generator=g)[:top].sort().values.int()
            row[-1] = nblk[b] - 1
            kind = (b + h) % 4
            if kind == 1 and len(row) > 63:
                row[63] = -1
            elif kind == 2:
                row[64:] = torch.cat([row[63:64], row[65:]]) if len(row) > 64 else row[64:]
            elif kind == 3 and len(row) > 66:
                row[65] = nblk[b] + 5  # (the next one is not greater)
            sel[b, h, :len(row)] = row
    a = synth.AttnInputs(q=_bf(121, B, Hq, D), k_cache=torch.zeros(n, Hkv, 16, D, dtype=torch.bfloat16),
                         v_cache=v.bfloat16(), block_table=table, context_lens=ctx, B=B, Hq=Hq, Hkv=Hkv, D=D,
                         block_size=16, max_blocks=n, num_blocks=n, max_context_len=16 * n)
    got = aflex.attn_sparse_decode(a.to(DEV), sel.to(DEV)).cpu().double()
    prev = torch.cat([torch.full((B, Hkv, 1), -1, dtype=torch.int32), sel[..., :-1]], -1)
    valid = (sel > prev) & (sel >= 0) & (sel < nblk[:, None, None])
    j = sel.clamp(0, n - 1).long()
    tokens = (ctx[:, None, None] - 16 * j).clamp(max=16).double() * valid
    blk = torch.gather(table.long()[:, None].expand(B, Hkv, n), 2, j)
    ref = torch.zeros(B, Hkv, D, dtype=torch.float64)
    ref.scatter_add_(2, (blk + head[:, None]) % D, tokens * (1 + blk // D))
    ref = (ref / tokens.sum(-1, keepdim=True)).repeat_interleave(Hq // Hkv, 1)
    assert bool(((got - ref).abs() <= 2.0 ** -8 * ref).all())


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("heads,R,inter", [((16, 4, 128), 128, True), ((16, 4, 128), 64, False), ((28, 4, 128), 96, True),
                                           ((8, 2, 64), 64, True), ((8, 2, 64), 16, False), ((5, 5, 64), 48, True)])
def test_rotation_bits_of_both_pairings_and_of_a_part(gpu_lib, packed, heads, R, inter):
    """As test_append_rotates_like_fp32_operations, for queries and cached keys."""
    Hq, Hkv, D = heads
    ctx = [40, 1, 7, 99, 16, 64]
    a = synth.custom_attention(131, 6, *heads, ctx, ctx_hi=112).to(DEV)
    (q, k, _), dev = _tokens(132, 6, heads, True)
    rope = aflex.rope_table(112, R, 1000.0)
    if packed:
        cu = torch.arange(7, dtype=torch.int32, device=DEV)
        out = aflex.rope_write(a, *dev, cu, rope.to(DEV), interleaved=inter)
    else:
        out = aflex.rope_append(a, *dev, rope.to(DEV), interleaved=inter)
    pos = torch.tensor(ctx) - 1
    i = torch.arange(R // 2)
    ia, ib = (2 * i, 2 * i + 1) if inter else (i, i + R // 2)
    c, s = rope[pos][:, None, :R // 2], rope[pos][:, None, R // 2:]

    def turned(x):
        y = x.clone()
        f, g = x[..., ia].float(), x[..., ib].float()
        y[..., ia], y[..., ib] = (f * c - g * s).bfloat16(), (g * c + f * s).bfloat16()
        return y

    assert torch.equal(out.cpu(), turned(q))
    kc = a.k_cache.cpu()
    got = torch.stack([kc[a.block_table[b, p // 16], :, p % 16] for b, p in enumerate(pos.tolist())])
    assert torch.equal(got, turned(k))


@pytest.mark.parametrize("n,top", [(4097, 600), (4200, 513), (4200, 1000), (8190, 1024)])
def test_block_select_of_more_blocks_than_lanes_hold_keys(gpu_lib, n, top):
    """Just above the short lists only some of the lanes have keys, fewer than the blocks that are wanted."""
    _choice(57, [16 * n - 3], (4, 1, 64), top, 1, 2)


def test_two_host_threads_on_one_stream(gpu_lib):
    """Each thread's choice and attention are those that it gets alone."""
    work = []
    for seed, ctx in ((141, [17000, 300]), (142, [16500, 2000])):
        a = synth.custom_attention(seed, 2, 8, 2, 64, ctx, ctx_hi=17000).to(DEV)
        s = aflex.block_summary(a)
        sel = aflex.block_select(a, a.q, s, 40)
        work.append((a, s, sel, aflex.attn_sparse_decode(a, sel)))
    torch.cuda.synchronize()
    wrong = []

    def run(a, s, sel, out):
        for _ in range(200):
            x = aflex.block_select(a, a.q, s, 40)
            y = aflex.attn_sparse_decode(a, sel)
            if not (torch.equal(x, sel) and torch.equal(y, out)):
                wrong.append(1)

    threads = [threading.Thread(target=run, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
        assert not t.is_alive()
    assert not wrong
