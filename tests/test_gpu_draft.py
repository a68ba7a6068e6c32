"""HIP operators of the 8-bit cache and of drafted tokens against the oracle.

Tolerances. Writes: queries as in the bf16 write: three fp32 roundings and one to
bf16. Cached rows are compared for equality with codes made from the formula's fp32
operations, which the plain expression repeats. Attention: out is rounded to bf16,
2^-8 of |out|. Over a bf16 cache a weight enters the product as two bf16 values, the
second rounded to 2^-8 of at most 2^-8 of it: 2^-16 of the weight. Over an 8-bit one
it is p 2^e over a reference of at most the largest p 2^e of the row, rounded to fp16:
2^-11 of it, or half the least step, 2^-25 of the largest: on a code c, 2^-25 max(p
2^e) |c| (`small` sums those). The products and the sum of the weights are fp32 sums
of n terms: at most 2 n 2^-24 of sum p |v|. A score is an fp32 sum of D products, its
scaling and the reference's subtraction 4 more roundings: (D + 4) 2^-24 of sum |q k|
scale; the exponent in the reference, of a magnitude up to E, adds E 2^-24. exp2
(itself off by 2^-22) turns that into as much of the weight, in the numerator and in
the denominator: 2 (D + 4) 2^-24 size + 2 E 2^-24 + 2^-21. Where the reference grows,
what came before is scaled by an exp2 of at most 2^-8: once 2^-22 in the sum and in the
product, the times before by 2^-8 less each: 2^-21. Hence
  |y - r| <= 2^-8 |r| + 1.01 ((w + 2 E 2^-24 + 2^-20 + 2 n 2^-24 + 2 (D + 4) 2^-24 size) sum p |v| + 2^-25 small)
with w = 2^-16 or 2^-11, and E = 16 where a test does not say otherwise.
Whatever is copied or masked is compared for equality.
"""
import threading

import pytest
import torch

from oracle import draft, longctx as lc
from paper_2608_01891_amd import aflex, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F8 = torch.float8_e4m3fn
HEADS = [(8, 2, 64), (64, 8, 128), (5, 5, 64), (28, 4, 128), (48, 3, 128), (3, 1, 128)]


def _rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def _bytes(seed, *shape):
    """Codes without NaN."""
    x = torch.randint(0, 256, shape, dtype=torch.uint8, generator=torch.Generator().manual_seed(seed))
    return torch.where(x & 0x7f == 0x7f, 0x30, x).to(torch.uint8).view(F8)


def _f8(a, seed):
    """An 8-bit cache on the host with a's table: random codes, rows of differing size."""
    c = aflex.F8Cache(a)
    k, ke = draft.encode(_rand(seed, a.num_blocks, a.Hkv, 16, a.D))
    g = torch.Generator().manual_seed(seed)
    size = torch.exp2(torch.randint(-3, 4, (a.num_blocks, a.Hkv, 16, 1), generator=g).float())
    v, ve = draft.encode(_rand(seed + 1, a.num_blocks, a.Hkv, 16, a.D) * size)
    c.k_cache, c.v_cache = k.float().to(F8), v.transpose(2, 3).contiguous().float().to(F8)
    c.kv_exp = torch.stack([ke, ve], 2).to(torch.int8).contiguous()
    return c


def _to(c, device=DEV):
    d = aflex.F8Cache.__new__(aflex.F8Cache)
    d.__dict__.update({k: v.to(device) if isinstance(v, torch.Tensor) else v for k, v in c.__dict__.items()})
    return d


def _dev(a):
    return _to(a) if isinstance(a, aflex.F8Cache) else a.to(DEV)


def _cu(counts):
    return [sum(counts[:i]) for i in range(len(counts) + 1)]


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _same(x, y):
    """Equal bits, NaN of either sign alike."""
    x, y = x.double(), y.double()
    return torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))


# --------------------------------------------------------------------- writes
def _turned(x, angles, inter):
    """The formula, each fp32 operation rounded."""
    if angles is None:
        return x.float()
    x, h = x.float(), angles.shape[-1] // 2
    c, s = angles[:, None, :h], angles[:, None, h:]
    ia, ib = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if inter else (slice(0, h), slice(h, 2 * h))
    y = x.clone()
    y[..., ia], y[..., ib] = x[..., ia] * c - x[..., ib] * s, x[..., ib] * c + x[..., ia] * s
    return y


def _check_write(c, cd, q, out, k, v, cu, angles, inter, rows=None):
    assert torch.equal(out.cpu()[rows] if rows is not None else out.cpu(),
                       (_turned(q, angles, inter).bfloat16())[rows] if rows is not None else
                       _turned(q, angles, inter).bfloat16()), "queries"
    kc, vc, ex = draft.write(c.k_cache, c.v_cache, c.kv_exp, c.block_table, c.context_lens, cu,
                             _turned(k, angles, inter), v)
    assert torch.equal(cd.kv_exp.cpu(), ex), "exponents"
    assert _same(cd.k_cache.cpu(), kc), "keys"
    assert _same(cd.v_cache.cpu(), vc), "values"


def _tokens(seed, T, heads, strided, odd=False):
    Hq, Hkv, D = heads
    x = _rand(seed, T, Hq + 2 * Hkv, D)
    if odd:  # rows of any size, zeros, subnormals, values that are not finite
        g = torch.Generator().manual_seed(seed)
        x = x * torch.exp2(torch.randint(-60, 60, (T, Hq + 2 * Hkv, 1), generator=g).float())
        x[0, Hq:], x[1, Hq:], x[2, Hq:] = 0.0, 1e-39, 3.0e38
        x[3, Hq::2, 5], x[4, Hq::2, D - 1], x[4, Hq::2, 0] = float("nan"), -float("inf"), float("inf")
        x[5, Hq:, 3:] = float("nan")
        x[6, Hq:, :] = 2.0 ** -130
        x[7, Hq:, 0] = 448.0 * 2.0 ** 20
    x = x.bfloat16()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if strided:
        y = x.to(DEV)
        return (q, k, v), (y[:, :Hq], y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:])
    return (q, k, v), tuple(t.contiguous().to(DEV) for t in (q, k, v))


def _filled(a, seed):
    c = aflex.F8Cache(a)
    c.k_cache, c.v_cache = _bytes(seed, *c.k_cache.shape), _bytes(seed + 1, *c.v_cache.shape)
    c.kv_exp = torch.randint(-9, 9, c.kv_exp.shape, generator=torch.Generator().manual_seed(seed)).to(torch.int8)
    return c


def test_every_value_of_a_row(gpu_lib):
    """All finite bf16 magnitudes of a few binades around each row's largest, both signs, K and V."""
    a = synth.custom_attention(1, 1, 1, 1, 128, [4096], ctx_hi=4096)
    c = _filled(a, 3)
    bits = (torch.arange(4096)[:, None] * 8 + torch.arange(128) // 2 % 8 + 0x3000) % 0x7f80
    x = (bits | (torch.arange(128) % 2 << 15)).to(torch.int32)
    x = torch.where(x >= 1 << 15, x - (1 << 16), x).to(torch.int16).view(torch.bfloat16)
    x[:, 0] = (x[:, 1].float().abs() * 300).clamp(max=3e38).bfloat16()
    x, cd = x[:, None], _to(c)
    q = x.clone()
    out = aflex.rope_write_f8(cd, q.to(DEV), x.to(DEV), x.to(DEV), _i32([0, 4096]), None, max_seqlen=4096)
    assert torch.equal(out.cpu(), q)
    kc, vc, ex = draft.write(c.k_cache, c.v_cache, c.kv_exp, c.block_table, c.context_lens, [0, 4096], x, x)
    assert torch.equal(cd.kv_exp.cpu(), ex) and _same(cd.k_cache.cpu(), kc) and _same(cd.v_cache.cpu(), vc)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("rot,inter,strided", [(1.0, False, True), (1.0, True, False), (0.5, False, False),
                                               (0.25, True, True), (0.0, False, True)])
def test_append(gpu_lib, heads, rot, inter, strided):
    ctx = [1, 16, 17, 31, 32, 33, 48, 100, 160, 5]
    a = synth.custom_attention(11, len(ctx), *heads, ctx, ctx_hi=160)
    R = int(rot * heads[2])
    c = _filled(a, 4)
    (q, k, v), dev = _tokens(12, a.B, heads, strided)
    rope = aflex.rope_table(160, R, 1000.0) if R else None
    cd = _to(c)
    out = aflex.rope_append_f8(cd, *dev, None if rope is None else rope.to(DEV), interleaved=inter)
    _check_write(c, cd, q, out, k, v, list(range(a.B + 1)), rope[torch.tensor(ctx) - 1] if R else None, inter)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("rot,inter,strided", [(1.0, False, True), (1.0, True, False), (0.5, True, True),
                                               (0.0, False, False)])
def test_write(gpu_lib, heads, rot, inter, strided):
    counts, past = [1, 16, 17, 0, 33, 5, 64, 2], [0, 0, 15, 9, 3, 11, 32, 14]
    ctx = [n + p for n, p in zip(counts, past)]
    a = synth.custom_attention(21, len(ctx), *heads, ctx, ctx_hi=112)
    R, T, cu = int(rot * heads[2]), sum(counts), _cu(counts)
    c = _filled(a, 5)
    (q, k, v), dev = _tokens(22, T, heads, strided)
    rope = aflex.rope_table(112, R, 1000.0) if R else None
    pos = torch.tensor([p + i for n, p in zip(counts, past) for i in range(n)])
    cd = _to(c)
    out = aflex.rope_write_f8(cd, *dev, _i32(cu), None if rope is None else rope.to(DEV), interleaved=inter)
    _check_write(c, cd, q, out, k, v, cu, rope[pos] if R else None, inter)


@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_any_size(gpu_lib, D):
    """Large and small rows, zeros, subnormals, infinities and NaN; append and write alike."""
    heads = (2, 3, D)
    a = synth.custom_attention(23, 12, *heads, [20 + i for i in range(12)], ctx_hi=48)
    c = _filled(a, 6)
    (q, k, v), dev = _tokens(24, 12, heads, False, odd=True)
    one, two = _to(c), _to(c)
    out = aflex.rope_append_f8(one, *dev, None)
    _check_write(c, one, q, out, k, v, list(range(13)), None, False) if not q.isnan().any() else None
    aflex.rope_write_f8(two, *dev, torch.arange(13, dtype=torch.int32, device=DEV), None, max_seqlen=1)
    assert torch.equal(one.kv_exp, two.kv_exp)
    assert _same(one.k_cache.cpu(), two.k_cache.cpu()) and _same(one.v_cache.cpu(), two.v_cache.cpu())
    b = synth.custom_attention(23, 1, *heads, [12], ctx_hi=48)  # as one prompt
    c = _filled(b, 7)
    three = _to(c)
    aflex.rope_write_f8(three, *dev, _i32([0, 12]), None, max_seqlen=12)
    kc, vc, ex = draft.write(c.k_cache, c.v_cache, c.kv_exp, c.block_table, c.context_lens, [0, 12], k, v)
    assert torch.equal(three.kv_exp.cpu(), ex) and _same(three.k_cache.cpu(), kc) and _same(three.v_cache.cpu(), vc)


def test_write_long_prompt_uses_several_heads_per_wave(gpu_lib):
    heads, counts = (48, 17, 64), [9000, 7007, 1, 0, 310]
    a = synth.custom_attention(25, len(counts), *heads, [n + 5 for n in counts], ctx_hi=9008)
    c = _filled(a, 8)
    T, cu = sum(counts), _cu(counts)
    (q, k, v), dev = _tokens(26, T, heads, True)
    rope = aflex.rope_table(9008, 64)
    cd = _to(c)
    out = aflex.rope_write_f8(cd, *dev, _i32(cu), rope.to(DEV), max_seqlen=9000)
    ang = rope[torch.tensor([5 + i for n in counts for i in range(n)])]
    _check_write(c, cd, q, out, k, v, cu, ang, False)


def test_drafts_take_their_positions(gpu_lib):
    heads, counts = (8, 2, 64), [7, 1, 20]
    a = synth.custom_attention(27, 3, *heads, [30, 1, 41], ctx_hi=48)
    c = _filled(a, 9)
    (q, k, v), dev = _tokens(28, 28, heads, False)
    rope = aflex.rope_table(60, 64)
    pos = torch.randint(0, 60, (28,), generator=torch.Generator().manual_seed(1))
    cd = _to(c)
    out = aflex.rope_write_f8(cd, *dev, _i32(_cu(counts)), rope.to(DEV), positions=pos.int().to(DEV), max_seqlen=20)
    _check_write(c, cd, q, out, k, v, _cu(counts), rope[pos], False)


def test_write_leaves_alone_what_has_no_place(gpu_lib):
    """Contexts that are empty or above the capacity, places before 0, positions outside the table, bad block ids."""
    heads, counts = (8, 2, 128), [3, 4, 5, 6, 20, 7]
    a = synth.custom_attention(29, 6, *heads, [20, 40, 33, 16, 30, 48], ctx_hi=64)
    a.context_lens = torch.tensor([0, -3, 65, 4, 30, 48], dtype=torch.int32)  # capacity 64; 2 tokens before place 0
    a.block_table[4, 0], a.block_table[5, 2] = -1, a.num_blocks
    c = _filled(a, 10)
    T, cu = sum(counts), _cu(counts)
    (q, k, v), dev = _tokens(30, T, heads, False)
    rope = aflex.rope_table(46, 128)
    pos = torch.tensor([max(int(a.context_lens[b]) - n + i, 0) for b, n in enumerate(counts) for i in range(n)])
    fill = torch.full((T, 8, 128), 7.0, dtype=torch.bfloat16)
    cd, out = _to(c), fill.to(DEV)
    aflex.rope_write_f8(cd, *dev, _i32(cu), rope.to(DEV), max_seqlen=20, q_out=out)
    kept = [r for b, n in enumerate(counts) for r in range(cu[b], cu[b + 1])
            if b in (3, 4, 5) and 0 <= int(a.context_lens[b]) - n + r - cu[b] < 46]
    ref = fill.clone()
    ref[kept] = _turned(q, rope[pos.clamp(max=45)], False).bfloat16()[kept]
    assert torch.equal(out.cpu(), ref)
    kt, vt = _turned(k, rope[pos.clamp(max=45)], False), v
    keep = a.block_table.clone()
    a.block_table[5, 2] = -1  # (rows 46 and 47 share that block)
    kc, vc, ex = draft.write(c.k_cache, c.v_cache, c.kv_exp, a.block_table, a.context_lens, cu, kt, vt)
    a.block_table = keep
    assert torch.equal(cd.kv_exp.cpu(), ex) and _same(cd.k_cache.cpu(), kc) and _same(cd.v_cache.cpu(), vc)


# ------------------------------------------------------------------ attention
def _check_attn(got, ref, n, D, what="", exps=16):
    out, mag, size, small = ref
    w = 2.0 ** -11 if small.any() else 2.0 ** -16  # an 8-bit cache, or bf16
    most = 1.01 * ((w + 2 * exps * 2.0 ** -24 + 2.0 ** -20 + 2 * n * 2.0 ** -24 + 2 * (D + 4) * 2.0 ** -24 * size[..., None]) * mag
                   + 2.0 ** -25 * small)
    err = (got.cpu().double() - out).abs()
    bad = ~(err <= 2.0 ** -8 * out.abs() + most)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} values, first at {bad.nonzero()[0].tolist()}"


def _random_masks(seed, counts):
    """Rows of any bits: none, all, one, and random ones."""
    g = torch.Generator().manual_seed(seed)
    m = torch.randint(-(1 << 62), 1 << 62, (sum(counts),), generator=g) * 2 + torch.randint(0, 2, (sum(counts),), generator=g)
    m[::7], m[3::7], m[5::7] = 0, -1, 1
    return m


def _trees(seed, counts):
    g = torch.Generator().manual_seed(seed)
    return aflex.tree_masks([[int(torch.randint(-1, max(i, 1), (1,), generator=g)) if i else -1 for i in range(n)]
                             for n in counts])


def _tree(a, counts, seed, masks, scale=0.0, q=None, max_drafts=None, out=None):
    T, cu = sum(counts), _cu(counts)
    q = _rand(seed, T, a.Hq, a.D).bfloat16() if q is None else q
    got = aflex.attn_tree(_dev(a), q.to(DEV), _i32(cu), None if masks is None else masks.to(DEV), max_drafts=max_drafts,
                          scale=scale, out=out)
    ref = draft.attention_tree(q, a.k_cache, a.v_cache, getattr(a, "kv_exp", None), a.block_table, a.context_lens, cu,
                               masks, scale)
    return got, ref


def _cache(seed, heads, ctx, f8, ctx_hi=None):
    a = synth.custom_attention(seed, len(ctx), *heads, ctx, ctx_hi=ctx_hi)
    return _f8(a, seed) if f8 else a


@pytest.mark.parametrize("heads", HEADS + [(16, 1, 64), (32, 2, 128), (7, 7, 128)])
def test_decode_f8(gpu_lib, heads):
    ctx = [1, 15, 16, 17, 63, 64, 65, 0, 129, 700, 1024, 333]
    c = _cache(31, heads, ctx, True)
    q = _rand(32, len(ctx), heads[0], heads[2]).bfloat16()
    got = aflex.attn_decode_f8(_to(c), q.to(DEV))
    ref = draft.attention_tree(q, c.k_cache, c.v_cache, c.kv_exp, c.block_table, c.context_lens,
                               list(range(len(ctx) + 1)))
    _check_attn(got, ref, 1024, heads[2])
    assert not got[7].any()


@pytest.mark.parametrize("heads,ctx", [((8, 1, 64), [40000]), ((16, 2, 128), [9000, 31, 20000, 4097]),
                                       ((4, 4, 128), [300 + 7 * i for i in range(150)])])
def test_decode_f8_splits_long_contexts(gpu_lib, heads, ctx):
    c = _cache(33, heads, ctx, True)
    q = _rand(34, len(ctx), heads[0], heads[2]).bfloat16()
    got = aflex.attn_decode_f8(_to(c), q.to(DEV))
    ref = draft.attention_tree(q, c.k_cache, c.v_cache, c.kv_exp, c.block_table, c.context_lens,
                               list(range(len(ctx) + 1)))
    _check_attn(got, ref, max(ctx), heads[2])
    assert torch.equal(got, aflex.attn_decode_f8(_to(c), q.to(DEV)))


COUNTS = [1, 5, 0, 2, 9, 4, 3, 1, 7]
CONTEXTS = [1, 5, 33, 40, 16, 700, 129, 64, 7]  # with and without tokens before the drafts


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("heads", HEADS + [(16, 1, 64), (32, 2, 128)])
@pytest.mark.parametrize("kind", ["chain", "tree", "any"])
def test_tree(gpu_lib, heads, f8, kind):
    a = _cache(41, heads, CONTEXTS, f8)
    masks = {"chain": None, "tree": _trees(42, COUNTS), "any": _random_masks(43, COUNTS)}[kind]
    got, ref = _tree(a, COUNTS, 44, masks)
    _check_attn(got, ref, 700, heads[2])
    assert torch.equal(got.cpu()[ref[1].sum(-1) == 0].double(), ref[0][ref[1].sum(-1) == 0])  # rows that see nothing


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("heads", [(8, 8, 64), (64, 8, 128), (28, 4, 128), (16, 1, 64), (15, 3, 128)])
@pytest.mark.parametrize("most", [2, 3, 4, 8, 11, 16, 33, 64])
def test_tree_of_many_drafts(gpu_lib, heads, f8, most):
    """Every number of row tiles per wave, waves that share a step, and rows that take several passes."""
    counts = [most, max(most // 2, 1), 1, most]
    a = _cache(45, heads, [most + 300, 200 + most, 1, most], f8)
    got, ref = _tree(a, counts, 46, _trees(47, counts) if most % 2 else _random_masks(48, counts))
    _check_attn(got, ref, 400, heads[2])


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("heads,most", [((8, 1, 128), 2), ((8, 2, 64), 12), ((16, 2, 128), 20)])
def test_tree_splits_long_contexts(gpu_lib, heads, f8, most):
    a = _cache(49, heads, [12001, 40, 7000 + most], f8)
    counts = [most, most // 2, most]
    got, ref = _tree(a, counts, 50, _trees(51, counts))
    _check_attn(got, ref, 12001, heads[2])
    again, _ = _tree(a, counts, 50, _trees(51, counts))
    assert torch.equal(got, again)


@pytest.mark.parametrize("f8", [False, True])
def test_tree_of_many_sequences(gpu_lib, f8):
    """More units than work-groups, pieces of several units each."""
    counts = [i % 4 for i in range(300)]
    a = _cache(52, (8, 4, 64), [(37 * i) % 150 + 4 for i in range(300)], f8)
    got, ref = _tree(a, counts, 53, None)
    _check_attn(got, ref, 160, 64)


def test_decode_f8_is_a_tree_of_one(gpu_lib):
    ctx = [100, 1, 3000, 17]
    c = _cache(54, (32, 8, 128), ctx, True)
    q = _rand(55, 4, 32, 128).bfloat16().to(DEV)
    one = aflex.attn_decode_f8(_to(c), q)
    two = aflex.attn_tree(_to(c), q, torch.arange(5, dtype=torch.int32, device=DEV), max_drafts=1)
    assert torch.equal(one, two)


@pytest.mark.parametrize("f8", [False, True])
def test_masked_places_do_not_matter(gpu_lib, f8):
    """NaN and infinities behind the context, in blocks that nobody owns, and in drafts that a row does not see."""
    counts, ctx = [6, 3], [39, 20]
    a = _cache(56, (8, 2, 128), ctx, f8)
    masks = _trees(57, counts) | 1
    masks[:6] &= ~(1 << 4)  # nobody sees draft 4 of the first sequence
    clean, ref = _tree(a, counts, 58, masks)
    _check_attn(clean, ref, 39, 128)
    b = _cache(56, (8, 2, 128), ctx, f8)
    nan = torch.tensor(0x7f, dtype=torch.uint8).view(F8) if f8 else torch.tensor(float("nan"), dtype=torch.bfloat16)
    kb = b.k_cache.view(torch.uint8) if f8 else b.k_cache
    vb = b.v_cache.view(torch.uint8) if f8 else b.v_cache
    nan = nan.view(torch.uint8) if f8 else nan
    for s, end in ((0, 39), (1, 20)):
        blk = int(b.block_table[s, (end - 1) // 16])
        kb[blk, :, end % 16:] = nan  # behind the context
        vb[blk, :, :, end % 16:] = nan
        if f8:
            b.kv_exp[blk, :, :, end % 16:] = torch.tensor([[127], [-128]], dtype=torch.int8)
    blk, o = int(b.block_table[0, 37 // 16]), 37 % 16  # draft 4 sits at place 33 + 4
    kb[blk, :, o] = nan
    got, _ = _tree(b, counts, 58, masks)
    assert torch.equal(got, clean)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("heads,ctx", [((2, 1, 64), 90), ((4, 1, 128), 90), ((8, 1, 64), 200), ((8, 1, 128), 6000),
                                       ((14, 1, 128), 200), ((16, 1, 64), 6000), ((12, 3, 128), 2500)])
@pytest.mark.parametrize("chain", [False, True])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(gpu_lib, heads, ctx, f8, chain):
    """Infinities and NaN in the values of drafts, and of tokens beside a block that does not exist."""
    Hq, Hkv, D = heads
    counts, lens = [6, 3], [ctx, 35]
    a, b = (_cache(105, heads, lens, f8, ctx_hi=ctx + 40) for _ in range(2))
    masks = None if chain else _trees(106, counts) & ~(1 << 4) | 1
    bad = [0, 2, 4]  # drafts of the first sequence
    full = torch.tensor([(2 << i) - 1 for n in counts for i in range(n)]) if chain else masks
    for c in (a, b):
        c.block_table[0, 1] = -1
        kv = (c.k_cache.view(torch.uint8), c.v_cache.view(torch.uint8)) if f8 else (c.k_cache, c.v_cache)
        for place in [lens[0] - 6 + j for j in bad] + [3]:
            blk, o = int(c.block_table[0, place // 16]), place % 16
            if f8:
                kv[1][blk, :, 5:9, o] = 0x7f if c is b else 0
            else:
                kv[1][blk, :, 5:9, o] = 0.0
                if c is b:
                    kv[1][blk, :, 5, o] = float("inf")
                    kv[1][blk, :, 6, o] = float("inf") if place % 2 else float("-inf")
                    kv[1][blk, :, 7, o] = float("nan")
    seen = torch.tensor([[bool(int(m) >> j & 1) for j in bad] for m in full[:6]])
    assert bool(seen.any(-1).all())  # (draft 0 is seen by all; place 3 too)
    q = _rand(107, 9, Hq, D).bfloat16()
    clean, _ = _tree(a, counts, 0, masks, q=q)
    got, ref = _tree(b, counts, 0, masks, q=q)
    keep = [d for d in range(D) if not 5 <= d < 9]
    assert torch.equal(got[:, :, keep], clean[:, :, keep]) and torch.equal(got[6:], clean[6:])
    assert torch.equal(got[:6, :, 8], clean[:6, :, 8]) or f8
    assert _same(got.cpu()[:6, :, 5:8], ref[0][:6, :, 5:8])
    # without the tokens that all rows see: rows that see no such draft are as if there were none
    for c in (a, b):
        kv = (c.k_cache.view(torch.uint8), c.v_cache.view(torch.uint8)) if f8 else (c.k_cache, c.v_cache)
        for place in (lens[0] - 6, 3):
            kv[1][int(c.block_table[0, place // 16]), :, 5:9, place % 16] = 0
    clean, _ = _tree(a, counts, 0, masks, q=q)
    got, ref = _tree(b, counts, 0, masks, q=q)
    none = ~seen[:, 1:].any(-1)
    assert bool(none.any()) and torch.equal(got[:6][none.to(DEV)], clean[:6][none.to(DEV)])
    assert _same(got.cpu()[:6, :, 5:8][~none], ref[0][:6, :, 5:8][~none])


@pytest.mark.parametrize("heads,counts", [((8, 2, 64), [1, 1, 1]), ((16, 1, 128), [1, 1, 1]), ((8, 2, 128), [5, 16, 7]),
                                          ((16, 2, 64), [7, 3, 16])])
@pytest.mark.parametrize("order", ["mixed", "small first", "large first"])
def test_values_of_any_size(gpu_lib, heads, counts, order):
    """Value rows of 2^-100 and zero beside ones of 2^60: the weights and their sum span more than a float does."""
    lens = [700, 40, 6000]
    c = _cache(108, heads, lens, True)
    e = c.kv_exp[:, :, 1]
    g = torch.Generator().manual_seed(109)
    e.copy_(torch.randint(-100, 61, e.shape, generator=g))
    if order != "mixed":  # by the place in the context
        for s, n in enumerate(lens):
            for j in range(-(-n // 16)):
                late = j >= (n // 16) // 2
                e[int(c.block_table[s, j])] = 60 if late == (order == "small first") else -100
    zero = torch.randint(0, 3, e.shape, generator=g) == 0
    c.v_cache.view(torch.uint8).masked_fill_(zero[:, :, None, :], 0)
    e.masked_fill_(zero, -100)
    got, ref = _tree(c, counts, 110, None)
    _check_attn(got, ref, 6000, heads[2], exps=128)
    e.masked_fill_(e > -60, -100)  # nothing but tiny rows
    c.v_cache.view(torch.uint8).masked_fill_((e == -100)[:, :, None, :], 0x34)
    got, ref = _tree(c, counts, 110, None)
    _check_attn(got, ref, 6000, heads[2], exps=128)


# A group of heads for each of the kernels that six drafts of an 8-bit cache take.
KERNELS = [(2, 1, 64), (4, 1, 128), (8, 1, 64), (8, 1, 128), (14, 1, 128)]


@pytest.mark.parametrize("heads", KERNELS)
@pytest.mark.parametrize("ctx", [6, 39, 6001])
@pytest.mark.parametrize("exp", [127, 121, -101, -128])
def test_exponents_of_drafts_that_nobody_sees(gpu_lib, heads, ctx, exp):
    """Whatever a cached draft holds that no row sees, rows that see nothing among them."""
    counts, lens = [6, 3], [ctx, 20]
    a, b = (_cache(113, heads, lens, True) for _ in range(2))
    masks = _trees(114, counts) & ~(1 << 4) | 1  # nobody sees draft 4
    masks[1] = 0
    place = ctx - 2
    blk, o = int(b.block_table[0, place // 16]), place % 16
    b.kv_exp[blk, :, :, o] = exp
    b.k_cache.view(torch.uint8)[blk, :, o] = 0x7f
    b.v_cache.view(torch.uint8)[blk, :, :, o] = torch.tensor([0x7f, 0x7e, 0xfe, 0x00] * (heads[2] // 4), dtype=torch.uint8)
    clean, ref = _tree(a, counts, 115, masks)
    _check_attn(clean, ref, ctx, heads[2])
    got, _ = _tree(b, counts, 115, masks)
    assert torch.equal(got, clean)


def _peak(heads, ctx, above, big, seed, exps=None):
    """A cache whose token 0 lies `above` (log2) over the others of each sequence, which are all alike in their
    scores, with the queries and the scale for it; token 0's values are zero but for channel 0."""
    c = _cache(seed, heads, [ctx, 40], True)
    for t in (c.k_cache, c.v_cache):
        t.view(torch.uint8).fill_(0)
    c.kv_exp.zero_()
    if exps is not None:
        c.kv_exp[:, :, 1] = exps
    c.v_cache.view(torch.uint8).fill_(big)
    for b in range(2):
        blk = int(c.block_table[b, 0])
        c.k_cache.view(torch.uint8)[blk, :, 0, 0] = 0x38  # 1
        c.v_cache.view(torch.uint8)[blk, :, 1:, 0] = 0
    q = torch.zeros(9, heads[0], heads[2], dtype=torch.bfloat16)
    q[:, :, 0] = 1.0
    return c, q, above * 0.6931471805599453


@pytest.mark.parametrize("heads", KERNELS)
@pytest.mark.parametrize("exp", [104, 112, 120])
@pytest.mark.parametrize("kind", ["flat", "peak", "beside -100"])
def test_values_of_the_largest_exponents(gpu_lib, heads, exp, kind):
    """Value rows of up to 2^120: many light tokens hold much of the weight."""
    lens, counts = [6001, 40], [6, 3]
    if kind == "peak":
        c, q, scale = _peak(heads, 6001, 18.3, 0x38, 117, exp)
    else:
        c, q, scale = _cache(117, heads, lens, True), None, 0.0
        e = c.kv_exp[:, :, 1]
        e.fill_(exp)
        codes = c.v_cache.view(torch.uint8)
        codes.copy_(torch.where(codes & 0x7f > 0x38, 0x34, codes).to(torch.uint8))  # (what they stand for is finite)
        if kind == "beside -100":
            e.masked_fill_(torch.randint(0, 2, e.shape, generator=torch.Generator().manual_seed(118)) == 0, -100)
    got, ref = _tree(c, counts, 119, None, q=q, scale=scale)
    assert bool(got.isfinite().all())
    _check_attn(got, ref, 6001, heads[2], exps=128)


@pytest.mark.parametrize("heads", KERNELS)
@pytest.mark.parametrize("ctx,above", [(100, 16.4), (300, 24.45), (6001, 25.5)])
def test_small_weights_beside_a_large_one(gpu_lib, heads, ctx, above):
    """Channels in which the token that takes nearly all of the weight holds 0. An fp16 weight's least step is 2^-24
    beside a largest weight of 2^7 or more: 2^-32 of the largest p 2^e on a code (`small`), not the 2^-25 above."""
    c, q, scale = _peak(heads, ctx, above, 0x38, 116)
    for counts in ([6, 3], [1, 1]):
        got, (out, mag, size, small) = _tree(c, counts, 0, None, scale=scale, q=q[:sum(counts)])
        _check_attn(got, (out, mag, size, small * 2.0 ** -7), ctx, heads[2])


@pytest.mark.parametrize("heads", [(8, 8, 64), (16, 1, 64), (12, 2, 128), (16, 1, 128)])
def test_weights_of_up_to_16_rows_have_two_parts(gpu_lib, heads):
    """Opposite values whose weights nearly cancel: with up to 16 rows a kv head a weight is two fp16 values, the second
    rounded to 2^-11 of at most 2^-11 of it, so the bound of a bf16 cache's two holds (no `small`, w = 2^-16)."""
    lens = [2, 2, 2, 3, 40, 2]
    c = _cache(127, heads, lens, True)
    codes = c.v_cache.view(torch.uint8)
    codes[..., 1::2] = codes[..., 0::2] ^ 0x80
    c.kv_exp[:, :, 1] = 0
    both = min(16 // (heads[0] // heads[1]), 2)  # drafts
    for counts, most in (([1] * 6, 1), ([1, both] * 3, None)):
        got, (out, mag, size, small) = _tree(c, counts, 128, None, scale=0.01, max_drafts=most)
        _check_attn(got, (out, mag, size, torch.zeros_like(small)), 40, heads[2])
    q = _rand(129, 6, heads[0], heads[2]).bfloat16()
    got = aflex.attn_decode_f8(_to(c), q.to(DEV), scale=0.01)
    out, mag, size, small = draft.attention_tree(q, c.k_cache, c.v_cache, c.kv_exp, c.block_table, c.context_lens,
                                                 list(range(7)), None, 0.01)
    _check_attn(got, (out, mag, size, torch.zeros_like(small)), 40, heads[2])


@pytest.mark.parametrize("heads,most", [((8, 2, 64), 2), ((16, 2, 128), 6), ((12, 1, 128), 11)])
@pytest.mark.parametrize("ctx", [100, 6001])
def test_large_values_over_a_bf16_cache(gpu_lib, heads, most, ctx):
    """Values of the largest magnitudes: a sum of them with its weights stays within floats where their mean does.
    (And small ones keep their bits.)"""
    a = _cache(120, heads, [ctx, 40], False)
    size = torch.rand(a.v_cache.shape, generator=torch.Generator().manual_seed(121)) * 0.5 + 0.25
    size[:, :, 1::2] *= -1
    for exp, scale in ((127, 0.0), (127, 1e-6), (-105, 0.0)):
        a.v_cache = (size * 2.0 ** exp).bfloat16()
        got, ref = _tree(a, [most, 1], 122, None, scale=scale)
        assert bool(got.isfinite().all())
        _check_attn(got, ref, ctx, heads[2])


@pytest.mark.parametrize("heads,most", [((8, 2, 64), 2), ((16, 2, 128), 6), ((12, 1, 128), 11)])
@pytest.mark.parametrize("ctx", [200, 6001])
def test_infinities_that_every_row_sees(gpu_lib, heads, most, ctx):
    """p times an infinity is that infinity, whichever parts p has, as over the cache's other attention calls."""
    a = _cache(123, heads, [ctx, 40], False)
    clean, _ = _tree(a, [most, 1], 124, None)
    inf = float("inf")
    for place, at in [(3, {5: inf, 6: inf, 7: -inf}), (77, {6: -inf, 8: inf}), (78, {8: inf, 9: float("nan")})]:
        blk = int(a.block_table[0, place // 16])
        for d, v in at.items():
            a.v_cache[blk, :, d, place % 16] = v
    got, ref = _tree(a, [most, 1], 124, None)
    assert _same(got.cpu()[:most, :, 5:10], ref[0][:most, :, 5:10])
    rest = [d for d in range(heads[2]) if not 5 <= d < 10]
    assert torch.equal(got[:, :, rest], clean[:, :, rest]) and torch.equal(got[most:], clean[most:])
    # a NaN among one kv head's scores: its rows are NaN, infinite values or not
    a.k_cache[int(a.block_table[0, 5]), -1, 9, 1] = float("nan")
    again, _ = _tree(a, [most, 1], 124, None)
    G = heads[0] // heads[1]
    assert bool(again[:most, -G:].isnan().all())
    assert _same(again[:most, :-G].cpu(), got[:most, :-G].cpu()) and torch.equal(again[most:], clean[most:])


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("heads,most", [((8, 8, 64), 1), ((64, 8, 128), 2), ((64, 8, 128), 6), ((32, 4, 64), 16)])
def test_units_that_share_work_groups(gpu_lib, f8, heads, most):
    """Contexts of a large bound: several units a work-group, and units cut between two of them."""
    counts = [1 + i % most for i in range(40)]
    a = _cache(111, heads, [(613 * i) % 900 + most for i in range(40)], f8, ctx_hi=6400)
    got, ref = _tree(a, counts, 112, None)
    _check_attn(got, ref, 920, heads[2])


@pytest.mark.parametrize("f8", [False, True])
def test_a_nan_that_is_seen_shows(gpu_lib, f8):
    a = _cache(59, (4, 2, 64), [40, 40], f8)
    blk = int(a.block_table[0, 0])
    if f8:
        a.k_cache.view(torch.uint8)[blk, 1, 3, 9] = 0x7f
    else:
        a.k_cache[blk, 1, 3, 9] = float("nan")
    got, _ = _tree(a, [2, 2], 60, None)
    got = got.isnan().all(-1).cpu()
    assert got.tolist() == [[False, False, True, True]] * 2 + [[False] * 4] * 2


@pytest.mark.parametrize("f8", [False, True])
def test_bad_block_ids_and_bounds(gpu_lib, f8):
    """Tokens of ids outside the pool are masked; contexts are cut to the host's bound; rows beyond max_drafts stay."""
    counts = [3, 4, 2, 3]
    a = _cache(61, (8, 2, 64), [100, 60, 90, 50], f8, ctx_hi=112)
    a.block_table[0, 2], a.block_table[1, 0], a.block_table[2, :] = -1, a.num_blocks, 1 << 30
    got, ref = _tree(a, counts, 62, None)
    _check_attn(got, ref, 100, 64)
    assert not got[7:9].any()
    a = _cache(63, (8, 2, 64), [100, 60, 90, 50], f8, ctx_hi=112)
    a.max_context_len = 70
    a.context_lens = torch.tensor([100, 60, -5, 50], dtype=torch.int32)
    q = _rand(64, 12, 8, 64).bfloat16()
    out = torch.full((12, 8, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    _tree(a, counts, 64, None, q=q, max_drafts=3, out=out)
    cut = a.context_lens.clamp(max=70)
    ref = draft.attention_tree(q, a.k_cache, a.v_cache, getattr(a, "kv_exp", None), a.block_table, cut, _cu(counts))
    rows = [r for r in range(12) if r != 6]
    _check_attn(out[rows], tuple(x[rows] for x in ref), 70, 64)
    assert bool((out[6] == 3.0).all()) and not out[7:9].any()


def test_scale_and_large_scores(gpu_lib):
    c = _cache(65, (8, 2, 128), [200, 50], True)
    for scale in (0.5, 1e-3):
        got, ref = _tree(c, [2, 3], 66, None, scale=scale)
        _check_attn(got, ref, 200, 128, f"scale {scale}")
    q = (_rand(67, 5, 8, 128) * 40).bfloat16()  # one token takes nearly all of the weight
    got, ref = _tree(c, [2, 3], 68, None, q=q)
    _check_attn(got, ref, 200, 128, "large")


def test_offsets_beyond_32_bits(gpu_lib):
    """Pools of more than 2^32 bytes: the blocks of a short context at their far end."""
    Hkv, D, n = 8, 128, 270000
    a = synth.custom_attention(69, 1, 16, Hkv, D, [100], ctx_hi=112)
    c = _f8(a, 70)
    far = _to(c)
    far.num_blocks = n
    far.k_cache = torch.zeros(n, Hkv, 16, D, dtype=torch.uint8, device=DEV).view(F8)
    far.v_cache = torch.zeros(n, Hkv, D, 16, dtype=torch.uint8, device=DEV).view(F8)
    far.kv_exp = torch.zeros(n, Hkv, 2, 16, dtype=torch.int8, device=DEV)
    assert far.k_cache.numel() > 1 << 32
    (q, k, v), dev = _tokens(71, 100, (16, Hkv, D), True)
    far.block_table = (n - 1 - torch.arange(7, dtype=torch.int32)).view(1, 7).to(DEV)
    near = aflex.F8Cache(a)
    near = _to(near)
    rope, cu = aflex.rope_table(112, D).to(DEV), _i32([0, 100])
    x = aflex.rope_write_f8(far, *dev, cu, rope, max_seqlen=100)
    y = aflex.rope_write_f8(near, *dev, cu, rope, max_seqlen=100)
    assert torch.equal(x, y)
    last = _i32([0, 4])
    one = aflex.attn_tree(far, x[96:], last, max_drafts=4)
    assert torch.equal(one, aflex.attn_tree(near, x[96:], last, max_drafts=4)) and bool(one.any())
    acc, cnt = _i32([[1, 3]]), _i32([2])
    assert torch.equal(aflex.cache_accept(far, last, acc, cnt), aflex.cache_accept(near, last, acc, cnt))
    assert torch.equal(aflex.attn_decode_f8(far, x[:1]), aflex.attn_decode_f8(near, x[:1]))


# --------------------------------------------------------------------- accept
@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("heads", [(8, 2, 64), (64, 8, 128), (5, 5, 64), (3, 1, 128)])
def test_accept(gpu_lib, heads, f8):
    counts = [7, 64, 1, 0, 20, 5, 9, 33, 6, 4, 3]
    ctx = [30, 64, 17, 10, 37, 21, 40, 65, 3, 70, 0]
    a = _cache(81, heads, [min(max(c, 1), 64) for c in ctx], f8, ctx_hi=64)
    a.context_lens = torch.tensor(ctx, dtype=torch.int32)
    a.context_lens[7], a.context_lens[9] = 65, 5  # above the capacity, with bad blocks
    a.block_table[6, 2] = -1
    g = torch.Generator().manual_seed(1)
    acc = torch.full((11, 64), -1, dtype=torch.int32)
    cnt = torch.zeros(11, dtype=torch.int32)
    for b, n in enumerate(counts):
        took = sorted(torch.randperm(n, generator=g)[:(n + 1) // 2].tolist())
        acc[b, :len(took)], cnt[b] = torch.tensor(took, dtype=torch.int32), len(took)
    acc[1, :64], cnt[1] = torch.arange(64), 64       # all of them: nothing moves
    acc[4, 3], cnt[4] = acc[4, 2], 8                 # does not ascend: stops there
    acc[5, 1], cnt[5] = 5, 3                         # no such draft
    cnt[6] = 99
    d = _dev(a)
    before = {k: getattr(d, k).clone() for k in ("context_lens", "block_table")}
    new = aflex.cache_accept(d, _i32(_cu(counts)), acc.to(DEV), cnt.to(DEV))
    kc, vc, ex, ctx_new = draft.accept(a.k_cache.view(torch.uint8) if f8 else a.k_cache,
                                       a.v_cache.view(torch.uint8) if f8 else a.v_cache, getattr(a, "kv_exp", None),
                                       a.block_table, a.context_lens, _cu(counts), acc, cnt)
    assert torch.equal(new.cpu(), ctx_new)
    assert torch.equal(d.k_cache.cpu().view(kc.dtype), kc) and torch.equal(d.v_cache.cpu().view(vc.dtype), vc)
    assert ex is None or torch.equal(d.kv_exp.cpu(), ex)
    assert all(torch.equal(getattr(d, k), v) for k, v in before.items())


# ------------------------------------------------------- a run of them together
@pytest.mark.parametrize("f8", [False, True])
def test_prompt_drafts_accept_and_decode(gpu_lib, f8):
    """A prompt, a tree of drafts, the accepted ones, the next token: as if the accepted tokens had come one by one."""
    heads = Hq, Hkv, D = 16, 2, 128
    lens, counts = [45, 16, 100], [6, 3, 9]
    parents = [[-1, 0, 0, 1, 3, -1], [-1, 0, 1], [-1, -1, 1, 1, 2, 4, 5, 0, 7]]
    paths = [[0, 1, 3], [0, 1, 2], [1, 2, 4, 5]]
    a = synth.custom_attention(91, 3, *heads, lens, ctx_hi=128)
    a.block_table = torch.arange(24, dtype=torch.int32).view(3, 8)
    a.num_blocks = 24
    a.k_cache, a.v_cache = _rand(92, 24, Hkv, 16, D).bfloat16(), _rand(93, 24, Hkv, D, 16).bfloat16()
    rope = aflex.rope_table(128, D)
    c = _to(aflex.F8Cache(a)) if f8 else a.to(DEV)
    write = aflex.rope_write_f8 if f8 else aflex.rope_write
    (pq, pk, pv), dev = _tokens(94, sum(lens), heads, True)
    write(c, *dev, _i32(_cu(lens)), rope.to(DEV), max_seqlen=100)
    ref = aflex.F8Cache(a)  # the same rows on the host, one sequence of writes
    T, cu = sum(counts), _cu(counts)
    (q, k, v), dev = _tokens(95, T, heads, False)
    c.context_lens = _i32([n + m for n, m in zip(lens, counts)])
    depth = [0] * T
    for b in range(3):
        for i, p in enumerate(parents[b]):
            depth[cu[b] + i] = depth[cu[b] + p] + 1 if p >= 0 else lens[b]
    qr = write(c, *dev, _i32(cu), rope.to(DEV), positions=_i32(depth), max_seqlen=9)
    masks = aflex.tree_masks(parents)
    out = aflex.attn_tree(c, qr, _i32(cu), masks.to(DEV), max_drafts=9)
    acc = torch.full((3, 5), -1, dtype=torch.int32)
    for b, p in enumerate(paths):
        acc[b, :len(p)] = torch.tensor(p)
    new = aflex.cache_accept(c, _i32(cu), acc.to(DEV), _i32([len(p) for p in paths]))
    assert new.cpu().tolist() == [48, 19, 104]
    c.context_lens = new + 1
    (q1, k1, v1), dev1 = _tokens(96, 3, heads, True)
    if f8:
        last = aflex.attn_decode_f8(c, aflex.rope_append_f8(c, *dev1, rope.to(DEV)))
    else:
        a_out = aflex.rope_append(c, *dev1, rope.to(DEV))
        c.q = a_out
        last = aflex.attn_decode(c)
    # the oracle: prompt, then the path's tokens, then the last one, as rows of one context
    ang = lambda pos: rope[torch.tensor(pos)]  # noqa: E731
    for b in range(3):
        rows = [cu[b] + i for i in paths[b]]
        p0, n = _cu(lens)[b], lens[b] + len(paths[b]) + 1
        kk = torch.cat([pk[p0:p0 + lens[b]], k[rows], k1[b:b + 1]])
        vv = torch.cat([pv[p0:p0 + lens[b]], v[rows], v1[b:b + 1]])
        kk = _turned(kk, ang(range(n)), False)
        table, ctx = torch.arange(8)[None], torch.tensor([n])
        if f8:
            z = torch.zeros(8, Hkv, 16, D), torch.zeros(8, Hkv, D, 16), torch.zeros(8, Hkv, 2, 16, dtype=torch.int8)
            kc, vc, ex = draft.write(*z, table, ctx, [0, n], kk, vv)
        else:
            kc, vc, ex = torch.zeros(8, Hkv, 16, D), torch.zeros(8, Hkv, D, 16), None
            i = torch.arange(n)
            kc[i // 16, :, i % 16], vc[i // 16, :, :, i % 16] = kk.bfloat16().float(), vv.float()
        qq = torch.cat([q[rows], q1[b:b + 1]])
        qq = _turned(qq, ang(range(lens[b], n)), False).bfloat16()
        want = draft.attention_tree(qq, kc, vc, ex, table, ctx, [0, len(rows) + 1])
        _check_attn(out[rows], tuple(x[:-1] for x in want), n, D, f"drafts of sequence {b}")
        if f8:  # (the bf16 decode attention has tolerances of its own)
            _check_attn(last[b:b + 1], tuple(x[-1:] for x in want), n, D, f"token of sequence {b}")
        else:
            assert bool(((last[b].cpu().double() - want[0][-1]).abs() <= 3 * 2.0 ** -8 * want[1][-1] + 1e-6).all())


def test_summaries_after_accepted_drafts(gpu_lib):
    """Drafts and their move leave no summaries; block_summary over the new lengths makes those of every full block,
    as the next choice of blocks needs them."""
    heads = Hq, Hkv, D = 16, 2, 128
    lens, counts = [45, 30, 100], [6, 20, 9]
    a = synth.custom_attention(130, 3, *heads, lens, ctx_hi=128)
    a.block_table = torch.arange(24, dtype=torch.int32).view(3, 8)
    a.num_blocks = 24
    a.k_cache, a.v_cache = torch.zeros(24, Hkv, 16, D).bfloat16(), torch.zeros(24, Hkv, D, 16).bfloat16()
    c, rope = a.to(DEV), aflex.rope_table(128, D).to(DEV)
    s = aflex.BlockSummary.of(c)
    (_, dev) = _tokens(131, sum(lens), heads, False)
    aflex.rope_write(c, *dev, _i32(_cu(lens)), rope, max_seqlen=100, summary=s)
    c.context_lens = _i32([n + m for n, m in zip(lens, counts)])
    (_, dev), cu = _tokens(132, sum(counts), heads, False), _i32(_cu(counts))
    aflex.rope_write(c, *dev, cu, rope, max_seqlen=20)
    acc = torch.full((3, 20), -1, dtype=torch.int32)
    for b, path in enumerate([[0, 2, 5], list(range(1, 20)), [0, 1, 2, 3, 4, 5, 6, 7, 8]]):
        acc[b, :len(path)] = torch.tensor(path)
    c.context_lens = aflex.cache_accept(c, cu, acc.to(DEV), _i32([3, 19, 9]))
    assert c.context_lens.tolist() == [48, 49, 109]
    aflex.block_summary(c, s)
    zero = aflex.BlockSummary.of(a)
    keys, exp = lc.block_summary(c.k_cache.cpu(), a.block_table, c.context_lens.cpu(), zero.keys, zero.exp)
    full = [int(a.block_table[b, j]) for b, n in enumerate((48, 49, 109)) for j in range(n // 16)]
    assert len(full) == 12
    assert torch.equal(s.keys.cpu()[full], keys[full]) and torch.equal(s.exp.cpu()[full], exp[full])


@pytest.mark.parametrize("f8", [False, True])
def test_captured_steps_replay(gpu_lib, f8):
    """Two graphs of a step each and eager calls between their replays; each graph has its own workspace."""
    heads, counts = (16, 2, 128), [5, 3, 8]
    a = _cache(97, heads, [3000, 40, 900], f8)
    d = [_dev(a), _dev(a)]
    cu, acc, cnt = _i32(_cu(counts)), _i32([[0, 2], [1, -1], [3, 7]]), _i32([2, 1, 2])
    q = [_rand(98 + i, 16, 16, 128).bfloat16().to(DEV) for i in range(2)]
    masks = _trees(99, counts).to(DEV)
    outs = [torch.empty_like(q[0]) for _ in range(2)]
    ctxs = [torch.empty(3, dtype=torch.int32, device=DEV) for _ in range(2)]
    ref = [aflex.attn_tree(d[i], q[i], cu, masks, max_drafts=8).clone() for i in range(2)]
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            aflex.attn_tree(d[i], q[i], cu, masks, max_drafts=8, out=outs[i])
            aflex.cache_accept(d[i], cu, acc, cnt, context_out=ctxs[i])
        graphs.append(g)
    names = ["k_cache", "v_cache"] + ["kv_exp"] * f8  # (all that the move changes)
    pools = [{k: getattr(x, k).clone() for k in names} for x in d]
    for _ in range(3):
        for i in range(2):
            for k in names:
                getattr(d[i], k).copy_(pools[i][k])
            outs[i].zero_()
        graphs[0].replay()
        graphs[1].replay()
        eager = aflex.attn_tree(_dev(a), q[0], cu, masks, max_drafts=8)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], ref[0]) and torch.equal(outs[1], ref[1]) and torch.equal(eager, ref[0])
        assert ctxs[0].tolist() == [2997, 38, 894]


def test_streams_and_host_threads(gpu_lib):
    """Calls on two streams at once, from two threads each with a stream of its own, and on one workspace in turn."""
    c = _to(_cache(101, (16, 2, 128), [5000, 300], True))
    q = [_rand(102 + i, 2, 16, 128).bfloat16().to(DEV) for i in range(2)]
    ref = [aflex.attn_decode_f8(c, x) for x in q]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]

    def work(i):
        for _ in range(20):
            got[i].append(aflex.attn_decode_f8(c, q[i], stream=streams[i]))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert all(torch.equal(x, ref[i]) for i in range(2) for x in got[i])
    ws = aflex.Workspace()
    for i in (0, 1, 0):
        assert torch.equal(aflex.attn_decode_f8(c, q[i], ws=ws), ref[i])


def test_bounds_are_read_on_the_call_s_stream(gpu_lib):
    """Without a bound from the caller, the starts are read behind the work of the stream that the call runs on."""
    heads, counts = (8, 2, 64), [40, 2]
    for f8 in (False, True):
        c = _dev(_cache(125, heads, [60, 30], f8))
        (_, dev), new, side = _tokens(126, 42, heads, False), _i32(_cu(counts)), torch.cuda.Stream()
        write = aflex.rope_write_f8 if f8 else aflex.rope_write
        want = [write(c, *dev, new, None, max_seqlen=40), aflex.attn_tree(c, dev[0], new, max_drafts=40)]
        calls = [lambda cu: write(c, *dev, cu, None, stream=side),
                 lambda cu: aflex.attn_tree(c, dev[0], cu, stream=side)]
        for call, ref in zip(calls, want):
            cu = _i32([0, 1, 2])
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                torch.cuda._sleep(20_000_000)
                cu.copy_(new)
            got = call(cu)
            torch.cuda.synchronize()
            assert torch.equal(got, ref)


def test_profile_names(gpu_lib):
    c = _to(_cache(103, (8, 2, 64), [100, 90], True))
    (q, k, v), dev = _tokens(104, 2, (8, 2, 64), False)
    cu = _i32([0, 1, 2])
    torch.cuda.synchronize()
    aflex.profile_start()
    x = aflex.rope_append_f8(c, *dev, None)
    aflex.rope_write_f8(c, *dev, cu, None, max_seqlen=1)
    aflex.attn_decode_f8(c, x)
    aflex.cache_accept(c, cu, _i32([[0], [0]]), _i32([1, 1]))
    names = aflex.profile_stop()
    assert {"rope_append_f8", "rope_write_f8", "attn_rows", "cache_accept"} <= set(names)
