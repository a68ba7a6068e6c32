"""Host-side checks of the 8-bit cache's and the drafts' entry points (no GPU needed): exports, refusals before
any launch, workspace sizes, argument blocks, and what the binding refuses."""
import ctypes
import os

import pytest
import torch

from paper_2608_01891_amd import aflex, synth

FAKE = 0x10000000  # aligned, never dereferenced: validation fails before any launch
INVALID, UNSUP, ALIGN, WS = (aflex.ERR_INVALID_ARG, aflex.ERR_UNSUPPORTED, aflex.ERR_ALIGNMENT, aflex.ERR_WORKSPACE)


@pytest.fixture(scope="module")
def lib():
    from paper_2608_01891_amd import build
    if not (os.path.exists(aflex.LIB_PATH) and os.path.exists(build.TENSOR_ARGS)):
        build.build(verbose=False)
    return aflex.load()


def test_exports_every_declared_symbol(lib):
    names = aflex.exported_names(aflex.DRAFT_HEADER)
    assert len(names) == 7
    for n in names:
        assert hasattr(lib, n), n


def _fill(cls, kw, **base):
    a = cls(**base)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _rope(**kw):
    return _fill(aflex.RopeF8Args, kw, q=FAKE, k_new=FAKE, v_new=FAKE, rope=FAKE, positions=None, cu_seqlens=FAKE,
                 q_out=FAKE, k_cache=FAKE, v_cache=FAKE, kv_exp=FAKE, block_table=FAKE, context_lens=FAKE,
                 B=2, T=20, Hq=8, Hkv=2, D=64, rotary_dim=64, interleaved=0, rope_len=100,
                 max_seqlen=15, block_size=16, max_blocks_per_seq=4, num_blocks=8)


BOTH = [(dict(q=None), INVALID), (dict(k_new=None), INVALID), (dict(q_out=None), INVALID), (dict(rope=None), INVALID),
        (dict(kv_exp=None), INVALID), (dict(v_cache=None), INVALID), (dict(B=0), INVALID), (dict(Hq=0), INVALID),
        (dict(Hkv=0), INVALID), (dict(num_blocks=0), INVALID), (dict(max_blocks_per_seq=0), INVALID),
        (dict(max_blocks_per_seq=(1 << 26) + 1), UNSUP),
        (dict(D=96), UNSUP), (dict(block_size=32), UNSUP), (dict(rotary_dim=65), INVALID),
        (dict(rotary_dim=24), INVALID), (dict(rotary_dim=-16), INVALID), (dict(rotary_dim=80), INVALID),
        (dict(rope_len=0), INVALID), (dict(q_stride=504), INVALID), (dict(q_stride=516), INVALID),
        (dict(k_stride=64), INVALID), (dict(v_stride=-128), INVALID), (dict(q=FAKE + 8), ALIGN),
        (dict(v_cache=FAKE + 2), ALIGN), (dict(rope=FAKE + 4), ALIGN), (dict(kv_exp=FAKE + 1), ALIGN),
        (dict(context_lens=FAKE + 2), ALIGN), (dict(positions=FAKE + 1), ALIGN), (dict(Hq=1 << 25), UNSUP)]


@pytest.mark.parametrize("kw,status", BOTH + [(dict(B=1 << 28, Hq=8), UNSUP)])
def test_rope_append_f8_rejects(lib, kw, status):
    assert lib.aflex_rope_append_f8(ctypes.byref(_rope(**kw)), None) == status
    assert lib.aflex_last_error().startswith(b"rope_append_f8")


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(cu_seqlens=None), INVALID), (dict(T=-1), INVALID), (dict(max_seqlen=-1), INVALID),
    (dict(max_seqlen=21), INVALID), (dict(B=70000), UNSUP), (dict(Hq=8192), UNSUP), (dict(cu_seqlens=FAKE + 1), ALIGN)])
def test_rope_write_f8_rejects(lib, kw, status):
    assert lib.aflex_rope_write_f8(ctypes.byref(_rope(**kw)), None) == status
    assert lib.aflex_last_error().startswith(b"rope_write_f8")


def test_nothing_to_do_is_no_launch(lib):
    assert lib.aflex_rope_write_f8(ctypes.byref(_rope(T=0, max_seqlen=0)), None) == aflex.OK
    for kw in (dict(T=0), dict(T=0, max_drafts=0)):
        assert lib.aflex_attn_tree(ctypes.byref(_tree(**kw)), ctypes.c_void_p(FAKE), 1 << 40, None) == aflex.OK


def _decode(**kw):
    return _fill(aflex.AttnF8Args, kw, q=FAKE, k_cache=FAKE, v_cache=FAKE, kv_exp=FAKE, block_table=FAKE,
                 context_lens=FAKE, out=FAKE, B=4, Hq=8, Hkv=2, D=64, block_size=16, max_blocks_per_seq=130,
                 num_blocks=320, max_context_len=2000, scale=0.0)


def _tree(**kw):
    return _fill(aflex.AttnTreeArgs, kw, q=FAKE, k_cache=FAKE, v_cache=FAKE, kv_exp=FAKE, block_table=FAKE,
                 context_lens=FAKE, cu_seqlens=FAKE, masks=FAKE, out=FAKE, B=4, T=30, Hq=8, Hkv=2, D=64, max_drafts=9,
                 block_size=16, max_blocks_per_seq=130, num_blocks=320, max_context_len=2000, scale=0.0)


ATTN = [(dict(q=None), INVALID), (dict(out=None), INVALID), (dict(k_cache=None), INVALID), (dict(block_table=None), INVALID),
        (dict(B=0), INVALID), (dict(Hq=7), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=0), INVALID), (dict(Hq=34), UNSUP),
        (dict(Hq=70000, Hkv=70000), UNSUP), (dict(D=96), UNSUP), (dict(block_size=32), UNSUP), (dict(num_blocks=0), INVALID),
        (dict(max_context_len=-1), INVALID), (dict(max_context_len=2081), INVALID), (dict(scale=-1.0), INVALID),
        (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(q=FAKE + 8), ALIGN),
        (dict(k_cache=FAKE + 8), ALIGN), (dict(kv_exp=FAKE + 4), ALIGN), (dict(out=FAKE + 2), ALIGN),
        (dict(context_lens=FAKE + 2), ALIGN)]


def _attn_rejects(lib, name, a, status, out=True):
    n = ctypes.c_size_t()
    assert getattr(lib, name)(ctypes.byref(a), ctypes.c_void_p(FAKE), 1 << 45, None) == status
    assert lib.aflex_last_error().decode().startswith(name[6:])
    if out:  # (the size does not depend on it)
        assert getattr(lib, name + "_workspace")(ctypes.byref(a), ctypes.byref(n)) == status


@pytest.mark.parametrize("kw,status", ATTN + [
    (dict(kv_exp=None), INVALID), (dict(B=1 << 20, max_blocks_per_seq=1 << 10, max_context_len=1 << 14), UNSUP),
    (dict(B=1 << 24, max_context_len=16), UNSUP)])
def test_attn_decode_f8_rejects(lib, kw, status):
    _attn_rejects(lib, "aflex_attn_decode_f8", _decode(**kw), status, out="out" not in kw or kw["out"] is not None)


@pytest.mark.parametrize("kw,status", ATTN + [
    (dict(cu_seqlens=None), INVALID), (dict(T=-1), INVALID), (dict(max_drafts=-1), INVALID), (dict(max_drafts=65), UNSUP),
    (dict(T=37), INVALID), (dict(T=1, max_drafts=0), INVALID), (dict(cu_seqlens=FAKE + 2), ALIGN),
    (dict(masks=FAKE + 4), ALIGN), (dict(B=1 << 18, T=1 << 24, max_drafts=64), UNSUP),
    (dict(B=1 << 19, max_blocks_per_seq=1 << 10, max_context_len=1 << 14), UNSUP),
    (dict(B=1 << 17, Hq=1 << 9, Hkv=1 << 9, T=1 << 22, max_drafts=64, max_context_len=0), UNSUP)])
def test_attn_tree_rejects(lib, kw, status):
    _attn_rejects(lib, "aflex_attn_tree", _tree(**kw), status, out="out" not in kw or kw["out"] is not None)


def test_workspaces(lib):
    n = ctypes.c_size_t()
    for name, a in (("aflex_attn_decode_f8", _decode()), ("aflex_attn_tree", _tree()),
                    ("aflex_attn_tree", _tree(kv_exp=None, masks=None))):
        query = getattr(lib, name + "_workspace")
        assert query(ctypes.byref(a), None) == INVALID
        assert query(ctypes.byref(a), ctypes.byref(n)) == aflex.OK and n.value > 0
        call = getattr(lib, name)
        assert call(ctypes.byref(a), ctypes.c_void_p(FAKE), n.value - 1, None) == WS
        assert call(ctypes.byref(a), None, n.value, None) == WS
        assert call(ctypes.byref(a), ctypes.c_void_p(FAKE + 128), n.value, None) == ALIGN
    # partial rows: those of the tokens, and one pass of rows per work-group
    big = _tree(B=8, T=8 * 64, Hq=64, Hkv=8, D=128, max_drafts=64, max_blocks_per_seq=4096, max_context_len=65536)
    assert lib.aflex_attn_tree_workspace(ctypes.byref(big), ctypes.byref(n)) == aflex.OK
    assert 8 * 64 * 64 * 130 * 4 < n.value < 1 << 30


@pytest.mark.parametrize("B,whole", [(40, False), (48, True), (64, True), (65, False), (95, False), (96, True), (256, True)])
def test_units_of_short_contexts_are_cut_where_they_do_not_balance(lib, B, whole):
    """Up to 2048 tokens units stay whole where they fill 3/4 to one round of work-groups (512 on 256 compute units) or
    3/2 and more: between those the last ones would run alone. Cut units need room for their partial rows."""
    n = ctypes.c_size_t()
    tree = _tree(B=B, T=B * 8, Hq=64, Hkv=8, D=128, max_drafts=8, max_blocks_per_seq=128, max_context_len=2048)
    assert lib.aflex_attn_tree_workspace(ctypes.byref(tree), ctypes.byref(n)) == aflex.OK
    assert (n.value < 1 << 20) == whole and (n.value > B * 8 * 64 * 128 * 4) == (not whole)


def _accept(**kw):
    return _fill(aflex.CacheAcceptArgs, kw, k_cache=FAKE, v_cache=FAKE, kv_exp=FAKE, block_table=FAKE,
                 context_lens=FAKE, cu_seqlens=FAKE, accepted=FAKE, accepted_counts=FAKE, context_out=FAKE + 64,
                 B=2, Hkv=2, D=64, max_accepted=5, block_size=16, max_blocks_per_seq=4, num_blocks=8)


@pytest.mark.parametrize("kw,status", [
    (dict(k_cache=None), INVALID), (dict(accepted=None), INVALID), (dict(accepted_counts=None), INVALID),
    (dict(context_out=None), INVALID), (dict(context_out=FAKE), INVALID), (dict(cu_seqlens=None), INVALID),
    (dict(B=0), INVALID), (dict(B=65536), UNSUP), (dict(Hkv=65536), UNSUP), (dict(D=32), UNSUP),
    (dict(block_size=8), UNSUP), (dict(max_accepted=0), INVALID), (dict(max_accepted=65), UNSUP),
    (dict(k_cache=FAKE + 8), ALIGN), (dict(kv_exp=FAKE + 8), ALIGN), (dict(accepted=FAKE + 2), ALIGN)])
def test_cache_accept_rejects(lib, kw, status):
    assert lib.aflex_cache_accept(ctypes.byref(_accept(**kw)), None) == status
    assert lib.aflex_last_error().startswith(b"cache_accept")


@pytest.mark.parametrize("name,count", [("context_lens", 2), ("cu_seqlens", 3), ("accepted_counts", 2),
                                        ("accepted", 10), ("block_table", 8)])
def test_cache_accept_keeps_its_output_apart(lib, name, count):
    """New lengths in an array that other work-groups of the sequence read, wholly or in part."""
    out = FAKE + 4096
    for at in (out, out + 4, out - 4 * (count - 1)):
        assert lib.aflex_cache_accept(ctypes.byref(_accept(context_out=out, **{name: at})), None) == INVALID
        assert b"overlap" in lib.aflex_last_error()


# ------------------------------------------------------------------ the binding
def _state():
    a = synth.custom_attention(0, 2, 8, 2, 64, [20, 33], ctx_hi=64)
    c = aflex.F8Cache(a)
    x = torch.zeros(2, 12, 64, dtype=torch.bfloat16)
    rope = aflex.rope_table(64, 32)
    cu = torch.tensor([0, 1, 2], dtype=torch.int32)
    acc, cnt = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    return a, c, (x[:, :8], x[:, 8:10], x[:, 10:]), rope, cu, acc, cnt


def _calls():
    a, c, qkv, rope, cu, acc, cnt = _state()
    return {
        "rope_append_f8": lambda: aflex.rope_append_f8(c, *qkv, rope),
        "rope_write_f8": lambda: aflex.rope_write_f8(c, *qkv, cu, rope, max_seqlen=1),
        "rope_write_f8, no bound": lambda: aflex.rope_write_f8(c, *qkv, cu, rope),
        "attn_decode_f8": lambda: aflex.attn_decode_f8(c, a.q),
        "attn_tree": lambda: aflex.attn_tree(c, a.q, cu, max_drafts=1),
        "attn_tree, bf16, no bound": lambda: aflex.attn_tree(a, a.q, cu),
        "cache_accept": lambda: aflex.cache_accept(c, cu, acc, cnt),
    }


@pytest.mark.parametrize("op", list(_calls()))
def test_host_tensors_are_refused_before_any_library_call(lib, monkeypatch, op):
    calls = []

    class Stub:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or aflex.OK

    monkeypatch.setattr(aflex, "_lib", Stub())
    with pytest.raises(ValueError, match="cuda device"):
        _calls()[op]()
    assert calls == []


def _host_calls(monkeypatch):
    """Calls of the binding on host tensors, up to the library: their argument blocks."""
    got, real = {}, aflex._call

    def block_of(items):
        held = []
        keep = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p)(
            lambda p, s: held.append(ctypes.string_at(p, 256)) or 7)
        assert real(ctypes.cast(keep, ctypes.c_void_p).value, -1, 5, None, 0, *items) == 7
        return held[0]

    def call(entry, dev, stream, ws, nbytes, *items):
        got["block"] = block_of(items)
        return aflex.OK if stream is not None else (aflex.OK, 0)

    monkeypatch.setattr(aflex, "_call", call)
    monkeypatch.setattr(aflex, "_stream", lambda s: 0)
    monkeypatch.setattr(aflex, "_default_ws", {})
    monkeypatch.setattr(aflex, "_need_gpu", lambda d: None)
    monkeypatch.setattr(aflex, "_empty", lambda stream, dev, *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype))
    monkeypatch.setattr(aflex.Workspace, "get", lambda self, n, d: torch.zeros(256, dtype=torch.uint8))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)

    def fields(c):
        b = c.from_buffer_copy(got["block"])
        return {f: getattr(b, f) for f, _ in c._fields_}

    return fields


def test_calls_lay_out_the_argument_blocks(lib, monkeypatch):
    """Every field of the C structs from a call of the binding, on host tensors."""
    fields = _host_calls(monkeypatch)
    a, c, (q, k, v), rope, cu, acc, cnt = _state()
    P = lambda t: t.data_ptr()  # noqa: E731
    out, pos, ctx = torch.empty_like(a.q), torch.zeros(2, dtype=torch.int32), torch.empty(2, dtype=torch.int32)
    pools = dict(k_cache=P(c.k_cache), v_cache=P(c.v_cache), kv_exp=P(c.kv_exp))
    where = dict(block_table=P(a.block_table), context_lens=P(a.context_lens))
    sizes = dict(B=2, Hkv=2, D=64, block_size=16, max_blocks_per_seq=4, num_blocks=a.num_blocks)
    aflex.rope_write_f8(c, q, k, v, cu, rope, max_seqlen=1, interleaved=True, positions=pos, q_out=out)
    assert fields(aflex.RopeF8Args) == dict(
        q=P(q), k_new=P(k), v_new=P(v), rope=P(rope), positions=P(pos), cu_seqlens=P(cu), q_out=P(out), T=2, Hq=8,
        rotary_dim=32, interleaved=1, rope_len=64, max_seqlen=1, q_stride=768, k_stride=768, v_stride=768,
        **pools, **where, **sizes)
    aflex.rope_append_f8(c, q, k, v, None, q_out=out)
    f = fields(aflex.RopeF8Args)
    assert (f["rope"], f["positions"], f["cu_seqlens"], f["rotary_dim"], f["rope_len"]) == (None, None, None, 0, 0)
    aflex.attn_decode_f8(c, a.q, out=out, scale=0.5)
    assert fields(aflex.AttnF8Args) == dict(q=P(a.q), out=P(out), Hq=8, max_context_len=64, scale=0.5, **pools, **where,
                                            **sizes)
    masks = aflex.tree_masks([[-1], [-1]])
    aflex.attn_tree(c, a.q, cu, masks, max_drafts=3, out=out, scale=0.25)
    want = dict(q=P(a.q), out=P(out), cu_seqlens=P(cu), masks=P(masks), T=2, Hq=8, max_drafts=3, max_context_len=64,
                scale=0.25, **pools, **where, **sizes)
    assert fields(aflex.AttnTreeArgs) == want
    aflex.attn_tree(a, a.q, cu, out=out)
    assert fields(aflex.AttnTreeArgs) == {**want, "masks": None, "max_drafts": 1, "scale": 0.0, "kv_exp": None,
                                          "k_cache": P(a.k_cache), "v_cache": P(a.v_cache)}
    aflex.cache_accept(c, cu, acc, cnt, context_out=ctx)
    assert fields(aflex.CacheAcceptArgs) == dict(cu_seqlens=P(cu), accepted=P(acc), accepted_counts=P(cnt),
                                                 context_out=P(ctx), max_accepted=3, **pools, **where, **sizes)
    aflex.cache_accept(a, cu, acc, cnt, context_out=ctx)
    assert fields(aflex.CacheAcceptArgs)["kv_exp"] is None


def test_tensors_that_the_binding_refuses(lib, monkeypatch):
    _host_calls(monkeypatch)
    a, c, (q, k, v), rope, cu, acc, cnt = _state()
    bad = aflex.F8Cache(a)
    bad.k_cache = a.k_cache
    for call in (lambda: aflex.rope_append_f8(bad, q, k, v, rope), lambda: aflex.attn_decode_f8(bad, a.q),
                 lambda: aflex.attn_tree(bad, a.q, cu), lambda: aflex.cache_accept(bad, cu, acc, cnt)):
        with pytest.raises(ValueError, match="k_cache: expected .* Float8_e4m3fn"):
            call()
    short = aflex.F8Cache(a)
    short.kv_exp = short.kv_exp[:-1]
    with pytest.raises(ValueError, match="kv_exp"):
        aflex.attn_decode_f8(short, a.q)
    with pytest.raises(ValueError, match="q: expected one row"):
        aflex.rope_append_f8(c, q[:1], k[:1], v[:1], rope)
    with pytest.raises(ValueError, match="masks: expected 2 dense Long"):
        aflex.attn_tree(c, a.q, cu, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="masks"):
        aflex.attn_tree(c, a.q, cu, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="q: expected"):
        aflex.attn_tree(c, a.q.transpose(0, 1), cu)
    with pytest.raises(ValueError, match="cu_seqlens"):
        aflex.attn_tree(c, a.q, cu.long(), max_drafts=1)
    with pytest.raises(ValueError, match="accepted"):
        aflex.cache_accept(c, cu, acc.t().contiguous().t(), cnt)
    with pytest.raises(ValueError, match="out: expected"):
        aflex.attn_decode_f8(c, a.q, out=a.q.float())


def test_empty_batches_of_rows_call_nothing(lib, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1)
    monkeypatch.setattr(aflex, "_need_gpu", lambda d: None)
    monkeypatch.setattr(aflex, "_call", lambda *a: pytest.fail("called"))
    a, c, (q, k, v), rope, _, _, _ = _state()
    cu = torch.zeros(3, dtype=torch.int32)
    out = torch.empty(0, 8, 64, dtype=torch.bfloat16)
    assert aflex.rope_write_f8(c, q[:0], k[:0], v[:0], cu, rope, max_seqlen=0, q_out=out) is out
    assert aflex.attn_tree(c, a.q[:0], cu, max_drafts=0, out=out) is out
