"""Host-side checks of the long-context entry points (no GPU needed): exports,
refusals before any launch, workspace sizes, and what the binding refuses."""
import ctypes
import os
import sys
import threading
import time

import numpy as np
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
    names = aflex.exported_names(aflex.LONGCTX_HEADER)
    assert len(names) == 7
    for n in names:
        assert hasattr(lib, n), n


def _fill(cls, kw, **base):
    a = cls(**base)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _rope(**kw):
    return _fill(aflex.RopeArgs, kw, q=FAKE, k_new=FAKE, v_new=FAKE, rope=FAKE, positions=None, cu_seqlens=FAKE,
                 q_out=FAKE, k_cache=FAKE, v_cache=FAKE, block_keys=FAKE, block_exp=FAKE, block_table=FAKE,
                 context_lens=FAKE, B=2, T=20, Hq=8, Hkv=2, D=64, rotary_dim=64, interleaved=0, rope_len=100,
                 max_seqlen=15, block_size=16, max_blocks_per_seq=4, num_blocks=8)


BOTH = [(dict(q=None), INVALID), (dict(k_new=None), INVALID), (dict(q_out=None), INVALID), (dict(rope=None), INVALID),
        (dict(block_keys=None), INVALID), (dict(block_exp=None), INVALID), (dict(B=0), INVALID), (dict(Hq=0), INVALID),
        (dict(Hkv=0), INVALID), (dict(num_blocks=0), INVALID), (dict(max_blocks_per_seq=0), INVALID),
        (dict(max_blocks_per_seq=(1 << 26) + 1), UNSUP),
        (dict(D=96), UNSUP), (dict(block_size=32), UNSUP), (dict(rotary_dim=65), INVALID),
        (dict(rotary_dim=24), INVALID), (dict(rotary_dim=-16), INVALID), (dict(rotary_dim=80), INVALID),
        (dict(rope_len=0), INVALID), (dict(q_stride=504), INVALID), (dict(q_stride=516), INVALID),
        (dict(k_stride=64), INVALID), (dict(v_stride=-128), INVALID), (dict(q=FAKE + 8), ALIGN),
        (dict(v_cache=FAKE + 2), ALIGN), (dict(rope=FAKE + 4), ALIGN), (dict(block_keys=FAKE + 1), ALIGN),
        (dict(context_lens=FAKE + 2), ALIGN), (dict(positions=FAKE + 1), ALIGN), (dict(Hq=1 << 25), UNSUP)]


@pytest.mark.parametrize("kw,status", BOTH + [(dict(B=1 << 28, Hq=8), UNSUP)])
def test_rope_append_rejects(lib, kw, status):
    assert lib.aflex_rope_append(ctypes.byref(_rope(**kw)), None) == status
    assert lib.aflex_last_error().startswith(b"rope_append")


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(cu_seqlens=None), INVALID), (dict(T=-1), INVALID), (dict(max_seqlen=-1), INVALID),
    (dict(max_seqlen=21), INVALID), (dict(B=70000), UNSUP), (dict(Hq=8192), UNSUP), (dict(cu_seqlens=FAKE + 1), ALIGN)])
def test_rope_write_rejects(lib, kw, status):
    assert lib.aflex_rope_write(ctypes.byref(_rope(**kw)), None) == status
    assert lib.aflex_last_error().startswith(b"rope_write")


def test_nothing_to_write_is_no_launch(lib):
    assert lib.aflex_rope_write(ctypes.byref(_rope(T=0, max_seqlen=0)), None) == aflex.OK
    assert lib.aflex_rope_write(ctypes.byref(_rope(rotary_dim=0, rope=None, rope_len=0, block_keys=None,
                                                   block_exp=None, T=0, max_seqlen=0)), None) == aflex.OK
    assert lib.aflex_block_summary(ctypes.byref(_summary(max_context_len=15)), None) == aflex.OK


def _summary(**kw):
    return _fill(aflex.BlockSummaryArgs, kw, k_cache=FAKE, block_keys=FAKE, block_exp=FAKE, block_table=FAKE,
                 context_lens=FAKE, B=2, Hkv=2, D=64, block_size=16, max_blocks_per_seq=4, num_blocks=8,
                 max_context_len=64)


@pytest.mark.parametrize("kw,status", [
    (dict(k_cache=None), INVALID), (dict(block_exp=None), INVALID), (dict(B=0), INVALID), (dict(B=65536), UNSUP),
    (dict(D=32), UNSUP), (dict(block_size=8), UNSUP), (dict(max_context_len=65), INVALID),
    (dict(max_context_len=-1), INVALID), (dict(k_cache=FAKE + 8), ALIGN), (dict(block_table=FAKE + 2), ALIGN)])
def test_block_summary_rejects(lib, kw, status):
    assert lib.aflex_block_summary(ctypes.byref(_summary(**kw)), None) == status
    assert lib.aflex_last_error().startswith(b"block_summary")


def _select(**kw):
    return _fill(aflex.BlockSelectArgs, kw, q=FAKE, block_keys=FAKE, block_exp=FAKE, block_table=FAKE,
                 context_lens=FAKE, selected=FAKE, B=2, Hq=8, Hkv=2, D=64, block_size=16, max_blocks_per_seq=40,
                 num_blocks=80, max_context_len=640, top_blocks=8, sink_blocks=1, recent_blocks=2)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), INVALID), (dict(selected=None), INVALID), (dict(B=0), INVALID), (dict(Hq=7), INVALID),
    (dict(Hq=34), UNSUP), (dict(D=256), UNSUP), (dict(block_size=64), UNSUP), (dict(max_context_len=641), INVALID),
    (dict(top_blocks=2), INVALID), (dict(top_blocks=0, sink_blocks=0, recent_blocks=0), INVALID),
    (dict(recent_blocks=0), INVALID), (dict(sink_blocks=-1), INVALID),
    (dict(sink_blocks=(1 << 31) - 1, recent_blocks=(1 << 31) - 1), INVALID),
    (dict(B=1 << 20, Hkv=8, max_blocks_per_seq=1 << 20, max_context_len=1 << 24), UNSUP),
    (dict(B=1 << 20, top_blocks=1 << 10), UNSUP),
    (dict(q=FAKE + 2), ALIGN), (dict(selected=FAKE + 2), ALIGN)])
def test_block_select_rejects(lib, kw, status):
    n = ctypes.c_size_t()
    a = _select(**kw)
    assert lib.aflex_block_select(ctypes.byref(a), ctypes.c_void_p(FAKE), 1 << 40, None) == status
    assert lib.aflex_last_error().startswith(b"block_select")
    assert lib.aflex_block_select_workspace(ctypes.byref(a), ctypes.byref(n)) == status


def test_block_select_workspace(lib):
    n = ctypes.c_size_t()
    a = _select()
    assert lib.aflex_block_select_workspace(ctypes.byref(a), ctypes.byref(n)) == aflex.OK
    need = n.value
    assert lib.aflex_block_select_workspace(ctypes.byref(a), None) == INVALID
    if need:
        assert lib.aflex_block_select(ctypes.byref(a), ctypes.c_void_p(FAKE), need - 1, None) == WS
        assert lib.aflex_block_select(ctypes.byref(a), None, need, None) == WS
        assert lib.aflex_block_select(ctypes.byref(a), ctypes.c_void_p(FAKE + 128), need, None) == ALIGN


def _sparse(top_blocks=8, selected=FAKE, **kw):
    a = aflex.AttnArgs(q=FAKE, k_cache=FAKE, v_cache=FAKE, block_table=FAKE, context_lens=FAKE, out=FAKE, B=4, Hq=8,
                       Hkv=2, D=64, block_size=16, max_blocks_per_seq=130, num_blocks=320, max_context_len=2000,
                       scale=0.0, split_tokens=0)
    for k, v in kw.items():
        setattr(a, k, v)
    return aflex.AttnSparseArgs(a, selected, top_blocks)


@pytest.mark.parametrize("kw,status", [
    (dict(selected=None), INVALID), (dict(top_blocks=0), INVALID), (dict(out=None), INVALID), (dict(q=None), INVALID),
    (dict(split_tokens=128), UNSUP), (dict(D=96), UNSUP), (dict(Hq=34), UNSUP), (dict(scale=-1.0), INVALID),
    (dict(top_blocks=(1 << 31) - 1), UNSUP), (dict(selected=FAKE + 2), ALIGN), (dict(q=FAKE + 8), ALIGN)])
def test_attn_sparse_rejects(lib, kw, status):
    a = _sparse(**kw)
    assert lib.aflex_attn_sparse_decode(ctypes.byref(a), ctypes.c_void_p(FAKE), 1 << 40, None) == status
    assert lib.aflex_last_error()


def test_attn_sparse_workspace_goes_by_the_chosen_blocks(lib):
    n = ctypes.c_size_t()
    sizes = []
    for top in (1, 64, 1 << 20):
        a = _sparse(top_blocks=top, B=64, Hq=64, Hkv=8, D=128, max_blocks_per_seq=4096, max_context_len=65536)
        assert lib.aflex_attn_sparse_decode_workspace(ctypes.byref(a), ctypes.byref(n)) == aflex.OK
        assert n.value >= 64 * 8 * 8 * (128 + 2) * 4
        assert lib.aflex_attn_sparse_decode(ctypes.byref(a), ctypes.c_void_p(FAKE), n.value - 1, None) == WS
        sizes.append(n.value)
    assert sizes[0] <= sizes[1] <= sizes[2]


def _calls():
    a = synth.custom_attention(0, 2, 8, 2, 64, [20, 33], ctx_hi=64)
    s = aflex.BlockSummary.of(a)
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    rope = aflex.rope_table(64, 64)
    cu = torch.tensor([0, 1, 2], dtype=torch.int32)
    sel = torch.zeros(2, 2, 3, dtype=torch.int32)
    return {
        "rope_append": lambda: aflex.rope_append(a, a.q, k, k, rope, summary=s),
        "rope_write": lambda: aflex.rope_write(a, a.q, k, k, cu, rope, max_seqlen=1),
        "block_summary": lambda: aflex.block_summary(a, s),
        "block_select": lambda: aflex.block_select(a, a.q, s, 3),
        "attn_sparse_decode": lambda: aflex.attn_sparse_decode(a, sel),
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


def _block_of(*items, dev=-1, call=None):
    """The argument block that items make, zeros behind it."""
    got = []
    keep = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p)(
        lambda p, s: got.append((ctypes.string_at(p, 256), s)) or 7)
    assert (call or aflex._call)(ctypes.cast(keep, ctypes.c_void_p).value, dev, 5, None, 0, *items) == 7
    assert got[0][1] == 5
    return got[0][0]


def test_rows_that_the_binding_refuses(lib):
    x = torch.zeros(3, 12, 64, dtype=torch.bfloat16)

    def rows(t, T, H, D):
        b = _block_of("q", t, aflex._ROWS, T, H, D, None)
        return int.from_bytes(b[:8], "little"), int.from_bytes(b[8:12], "little")

    y = x[:, 2:10]
    assert rows(y, 3, 8, 64) == (y.data_ptr(), 12 * 64)
    assert rows(x[:1, :1], 1, 1, 64) == (x.data_ptr(), 0)
    for bad in (x.float()[:, :8], x[:, :7], x[:, 0:8].transpose(0, 1).contiguous().transpose(0, 1),
                x[:1, :8].expand(3, 8, 64), x[..., ::2], x[:, ::2], x[:2, :8], x[0, :8]):
        with pytest.raises(ValueError, match="q: expected bf16"):
            rows(bad, 3, 8, 64)


def test_dense_tensors_that_the_binding_refuses(lib):
    x = torch.zeros(3, 12, 64, dtype=torch.bfloat16)
    n = x.numel()
    b = _block_of("t", x, aflex._BF16, n, 9, "u", None, aflex._F32, 5)
    assert b[:8] == x.data_ptr().to_bytes(8, "little") and b[8:12] == bytes([9, 0, 0, 0]) and not any(b[12:])
    for bad, code, count in ((x[:, :8], 0, 3 * 8 * 64), (x.float(), 0, n), (x, 1, n), (x, 0, n + 1), (x.to("meta"), 0, n),
                             (x, 9, n)):
        with pytest.raises(ValueError, match="t: expected .* dense"):
            _block_of("t", bad, code, count)
    for item in (("q", x, aflex._ROWS, 3, 12, 64), ("q", x, aflex._BF16, n)):  # a host tensor where cuda:0 is meant
        with pytest.raises(ValueError, match="cuda:0"):
            _block_of(*item, dev=0)
    for item in (("t", 5, 0, 1), ("t", x, 0), ("t", x), (x,), (None,), ("q", None, aflex._ROWS, 3, 12, 64)):
        with pytest.raises(TypeError):
            _block_of(*item)
    with pytest.raises(OverflowError):
        _block_of(1 << 31)
    with pytest.raises(TypeError, match="too long"):
        _block_of(*range(65))
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode() as mode, pytest.raises((RuntimeError, ValueError)):  # without memory
        _block_of("t", mode.from_tensor(x), aflex._BF16, n)


def test_calls_lay_out_the_argument_blocks(lib, monkeypatch):
    """Every field of the C structs from a call of the binding, on host tensors."""
    got, real = {}, aflex._call

    def call(entry, dev, stream, ws, nbytes, *items):
        got["block"] = _block_of(*items, call=real)
        return aflex.OK if stream is not None else (aflex.OK, 0)

    monkeypatch.setattr(aflex, "_call", call)
    monkeypatch.setattr(aflex, "_stream", lambda s: 0)
    monkeypatch.setattr(aflex, "_default_ws", {})
    monkeypatch.setattr(aflex, "_need_gpu", lambda d: None)
    monkeypatch.setattr(aflex.Workspace, "get", lambda self, n, d: torch.zeros(256, dtype=torch.uint8))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    a = synth.custom_attention(0, 2, 8, 2, 64, [20, 33], ctx_hi=64)
    s = aflex.BlockSummary.of(a)
    x = torch.zeros(2, 12, 64, dtype=torch.bfloat16)
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:]
    rope = aflex.rope_table(64, 32)
    pos, cu = torch.zeros(2, dtype=torch.int32), torch.tensor([0, 1, 2], dtype=torch.int32)
    out, sel = torch.empty_like(a.q), torch.zeros(2, 2, 3, dtype=torch.int32)

    def fields(c):
        b = c.from_buffer_copy(got["block"])
        return {f: getattr(b, f) for f, _ in c._fields_}

    P = lambda t: t.data_ptr()  # noqa: E731
    cache = dict(k_cache=P(a.k_cache), block_table=P(a.block_table), context_lens=P(a.context_lens))
    sizes = dict(B=2, Hkv=2, D=64, block_size=16, max_blocks_per_seq=4, num_blocks=a.num_blocks)
    aflex.rope_write(a, q, k, v, cu, rope, max_seqlen=1, interleaved=True, positions=pos, summary=s, q_out=out)
    assert fields(aflex.RopeArgs) == dict(
        q=P(q), k_new=P(k), v_new=P(v), rope=P(rope), positions=P(pos), cu_seqlens=P(cu), q_out=P(out),
        v_cache=P(a.v_cache), block_keys=P(s.keys), block_exp=P(s.exp), T=2, Hq=8, rotary_dim=32, interleaved=1,
        rope_len=64, max_seqlen=1, q_stride=768, k_stride=768, v_stride=768, **cache, **sizes)
    aflex.rope_append(a, q, k, v, None, q_out=out)
    f = fields(aflex.RopeArgs)
    assert (f["rope"], f["positions"], f["cu_seqlens"], f["block_keys"], f["block_exp"]) == (None,) * 5
    assert (f["rotary_dim"], f["rope_len"], f["interleaved"]) == (0, 0, 0)
    aflex.block_summary(a, s)
    assert fields(aflex.BlockSummaryArgs) == dict(block_keys=P(s.keys), block_exp=P(s.exp), max_context_len=64, **cache,
                                                  **sizes)
    aflex.block_select(a, a.q, s, 3, 1, 2, out=sel)
    del cache["k_cache"]
    assert fields(aflex.BlockSelectArgs) == dict(
        q=P(a.q), block_keys=P(s.keys), block_exp=P(s.exp), selected=P(sel), Hq=8, max_context_len=64, top_blocks=3,
        sink_blocks=1, recent_blocks=2, **cache, **sizes)
    aflex.attn_sparse_decode(a, sel, out=out, scale=0.5)
    f = fields(aflex.AttnSparseArgs)
    assert (f["selected"], f["top_blocks"]) == (P(sel), 3)
    assert fields(aflex.AttnArgs) == dict(
        q=P(a.q), k_cache=P(a.k_cache), v_cache=P(a.v_cache), out=P(out), Hq=8, max_context_len=64, scale=0.5,
        split_tokens=0, **cache, **sizes)


def _no_gpu(monkeypatch):
    """Calls of the binding run on host tensors, up to aflex._call."""
    monkeypatch.setattr(aflex, "_stream", lambda s: 0)
    monkeypatch.setattr(aflex, "_default_ws", {})
    monkeypatch.setattr(aflex, "_need_gpu", lambda d: None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)


@pytest.mark.parametrize("own_ws", [False, True])
@pytest.mark.parametrize("op", ["block_select", "attn_sparse_decode"])
def test_a_workspace_is_in_one_host_thread_at_a_time(lib, monkeypatch, op, own_ws):
    """The two launches of a call communicate through the workspace: a second thread's call
    on the same stream may not launch between them."""
    _no_gpu(monkeypatch)
    monkeypatch.setattr(aflex.Workspace, "get", lambda self, n, d: self.__dict__.setdefault(
        "host", torch.zeros(256, dtype=torch.uint8)))
    inside, met, entered = {}, [], threading.Event()

    def call(entry, dev, stream, ws, nbytes, *items):
        if stream is None:
            return aflex.OK, 256
        inside[ws] = inside.get(ws, 0) + 1
        if inside[ws] > 1:
            met.append(ws)
        if entered.is_set():
            time.sleep(0.01)
        else:
            entered.set()
            time.sleep(0.3)  # the second thread comes here meanwhile, if it can
        inside[ws] -= 1
        return aflex.OK

    monkeypatch.setattr(aflex, "_call", call)
    a = synth.custom_attention(0, 2, 8, 2, 64, [20, 33], ctx_hi=64)
    s, sel = aflex.BlockSummary.of(a), torch.zeros(2, 2, 3, dtype=torch.int32)
    kw = {"ws": aflex.Workspace()} if own_ws else {}
    run = {"block_select": lambda: aflex.block_select(a, a.q, s, 3, out=sel, **kw),
           "attn_sparse_decode": lambda: aflex.attn_sparse_decode(a, sel, out=torch.empty_like(a.q), **kw)}[op]
    threads = [threading.Thread(target=run) for _ in range(2)]
    threads[0].start()
    assert entered.wait(10)
    threads[1].start()
    for t in threads:
        t.join(20)
        assert not t.is_alive()
    assert not met and len(inside) >= 1


def test_older_operators_load_without_the_call_module(lib, monkeypatch):
    """The library alone serves the operators that are called through ctypes; the long-context ones say what is missing."""
    calls = _calls()
    import paper_2608_01891_amd as package
    monkeypatch.delattr(package, "_tensor_args", raising=False)
    monkeypatch.setitem(sys.modules, "paper_2608_01891_amd._tensor_args", None)  # its import fails
    monkeypatch.setattr(aflex, "_lib", None)
    monkeypatch.setattr(aflex, "_call", None)
    monkeypatch.setattr(aflex.atexit, "register", lambda f: None)
    assert aflex.load().aflex_kv_append(None, None) == INVALID
    for op in calls.values():
        with pytest.raises(RuntimeError, match="_tensor_args.so cannot be loaded"):
            op()


def test_sizes_may_be_whole_numbers_of_other_types(lib):
    """numpy's integers, as max() of an array of lengths gives; not strings, lists or fractions of them."""
    b = _block_of(np.int64(640), np.int32(-3), np.uint8(7), True, 5)
    assert [int.from_bytes(b[4 * i:4 * i + 4], "little", signed=True) for i in range(5)] == [640, -3, 7, 1, 5]
    assert _block_of(np.float64(0.5))[:4] == _block_of(0.5)[:4]
    with pytest.raises(OverflowError):
        _block_of(np.int64(1 << 31))
    for bad in (np.float32(2.0), [3], b"4", torch.ones(2)):
        with pytest.raises(TypeError):
            _block_of(bad)


def test_more_threads_than_a_launch_takes_are_refused(lib):
    """2^32 threads along one dimension: refused here, not left to the runtime."""
    n = ctypes.c_size_t()
    assert lib.aflex_rope_append(ctypes.byref(_rope(B=1 << 25, Hq=2, Hkv=2, D=64)), None) == UNSUP
    assert lib.aflex_rope_append(ctypes.byref(_rope(B=1 << 22, Hq=128, Hkv=1, D=128)), None) == UNSUP
    assert lib.aflex_rope_write(ctypes.byref(_rope(T=1 << 29, max_seqlen=(1 << 28) - 31)), None) == UNSUP
    few = dict(B=1 << 23, Hkv=2, Hq=2, max_blocks_per_seq=4, max_context_len=64)
    a = _select(top_blocks=4, sink_blocks=1, recent_blocks=1, **few)
    assert lib.aflex_block_select_workspace(ctypes.byref(a), ctypes.byref(n)) == UNSUP
    a.B -= 1
    assert lib.aflex_block_select_workspace(ctypes.byref(a), ctypes.byref(n)) == aflex.OK and n.value == 0
    a = _sparse(top_blocks=4, **few)
    assert lib.aflex_attn_sparse_decode_workspace(ctypes.byref(a), ctypes.byref(n)) == UNSUP
    a.attn.B -= 1
    assert lib.aflex_attn_sparse_decode_workspace(ctypes.byref(a), ctypes.byref(n)) == aflex.OK


def test_block_select_workspace_of_two_launches(lib):
    """Above 1024 blocks the scores' keys are in the workspace, rows of a multiple of 4."""
    n = ctypes.c_size_t()
    a = _select(max_blocks_per_seq=1030, max_context_len=1025 * 16 + 1)
    assert lib.aflex_block_select_workspace(ctypes.byref(a), ctypes.byref(n)) == aflex.OK
    need = n.value
    assert need >= 2 * 2 * 1028 * 4
    assert lib.aflex_block_select(ctypes.byref(a), ctypes.c_void_p(FAKE), need - 1, None) == WS
    assert lib.aflex_block_select(ctypes.byref(a), None, need, None) == WS
    assert lib.aflex_block_select(ctypes.byref(a), ctypes.c_void_p(FAKE + 128), need, None) == ALIGN
    a = _select(max_blocks_per_seq=1030, max_context_len=1024 * 16)
    assert lib.aflex_block_select_workspace(ctypes.byref(a), ctypes.byref(n)) == aflex.OK and n.value == 0
