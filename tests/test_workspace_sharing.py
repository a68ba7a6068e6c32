"""Workspaces shared by host threads and by streams (no GPU needed: the library
is a stub). One host thread at a time: the launches of a call communicate
through it. Its use on a stream other than its own is recorded."""
import ctypes
import threading
import time

import pytest
import torch

from paper_2608_01891_amd import aflex, synth


class Lib:
    """Entry points that note which workspaces are in use; the first call stays for a while."""

    def __init__(self):
        self.inside, self.met, self.entered = {}, [], threading.Event()

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            def query(*args):
                ctypes.cast(args[-1], ctypes.POINTER(ctypes.c_size_t))[0] = 256
                return aflex.OK
            return query

        def enter(*args):
            at = 5 if "af_" in name else 1
            ws = args[at + 1 if "layer" in name else at]
            self.inside[ws] = self.inside.get(ws, 0) + 1
            if self.inside[ws] > 1:
                self.met.append(ws)
            if not self.entered.is_set():
                self.entered.set()
                time.sleep(0.3)
            self.inside[ws] -= 1
            return aflex.OK
        return enter


@pytest.mark.parametrize("own_ws", [False, True])
@pytest.mark.parametrize("op", ["attn_decode", "ffn_swiglu", "moe_ffn", "linear", "moe_block", "af_pipeline_step",
                                "af_layer_step"])
def test_one_host_thread_at_a_time(monkeypatch, op, own_ws):
    lib, host = Lib(), torch.zeros(256, dtype=torch.uint8)
    monkeypatch.setattr(aflex, "_lib", lib)
    monkeypatch.setattr(aflex, "_default_ws", {})
    monkeypatch.setattr(aflex, "_need_gpu", lambda d: None)
    monkeypatch.setattr(aflex, "_stream", lambda s: 0)
    monkeypatch.setattr(aflex, "_ws", lambda *args, **kw: (host.data_ptr(), 256))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: None)
    w = synth.tiny_layer()
    x, moe, logits = synth.custom_ffn(1, 4, 64, 64, E=4)
    layer = type("Layer", (), dict(k_new=x, v_new=x, w_o=x, x_in=x, norm_weight=x, router_weight=x, eps=1e-5))
    kw = {"ws": aflex.Workspace()} if own_ws else {}
    side = {"stream_a": object(), "stream_f": object(), "join": False}
    run = {
        "attn_decode": lambda: aflex.attn_decode(w.attn, **kw),
        "ffn_swiglu": lambda: aflex.ffn_swiglu(w.x, w.ffn, **kw),
        "moe_ffn": lambda: aflex.moe_ffn(x, moe, logits, 2, **kw),
        "linear": lambda: aflex.linear(x, x, **kw),
        "moe_block": lambda: aflex.moe_block(x, moe, x[0], x, 2, **kw),
        "af_pipeline_step": lambda: aflex.af_pipeline_step(w.attn, moe, logits, 2, [4], **side, **kw),
        "af_layer_step": lambda: aflex.af_layer_step(w.attn, moe, layer, 2, [4], **side, **kw),
    }[op]
    threads = [threading.Thread(target=run) for _ in range(2)]
    threads[0].start()
    assert lib.entered.wait(10)
    threads[1].start()
    for t in threads:
        t.join(20)
        assert not t.is_alive()
    assert len(lib.inside) == 1 and not lib.met


class Buffer:
    device = torch.device("cuda:0")

    def __init__(self):
        self.recorded = []

    def record_stream(self, s):
        self.recorded.append(s)

    def get_device(self):
        return 0

    def data_ptr(self):
        return 256

    def numel(self):
        return 1 << 20


@pytest.mark.parametrize("stream", [None, "given"])
@pytest.mark.parametrize("call", ["_run", "_run_own_ws"])
def test_use_on_another_stream_is_recorded(monkeypatch, call, stream):
    """Also where the other stream is the current one, and no stream is given."""
    monkeypatch.setattr(aflex, "_lib", Lib())
    monkeypatch.setattr(aflex, "_call", lambda *args: aflex.OK)
    monkeypatch.setattr(aflex, "_entry", {"aflex_linear": 0})
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: "current")
    ws = aflex.Workspace()
    ws.buf, ws.home = Buffer(), 7
    for handle, want in ((7, []), (9, [stream or "current"])):
        monkeypatch.setattr(aflex, "_stream", lambda s: handle)
        if call == "_run":
            aflex._run("aflex_linear", aflex.LinearArgs(), "linear", Buffer.device, ws, stream)
        else:
            aflex._run_own_ws("aflex_linear", 0, ws, stream)
        assert ws.buf.recorded == want
