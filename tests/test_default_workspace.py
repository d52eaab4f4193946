"""A call without a workspace makes and clears one on the stream that it was given (no GPU: the library and the streams are
stand-ins that record who was asked for what, where)."""
import contextlib

import pytest
import torch

from paper_2501_06807_amd import _lib as L


class Stream:
    device, cuda_stream = torch.device("cpu"), 77


@pytest.fixture
def made(monkeypatch):
    now, seen = [None], []

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    class Library:
        def __getattr__(self, name):
            return lambda *args: 0

    def workspace(nbytes, device="cuda"):
        seen.append(now[-1])
        return torch.zeros(256, dtype=torch.uint8)

    monkeypatch.setattr(L, "lib", lambda: Library())
    monkeypatch.setattr(L, "_contig", lambda *ts: None)
    monkeypatch.setattr(L, "_rows", lambda t, what, dtype, heads=None: (0, None, t.shape))
    monkeypatch.setattr(L, "_on", lambda device, stream, *ts: 0)
    monkeypatch.setattr(L, "_call", lambda *args: None)
    monkeypatch.setattr(L, "workspace", workspace)
    monkeypatch.setattr(L.torch.cuda, "stream", on)
    return seen


def calls(stream):
    kv, q = torch.zeros(1, 1, 2, 32, 64), torch.zeros(1, 1, 4, 64)
    win, idx, few = torch.zeros(1, 1, 4, 8, 64), torch.zeros(1, 1, 2, 16, dtype=torch.int32), torch.zeros(1, 1, 2, 16, 64)
    cent, scent, sel = torch.zeros(1, 1, 2, 2, 64), torch.zeros(1, 1, 2, 1, 64), torch.zeros(1, 1, 2, 1, dtype=torch.int32)
    cfg = L.select_cfg(16, 2, 1, 1)
    if stream is None:
        stream = dict()
    else:
        stream = dict(stream=stream)

    class Paged:
        L, B, d, dtype, device, ref = 1, 1, 64, torch.float32, torch.device("cpu"), None

        def dims(self, n):
            return None

    return {
        "evict": lambda: L.mpc_static_evict(win, kv, kv, idx, few, few, keep=16, local_keep=2, sm_scale=1.0, **stream),
        "prefill": lambda: L.mpc_prefill(win, kv, kv, idx, few, few, cent[:, :, :, :1], scent, cfg, keep=16, local_keep=2, sm_scale=1.0,
                                         **stream),
        "attend": lambda: L.mpc_sparse_decode_attn(q, kv, kv, sel, q, cluster_size=16, sm_scale=1.0, **stream),
        "step": lambda: L.mpc_decode_step(q, cent, scent, kv, kv, sel, q, cfg, sm_scale=1.0, **stream),
        "paged": lambda: L.mpc_paged_attn(q[:, :, :, None], Paged(), q[:, :, :, None], sm_scale=1.0, **stream),
    }


@pytest.mark.parametrize("name", ["evict", "prefill", "attend", "step", "paged"])
def test_workspaces_are_made_on_the_stream_of_the_call(made, monkeypatch, name):
    monkeypatch.setattr(L, "_stream", lambda stream: None)
    stream = Stream()
    calls(stream)[name]()
    assert made == [stream]
    calls(None)[name]()
    assert made == [stream, None]
