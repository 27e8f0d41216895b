"""A call on a stream of the caller's choice that brings no workspace takes one
from that stream's pool. (From another stream's pool it would be handed out
again, and written, while the call's kernels still use it.) Without a GPU: the
library and torch's stream context are stand-ins.
"""

import contextlib

import pytest
import torch


class Side:
    cuda_stream = 4096


@pytest.fixture
def taken(monkeypatch):
    """The binding with a library that launches nothing, and the streams on
    which torch.empty was called."""
    from paper_2606_04945_gb300 import build
    build.build()
    from paper_2606_04945_gb300 import abi
    current, streams, empty, real = [None], [], torch.empty, abi.lib

    class Library:
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith("_workspace_size") else lambda *args: 0

    @contextlib.contextmanager
    def on(stream):
        before, current[0] = current[0], stream
        yield
        current[0] = before

    def recorded(*args, **kw):
        streams.append(current[0])
        return empty(*args, **kw)

    monkeypatch.setattr(abi, "lib", Library())
    monkeypatch.setattr(abi, "_stream", lambda stream: None)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", recorded)
    return abi, streams


def half(*shape):
    return torch.zeros(*shape, dtype=torch.float16)


@pytest.mark.parametrize("stream", [None, Side()])
def test_cache_attention(taken, stream):
    abi, streams = taken
    codes = torch.zeros(2, 1, 16, 64, dtype=torch.uint8)
    cache = abi.KVCache(codes, codes.clone(), torch.zeros(2, 1), torch.zeros(2, 1))
    i = lambda *v: torch.tensor(v, dtype=torch.int32)
    abi.kv_cache_attention(half(3, 64), cache, i(0, 1)[None], i(3), i(0, 3), half(3, 64), max_new=3, max_len=3,
                           stream=stream)
    assert streams == [stream]


@pytest.mark.parametrize("stream", [None, Side()])
@pytest.mark.parametrize("call", ["sgat_quantize_act_dense", "sgat_prepare_weight_dense", "tac_calibrate",
                                  "attention_pv_tac"])
def test_quantised_calls(taken, call, stream):
    abi, streams = taken
    x, byte, f = half(4, 128), torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4)
    args = dict(sgat_quantize_act_dense=(x, None, f, f, x, 128, 0, 0, byte, f),
                sgat_prepare_weight_dense=(x, f, x, byte, f),
                tac_calibrate=(x, x, 64, torch.zeros(2, 64, 64), torch.zeros(2, 64)),
                attention_pv_tac=(x, x, x, 1, byte, f, half(4, 128)))[call]
    getattr(abi, call)(*args, stream=stream)
    assert streams == [stream]
