"""What the binding allocates for a call on another stream than the current one belongs to that stream: a workspace
cleared on the current one would be cleared at any time beside the kernel, and memory of the current stream that the
binding lets go of is another tensor's as soon as the call returns.  No GPU needed: the tensors pass for CUDA ones, the
library is a stand-in, and allocations note the stream that is current."""
import contextlib
import types

import pytest
import torch

import paper_2606_31315_gb300 as bp
from paper_2606_31315_gb300 import _binding

SIDE = types.SimpleNamespace(cuda_stream=0x1234)


class OnGpu(torch.Tensor):
    is_cuda = True


def z(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def i32(*shape):
    return z(*shape, dtype=torch.int32)


def f32(*shape):
    return z(*shape, dtype=torch.float32)


CALLS = {  # entry point: what it is given
    "block_attention": lambda: (z(4, 2, 128), z(9, 1, 128), z(9, 1, 128), i32(2), i32(2), 4, 9),
    "block_attention_paged": lambda: (z(4, 2, 128), z(16, 1, 128), z(16, 1, 128), i32(2), i32(2), i32(1, 1), 16, 9, 4, 9),
    "qk_norm_rope": lambda: (z(4, 2, 128), z(4, 1, 128), None, i32(4)),
    "qkv_append": lambda: (z(4, 4, 128), z(16, 1, 128), z(16, 1, 128), i32(2), i32(2), i32(1, 1), 16, None),
    "chunk_attention_paged": lambda: (z(4, 2, 128), z(16, 1, 128), z(16, 1, 128), i32(2), i32(2), i32(1, 1), 16, 4, 9),
    "spec_accept": lambda: (f32(5, 32), f32(4, 32), i32(4), i32(2), 1.0, f32(4), f32(1)),
    "verify_epilogue": lambda: (z(32, 64), z(5, 64), z(4, 64), i32(4), i32(2), 1.0, f32(4), f32(1)),
    "verify_commit": lambda: (i32(1), i32(1), i32(5), i32(2), 64),
    "tau_select": lambda: (f32(3, 4), [2, 4], 4, 0.5, i32(3)),
    "policy_select": lambda: (z(3, 64), z(32, 64), f32(32), z(4, 32), f32(4), i32(4)),
}


@pytest.fixture
def seen(monkeypatch):
    """(streams that were current at an allocation, the library's calls)."""
    now, streams, calls = [None], [], []

    @contextlib.contextmanager
    def stream(s):
        before, now[0] = now[0], s
        yield
        now[0] = before

    for name in ("empty", "zeros", "empty_like"):
        def allocate(*args, _plain=getattr(torch, name), **kwargs):
            streams.append(now[0])
            return _plain(*args, **kwargs).as_subclass(OnGpu)
        monkeypatch.setattr(torch, name, allocate)

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("_workspace_size"):
                    return 4096
                calls.append((name, args))
                return 0
            return call

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(_binding, "load", lambda lib=Library(): lib)
    return streams, calls


@pytest.mark.parametrize("name", CALLS)
def test_defaults_belong_to_the_calls_stream(seen, name):
    streams, calls = seen
    args = CALLS[name]()
    del streams[:]
    getattr(bp, name)(*args, stream=SIDE)
    assert [(c[0], c[1][-1]) for c in calls] == [("bp_" + name, SIDE.cuda_stream)]
    assert streams and all(s is SIDE for s in streams)


def test_without_a_stream_nothing_is_switched(seen, monkeypatch):
    streams, calls = seen
    monkeypatch.setattr(_binding, "_stream", lambda s: 7 if s is None else s.cuda_stream)
    for name, given in CALLS.items():
        getattr(bp, name)(*given())
        assert calls[-1][0] == "bp_" + name and calls[-1][1][-1] == 7
    assert all(s is None for s in streams)


def test_a_workspace_is_cleared_on_its_stream(seen):
    streams, _ = seen
    bp.workspace(256, "cpu")
    bp.workspace(256, "cpu", SIDE)
    assert streams == [None, SIDE]
