"""What the entry points of the cache in 8 bits refuse, at the C interface and in the binding, and where the binding allocates: no
GPU needed."""
import contextlib
import ctypes
import types

import numpy as np
import pytest
import torch

import paper_2606_31315_gb300 as bp
from _fp8 import VALUES, codes_of, least_exponent
from paper_2606_31315_gb300 import _binding, _build

P, WS = 0x10000, 0x20000  # never read: every call here is refused, or has nothing to do
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 4


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return bp.load()


def _append(lib, **change):
    a = dict(kc=P, ks=P, vc=P, vs=P, k=P, kst=1024, v=P, vst=6144, cn=P, ck=P, bt=P, pps=10, page=64, np=100, s=3, t=5, hk=8, d=128,
             dt=1, ws=WS, wsb=256)
    a.update(change)
    return lib.bp_kv_append_fp8(a["kc"], a["ks"], a["vc"], a["vs"], a["k"], a["kst"], a["v"], a["vst"], a["cn"], a["ck"], a["bt"],
                                a["pps"], a["page"], a["np"], a["s"], a["t"], a["hk"], a["d"], a["dt"], a["ws"], a["wsb"], None)


def _attend(lib, **change):
    a = dict(q=P, qs=4096, k=P, ks=P, v=P, vs=P, o=P, lse=None, cq=P, ck=P, bt=P, pps=10, page=64, np=100, s=3, t=5, mq=5, mk=600,
             hq=32, hk=8, d=128, dt=1, mask=0, win=0, scale=0.0, ws=WS, wsb=1 << 30)
    a.update(change)
    return lib.bp_chunk_attention_paged_fp8(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["o"], a["lse"], a["cq"], a["ck"],
                                            a["bt"], a["pps"], a["page"], a["np"], a["s"], a["t"], a["mq"], a["mk"], a["hq"],
                                            a["hk"], a["d"], a["dt"], a["mask"], a["win"], ctypes.c_float(a["scale"]), a["ws"],
                                            a["wsb"], None)


def _pages(lib, **change):
    a = dict(bt=P, old=P, new=P, free=P, nf=P, s=3, pps=10, page=64, np=100, t=5, pos=P, slots=P, cn=P, ck=P, miss=P, ws=WS, wsb=256)
    a.update(change)
    return lib.bp_pages_update(a["bt"], a["old"], a["new"], a["free"], a["nf"], a["s"], a["pps"], a["page"], a["np"], a["t"], a["pos"],
                               a["slots"], a["cn"], a["ck"], a["miss"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("change,status", [
    (dict(t=-1), INVALID), (dict(s=-1), INVALID), (dict(kc=None), INVALID), (dict(ks=None), INVALID), (dict(vs=None), INVALID),
    (dict(v=None), INVALID), (dict(cn=None), INVALID), (dict(bt=None), INVALID), (dict(hk=0), INVALID), (dict(page=48), INVALID),
    (dict(page=8), INVALID), (dict(np=0), INVALID), (dict(pps=0), INVALID), (dict(np=1 << 26), INVALID), (dict(dt=5), INVALID),
    (dict(kst=1016), INVALID), (dict(kst=1028), INVALID), (dict(vst=6146), INVALID), (dict(dt=0, kst=1026), INVALID),
    (dict(kc=P + 8), INVALID), (dict(k=P + 2), INVALID), (dict(d=24, hk=1, kst=24, vst=24), UNSUPPORTED), (dict(ws=None), WORKSPACE),
    (dict(ws=WS + 16), WORKSPACE), (dict(wsb=255), WORKSPACE), (dict(s=0), OK), (dict(t=0, k=None), OK)])
def test_append_refusals(lib, change, status):
    assert _append(lib, **change) == status


@pytest.mark.parametrize("change", [dict(d=1 << 19, hk=1, kst=1 << 19, vst=1 << 19, page=16), dict(d=1 << 20, hk=1, kst=1 << 20, vst=1 << 20, page=16),
                                    dict(d=1 << 18, hk=1, kst=1 << 18, vst=1 << 18, page=16), dict(d=1024, kst=8192, vst=8192, page=1 << 20)])
def test_append_refuses_pages_of_too_many_pieces(lib, change):
    assert _append(lib, **change) == UNSUPPORTED


@pytest.mark.parametrize("change", [dict(np=(1 << 30) + 1), dict(t=(1 << 30) + 1), dict(t=(1 << 31) - 1)])
def test_pages_refuses_numbers_past_2_30(lib, change):
    assert _pages(lib, **change) == UNSUPPORTED


@pytest.mark.parametrize("change,status", [
    (dict(t=-1), INVALID), (dict(q=None), INVALID), (dict(ks=None), INVALID), (dict(vs=None), INVALID), (dict(o=None), INVALID),
    (dict(bt=None), INVALID), (dict(hq=30), INVALID), (dict(hk=0), INVALID), (dict(mask=2), INVALID), (dict(dt=9), INVALID),
    (dict(win=-1), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(page=96), INVALID),
    (dict(mk=641), INVALID), (dict(mq=0), INVALID), (dict(np=1 << 26), INVALID), (dict(qs=4095), INVALID), (dict(qs=4100), INVALID),
    (dict(q=P + 4), INVALID), (dict(k=P + 8), INVALID), (dict(dt=0), UNSUPPORTED), (dict(d=96), UNSUPPORTED),
    (dict(hq=129, hk=1, qs=129 * 128), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(wsb=256), WORKSPACE), (dict(t=0, q=None), OK),
    (dict(s=0, ks=None), OK)])
def test_attention_refusals(lib, change, status):
    assert _attend(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(t=-1), INVALID), (dict(s=-1), INVALID), (dict(np=-1), INVALID), (dict(s=0), INVALID), (dict(bt=None), INVALID),
    (dict(old=None), INVALID), (dict(new=None), INVALID), (dict(free=None), INVALID), (dict(nf=None), INVALID), (dict(pps=0), INVALID),
    (dict(page=24), INVALID), (dict(pps=1 << 26), INVALID), (dict(s=16385), UNSUPPORTED), (dict(ws=None), WORKSPACE),
    (dict(ws=WS + 64), WORKSPACE), (dict(wsb=128), WORKSPACE)])
def test_pages_refusals(lib, change, status):
    assert _pages(lib, **change) == status


class OnGpu(torch.Tensor):
    is_cuda = True


def z(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def i32(*shape):
    return z(*shape, dtype=torch.int32)


def u8(*shape):
    return z(*shape, dtype=torch.uint8)


APPEND = lambda: [u8(32, 1, 128), u8(2, 1), u8(32, 1, 128), u8(2, 1), z(4, 1, 128), z(4, 1, 128), i32(2), i32(2), i32(1, 1), 16]  # noqa: E731
ATTEND = lambda: [z(4, 2, 128), u8(32, 1, 128), u8(2, 1), u8(32, 1, 128), u8(2, 1), i32(2), i32(2), i32(1, 1), 16, 4, 9]  # noqa: E731
PAGES = lambda: [i32(2, 4), i32(2), i32(2), i32(9), i32(1), 16, 7]  # noqa: E731


@pytest.fixture
def seen(monkeypatch):
    """(streams that were current at an allocation, the library's calls)."""
    now, streams, calls = [None], [], []

    @contextlib.contextmanager
    def stream(s):
        before, now[0] = now[0], s
        yield
        now[0] = before

    for name in ("empty", "zeros"):
        def allocate(*args, _plain=getattr(torch, name), **kwargs):
            streams.append(now[0])
            kwargs.pop("device", None)
            return _plain(*args, **kwargs).as_subclass(OnGpu)
        monkeypatch.setattr(torch, name, allocate)

    class Lib:
        def __getattr__(self, name):
            return (lambda *a: 1 << 20) if name.endswith("size") else (lambda *a: calls.append((name, a)) or 0)

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(_binding, "load", lambda: Lib())
    return streams, calls


@pytest.mark.parametrize("name,given", [("kv_append_fp8", APPEND), ("chunk_attention_paged_fp8", ATTEND), ("pages_update", PAGES)])
def test_allocations_belong_to_the_calls_stream(seen, name, given):
    streams, calls = seen
    args = given()
    streams.clear()
    side = types.SimpleNamespace(cuda_stream=0x1234)
    getattr(bp, name)(*args, stream=side)
    assert streams and all(s is side for s in streams)
    assert calls[0][0] == "bp_" + name and calls[0][1][-1] == 0x1234


@pytest.mark.parametrize("name,given,place,bad", [
    ("kv_append_fp8", APPEND, 0, lambda: z(32, 1, 128)), ("kv_append_fp8", APPEND, 1, lambda: u8(3, 1)),
    ("kv_append_fp8", APPEND, 3, lambda: z(2, 1, dtype=torch.float32)), ("kv_append_fp8", APPEND, 4, lambda: z(4, 1, 128, dtype=torch.float16)),
    ("kv_append_fp8", APPEND, 5, lambda: z(4, 2, 128)), ("kv_append_fp8", APPEND, 6, lambda: i32(3)), ("kv_append_fp8", APPEND, 9, lambda: 12),
    ("kv_append_fp8", APPEND, 8, lambda: torch.ones(1, 1, dtype=torch.int32)), ("kv_append_fp8", APPEND, 2, lambda: u8(64, 1, 128)[::2]),
    ("chunk_attention_paged_fp8", ATTEND, 0, lambda: z(4, 2, 64)), ("chunk_attention_paged_fp8", ATTEND, 0, lambda: z(4, 2, 128, dtype=torch.float32)),
    ("chunk_attention_paged_fp8", ATTEND, 2, lambda: i32(2, 1)), ("chunk_attention_paged_fp8", ATTEND, 5, lambda: i32(4)),
    ("pages_update", PAGES, 1, lambda: i32(3)), ("pages_update", PAGES, 4, lambda: i32(2)), ("pages_update", PAGES, 0, lambda: z(2, 4, dtype=torch.int64))])
def test_binding_refusals(seen, name, given, place, bad):
    args = given()
    args[place] = bad()
    with pytest.raises(ValueError):
        getattr(bp, name)(*args)
    assert not seen[1]


def test_binding_refusals_of_outputs(seen):
    for more in (dict(positions=i32(6)), dict(slots=i32(7)), dict(cu_new=i32(2)), dict(missing=i32(2))):
        with pytest.raises(ValueError):
            bp.pages_update(*PAGES(), **more)
    with pytest.raises(ValueError):
        bp.pages_update(*PAGES()[:-1], None, positions=i32(7))
    with pytest.raises(ValueError):
        bp.chunk_attention_paged_fp8(*ATTEND(), lse=z(4, 2))
    assert not seen[1]


def test_the_reference_is_e4m3():
    """Its table and its rounding against torch's type, over every bf16 number that it holds."""
    codes = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(codes.view(torch.float8_e4m3fn).double().numpy(), VALUES)
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    x = x[x.abs() <= 448]
    got = torch.from_numpy(codes_of(x.double().numpy()))
    assert torch.equal(got.view(torch.float8_e4m3fn).float(), x.to(torch.float8_e4m3fn).float())
    assert least_exponent(448.0) == 127 and least_exponent(448.5) == 128 and least_exponent(0.0) == 1 and least_exponent(1.0) == 119
