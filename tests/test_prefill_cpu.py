"""What the prefill entry points refuse, at the C interface and in the binding: no GPU needed."""
import ctypes

import pytest
import torch

import paper_2606_31315_gb300 as bp
from paper_2606_31315_gb300 import _build

P, WS = 0x10000, 0x20000  # never read: every call here is refused, or has nothing to do
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 4


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return bp.load()


def _rope(lib, **change):
    a = dict(q=P, qs=4096, k=P, ks=1024, qo=P, qos=4096, ko=P, kos=1024, qw=P, kw=P, cs=P, pos=P, t=5, hq=32, hk=8, d=128,
             r=128, mp=64, il=0, dt=1, eps=1e-6, ws=WS, wsb=256)
    a.update(change)
    return lib.bp_qk_norm_rope(a["q"], a["qs"], a["k"], a["ks"], a["qo"], a["qos"], a["ko"], a["kos"], a["qw"], a["kw"],
                               a["cs"], a["pos"], a["t"], a["hq"], a["hk"], a["d"], a["r"], a["mp"], a["il"], a["dt"],
                               ctypes.c_float(a["eps"]), a["ws"], a["wsb"], None)


def _append(lib, **change):
    a = dict(q=P, qs=6144, k=P, ks=6144, v=P, vs=6144, qo=P, qos=4096, qw=None, kw=None, cs=P, pos=None, kc=P, vc=P, cn=P,
             ck=P, bt=P, pps=10, page=64, np=100, s=3, t=5, hq=32, hk=8, d=128, r=128, mp=64, il=0, dt=1, eps=1e-6, ws=WS,
             wsb=256)
    a.update(change)
    return lib.bp_qkv_append(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["qo"], a["qos"], a["qw"], a["kw"], a["cs"],
                             a["pos"], a["kc"], a["vc"], a["cn"], a["ck"], a["bt"], a["pps"], a["page"], a["np"], a["s"],
                             a["t"], a["hq"], a["hk"], a["d"], a["r"], a["mp"], a["il"], a["dt"], ctypes.c_float(a["eps"]),
                             a["ws"], a["wsb"], None)


def _chunk(lib, **change):
    a = dict(q=P, qs=4096, k=P, v=P, o=P, lse=None, cq=P, ck=P, bt=P, pps=10, page=64, np=100, s=3, t=5, mq=5, mk=600, hq=32,
             hk=8, d=128, dt=1, mask=0, win=0, scale=0.0, ws=WS, wsb=1 << 30)
    a.update(change)
    return lib.bp_chunk_attention_paged(a["q"], a["qs"], a["k"], a["v"], a["o"], a["lse"], a["cq"], a["ck"], a["bt"], a["pps"],
                                        a["page"], a["np"], a["s"], a["t"], a["mq"], a["mk"], a["hq"], a["hk"], a["d"],
                                        a["dt"], a["mask"], a["win"], ctypes.c_float(a["scale"]), a["ws"], a["wsb"], None)


@pytest.mark.parametrize("change,status", [
    (dict(t=-1), INVALID), (dict(hq=-1), INVALID), (dict(q=None), INVALID), (dict(ko=None), INVALID), (dict(pos=None), INVALID),
    (dict(cs=None), INVALID), (dict(mp=0), INVALID), (dict(r=256), INVALID), (dict(r=-16), INVALID), (dict(il=2), INVALID),
    (dict(dt=7), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(qs=4088), INVALID), (dict(qs=4097), INVALID), (dict(q=P + 8), INVALID), (dict(qw=P + 2), INVALID),
    (dict(cs=P + 4), INVALID), (dict(r=24), UNSUPPORTED), (dict(d=100, r=16), UNSUPPORTED), (dict(d=264, r=16), UNSUPPORTED),
    (dict(ws=None), WORKSPACE), (dict(ws=WS + 16), WORKSPACE), (dict(wsb=255), WORKSPACE), (dict(t=0, q=None), OK),
    (dict(hq=0, hk=0, q=None, k=None), OK)])
def test_rope_refusals(lib, change, status):
    assert _rope(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(t=-1), INVALID), (dict(s=-1), INVALID), (dict(kc=None), INVALID), (dict(cn=None), INVALID), (dict(bt=None), INVALID),
    (dict(hk=0), INVALID), (dict(page=48), INVALID), (dict(page=8), INVALID), (dict(np=0), INVALID), (dict(pps=0), INVALID),
    (dict(np=1 << 26), INVALID), (dict(v=None), INVALID), (dict(qo=None), INVALID), (dict(vs=1016), INVALID),
    (dict(ks=6145), INVALID), (dict(vc=P + 2), INVALID), (dict(mp=0), INVALID), (dict(r=40), UNSUPPORTED),
    (dict(d=4, r=0), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(wsb=100), WORKSPACE), (dict(s=0), OK), (dict(t=0), OK)])
def test_append_refusals(lib, change, status):
    assert _append(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(t=-1), INVALID), (dict(q=None), INVALID), (dict(o=None), INVALID), (dict(bt=None), INVALID), (dict(hq=30), INVALID),
    (dict(hk=0), INVALID), (dict(mask=2), INVALID), (dict(dt=9), INVALID), (dict(win=-1), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(page=96), INVALID), (dict(mk=641), INVALID), (dict(mq=0), INVALID), (dict(np=1 << 26), INVALID),
    (dict(qs=4095), INVALID), (dict(qs=4100), INVALID), (dict(q=P + 4), INVALID), (dict(k=P + 8), INVALID),
    (dict(dt=0), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(hq=129, hk=1, qs=129 * 128), UNSUPPORTED),
    (dict(ws=None), WORKSPACE), (dict(ws=WS + 8), WORKSPACE), (dict(wsb=256), WORKSPACE), (dict(t=0, q=None), OK),
    (dict(s=0), OK)])
def test_chunk_refusals(lib, change, status):
    assert _chunk(lib, **change) == status


def test_workspace_size(lib):
    for d in (64, 128):
        n = bp.chunk_attention_workspace_size(3, 100, 32, 8, d)
        # two parts of 256 rows for each of up to 192 CTAs: the columns, (m, l) of a row, 16 bytes a CTA
        assert n == 256 + 192 * (2 * 256 * (4 * d + 8) + 16)
        assert _chunk(lib, d=d, qs=32 * d, wsb=n - 1) == WORKSPACE


def test_binding_refuses_what_is_not_on_the_gpu():
    bp.build()
    x, w = torch.zeros(2, 4, 64), torch.zeros(256, dtype=torch.uint8)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        bp.qk_norm_rope(x, x, None, i, ws=w)
    with pytest.raises(ValueError):
        bp.qk_norm_rope(x.half(), None, None, i, ws=w)
    with pytest.raises(ValueError):
        bp.qkv_append(x, x, x, i, i, i[None], 16, None, ws=w)
    with pytest.raises(ValueError):
        bp.chunk_attention_paged(x, x, x, i, i, i[None], 16, 1, 1, ws=w)
