"""kv_append_fp8 against its definition in 64 bits: codes and scales have to be equal."""
import math

import numpy as np
import pytest
import torch

import paper_2606_31315_gb300 as bp
from _fp8 import Append, random_cache

pytestmark = pytest.mark.gpu


def offsets(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32), device="cuda")


def both(c, k, v, ctxs, news, ws=None, **more):
    """The call, and its definition; returns the workspace."""
    page, table = c["page"], c["table"].cpu().numpy()
    wanted = []
    for name, x in (("k", k), ("v", v)):
        ref = Append(c[name].view(torch.uint8).cpu().numpy(), c[name + "_scale"].cpu().numpy(), page)
        first = 0
        for s, (n, held) in enumerate(zip(news, ctxs)):
            ref(x[first:first + n].float().cpu().numpy(), held, table[s])
            first += n
        wanted.append(ref)
    ws = bp.workspace(256, "cuda") if ws is None else ws
    bp.kv_append_fp8(c["k"], c["k_scale"], c["v"], c["v_scale"], k, v, offsets(news), offsets([a + n for a, n in zip(ctxs, news)]),
                     c["table"], page, ws=ws, **more)
    for name, ref in zip("kv", wanted):
        got = c[name].view(torch.uint8).cpu().numpy()
        same = (got == ref.codes) | ((got & 127 == 127) & (ref.codes & 127 == 127))
        assert same.all(), (name, np.argwhere(~same)[:3])
        np.testing.assert_array_equal(c[name + "_scale"].cpu().numpy(), ref.scale)
    return ws


def make(ctxs, news, hkv, dim, page, dtype, seed=0):
    """A cache with room for all, that holds ctxs; new rows of sizes that make some scales grow and others not."""
    g = torch.Generator().manual_seed(seed)
    c = random_cache(g, [a + n for a, n in zip(ctxs, news)], hkv, dim, page)
    t = sum(news)
    size = torch.pow(2.0, torch.randint(-8, 5, (t, hkv, 1), generator=g).float())
    k = (torch.randn(t, hkv, dim, generator=g) * size).to(dtype).cuda()
    v = (torch.randn(t, hkv, dim, generator=g) * size.flip(0)).to(dtype).cuda()
    return c, k, v


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hkv,dim", [(8, 128), (2, 64), (1, 16), (3, 80), (1, 256)])
@pytest.mark.parametrize("page", [16, 64])
def test_ragged_blocks(dtype, hkv, dim, page):
    ctxs, news = [0, 5, 16, 63, 100, 31, 64], [1, 11, 16, 2, 0, 50, 130]
    c, k, v = make(ctxs, news, hkv, dim, page, dtype)
    assert bp.get_status(both(c, k, v, ctxs, news)) == 0


@pytest.mark.parametrize("page", [16, 128, 256])
def test_a_prompt_and_single_tokens(page):
    ctxs, news = [700, 30, 0, 99], [600, 1, 333, 1]
    c, k, v = make(ctxs, news, 2, 128, page, torch.bfloat16, seed=1)
    assert bp.get_status(both(c, k, v, ctxs, news)) == 0


def test_token_by_token_and_a_rollback():
    """A page filled a token at a time, its scale growing; rows dropped and written again keep the scale that it grew to."""
    ctxs = [3, 20]
    c, _, _ = make(ctxs, [30, 30], 2, 64, 16, torch.bfloat16, seed=2)
    g = torch.Generator().manual_seed(3)
    ws = bp.workspace(256, "cuda")
    for step in range(24):
        x = (torch.randn(2, 2, 64, generator=g) * 1.5 ** step / 100).to(torch.bfloat16).cuda()
        both(c, x, x * 0.25, ctxs, [1, 1], ws)
        ctxs = [a + 1 for a in ctxs] if step % 5 != 4 else [a - 2 for a in ctxs]
    assert bp.get_status(ws) == 0


def test_ties_zeros_and_ends_of_the_range():
    """Halves between two codes go to the even one; a page of zeros has the least scale; the largest numbers of fp32."""
    news = [32, 16, 16, 16]
    c, k, v = make([0, 0, 0, 0], news, 1, 64, 16, torch.float32, seed=4)
    steps = torch.arange(32 * 64, device="cuda").float()
    k[:32, 0] = ((steps % 512) / 16).view(32, 64) * 8  # every eighth, up to 256: ties of every binade
    v[:32, 0] = -(steps % 64).view(32, 64) * 2.0 ** -140  # numbers below the normal ones
    k[32:48], v[32:48] = 0.0, -0.0
    k[48:64] = torch.finfo(torch.float32).max
    v[48:64] = torch.linspace(-448, 448, 64, device="cuda")
    v[64:80] = torch.nextafter(torch.tensor(448.0), torch.tensor(1e9)).item()
    assert bp.get_status(both(c, k, v, [0] * 4, news)) == 0


def test_what_is_not_finite():
    """Becomes NaN, and no scale's business."""
    c, k, v = make([4, 0], [20, 9], 2, 128, 16, torch.bfloat16, seed=5)
    k[3, 0, 7], k[4, 1, :] = math.inf, math.nan
    v[0, 0, 0], v[21:29] = -math.inf, math.nan
    assert bp.get_status(both(c, k, v, [4, 0], [20, 9])) == 0


def test_views_and_padding():
    """Rows of a packed projection; rows past the last sequence's are not looked at, and nothing is written for them."""
    ctxs, news = [7, 40], [5, 21]
    c, k, v = make(ctxs, news, 4, 64, 16, torch.bfloat16, seed=6)
    packed = torch.full((40, 16, 64), math.nan, device="cuda", dtype=torch.bfloat16)
    packed[:26, 8:12], packed[:26, 12:] = k, v
    assert bp.get_status(both(c, packed[:, 8:12], packed[:, 12:], ctxs, news)) == 0


def test_refused_by_the_device():
    """A page that has no place is reported and not written; the others are."""
    ctxs, news = [10, 30], [12, 12]
    c, k, v = make(ctxs, news, 2, 64, 16, torch.bfloat16, seed=7)
    for bad in (-1, 1 << 24):
        d = {n: x.clone() if torch.is_tensor(x) else x for n, x in c.items()}
        d["table"][0, 1] = bad  # sequence 0's keys 16 to 21
        ws = bp.workspace(256, "cuda")
        bp.kv_append_fp8(d["k"], d["k_scale"], d["v"], d["v_scale"], k, v, offsets(news), offsets([22, 42]), d["table"], 16, ws=ws)
        assert bp.get_status(ws) == 6
        e = {n: x.clone() if torch.is_tensor(x) else x for n, x in c.items()}
        keep = int(c["table"][0, 1])
        both(e, k, v, ctxs, news)
        for n in ("k", "v"):
            e[n].view(torch.uint8)[keep * 16:keep * 16 + 16] = c[n].view(torch.uint8)[keep * 16:keep * 16 + 16]
            e[n + "_scale"][keep] = c[n + "_scale"][keep]
            assert torch.equal(d[n].view(torch.uint8), e[n].view(torch.uint8)) and torch.equal(d[n + "_scale"], e[n + "_scale"])
    # more new rows than keys: before key 0
    ws = bp.workspace(256, "cuda")
    bp.kv_append_fp8(c["k"], c["k_scale"], c["v"], c["v_scale"], k[:12], v[:12], offsets([12]), offsets([5]), c["table"][:1], 16, ws=ws)
    assert bp.get_status(ws) == 6


def test_captured_and_on_another_stream():
    ctxs, news = [10, 30], [12, 12]
    c, k, v = make(ctxs, news, 2, 64, 16, torch.bfloat16, seed=8)
    d = {n: x.clone() if torch.is_tensor(x) else x for n, x in c.items()}
    cu_new, cu_kv, ws = offsets(news), offsets([22, 42]), bp.workspace(256, "cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        bp.kv_append_fp8(d["k"], d["k_scale"], d["v"], d["v_scale"], k, v, cu_new, cu_kv, d["table"], 16, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(d["k_scale"], c["k_scale"])
    graph.replay()
    torch.cuda.synchronize()
    both(c, k, v, ctxs, news)
    assert torch.equal(d["k"].view(torch.uint8), c["k"].view(torch.uint8)) and torch.equal(d["v_scale"], c["v_scale"])
