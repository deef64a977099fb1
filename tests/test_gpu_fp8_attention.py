"""chunk_attention_paged_fp8 against 64 bits: both kernels (calls whose rows fit one stream, and others), head layouts, pages, masks
that leave a row empty, scales far apart, what is not a number, and how it is called."""
import math

import pytest
import torch

import paper_2606_31315_gb300 as bp
from _fp8 import attention, random_cache

pytestmark = pytest.mark.gpu


def offsets(lengths):
    return torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


def workspace(news, q, hkv):
    return bp.workspace(bp.chunk_attention_workspace_size(len(news), q.shape[0], q.shape[1], hkv, q.shape[2]), "cuda")


def run(c, q, news, lens, causal=True, window=0, scale=0.0, ws=None, most=None, **more):
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    out = torch.full(q.shape, 7.0, device="cuda", dtype=torch.bfloat16)
    hkv = c["k"].shape[1]
    ws = workspace(news, q, hkv) if ws is None else ws
    bp.chunk_attention_paged_fp8(q, c["k"], c["k_scale"], c["v"], c["v_scale"], offsets(news), offsets(lens), c["table"], c["page"],
                                 most or max(news), max(lens), mask=bp.MASK_CAUSAL if causal else bp.MASK_BIDIR, window=window,
                                 softmax_scale=scale, out=out, lse=lse, ws=ws, **more)
    return out, lse, ws


def check(c, q, news, lens, causal=True, window=0, scale=0.0, **more):
    out, lse, ws = run(c, q, news, lens, causal, window, scale, **more)
    assert bp.get_status(ws) == 0
    o, z, bound, z_bound = attention(c, q, news, lens, causal, window, scale)
    assert torch.equal(torch.isnan(out), torch.isnan(o)) and torch.equal(torch.isnan(lse), torch.isnan(z))
    fine = ~torch.isnan(o)
    over = ((out.double() - o).abs() - bound)[fine]
    assert over.max() <= 0, (float(over.max()), float((out.double() - o)[fine].abs().max()))
    empty = z == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    seen = ~empty & ~torch.isnan(z)
    assert ((lse.double() - z).abs() - z_bound)[seen].max() <= 0
    return out, lse


def make(ctxs, news, hq, hkv, dim, page, seed=0, spread=2):
    g = torch.Generator().manual_seed(seed)
    lens = [c + n for c, n in zip(ctxs, news)]
    c = random_cache(g, lens, hkv, dim, page, spread)
    q = (1.5 * torch.randn(sum(news), hq, dim, generator=g)).to(torch.bfloat16).cuda()
    return c, q, lens


HEADS = [(32, 8, 128), (8, 2, 64), (12, 4, 128), (10, 2, 64), (3, 3, 128), (128, 1, 64)]


@pytest.mark.parametrize("hq,hkv,dim", HEADS)
@pytest.mark.parametrize("page", [16, 64])
def test_single_tokens(hq, hkv, dim, page):
    ctxs = [0, 1, 15, 16, 127, 128, 129, 700, 2000]
    check(*make(ctxs, [1] * len(ctxs), hq, hkv, dim, page)[:2], [1] * len(ctxs), [c + 1 for c in ctxs])


@pytest.mark.parametrize("hq,hkv,dim", HEADS[:5])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 100), (False, 300)])
def test_ragged_blocks(hq, hkv, dim, causal, window):
    ctxs, news = [0, 5, 300, 129, 64, 1111, 0], [9, 16, 1, 0, 25, 17, 1]
    c, q, lens = make(ctxs, news, hq, hkv, dim, 32)
    check(c, q, news, lens, causal, window)


@pytest.mark.parametrize("hq,hkv,dim", HEADS)
@pytest.mark.parametrize("page", [16, 128, 512])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 130)])
def test_chunks_of_prompts(hq, hkv, dim, page, causal, window):
    ctxs, news = [0, 200, 37, 500, 0], [257, 64, 1, 130, 300]
    c, q, lens = make(ctxs, news, hq, hkv, dim, page)
    check(c, q, news, lens, causal, window)


@pytest.mark.parametrize("news", [[1], [31], [33], [64], [65], [300]])
@pytest.mark.parametrize("dim", [64, 128])
def test_long_context_is_cut_and_merged(news, dim):
    c, q, lens = make([9000], news, 8, 2, dim, 64, seed=3)
    check(c, q, news, lens)


@pytest.mark.parametrize("new", [40, 200])
def test_rows_that_see_no_key(new):
    """Fewer keys than new tokens: the first rows stand before key 0.  Zeros, and -inf."""
    c, q, _ = make([0, 10], [new, 5], 8, 2, 128, 16)
    out, lse = check(c, q, [new, 5], [new - 30, 15])
    assert (out[:30] == 0).all() and (lse[:30] == -math.inf).all()
    out, lse = check(c, q, [new, 5], [0, 15])
    assert (out[:new] == 0).all()


@pytest.mark.parametrize("new", [16, 150])
@pytest.mark.parametrize("spread", [8, 30])
def test_scales_far_apart(new, spread):
    """Pages whose scales lie up to 2^60 apart: a row's output is off by its bound, for 8 powers, or by as much of the largest
    values' share (what is 2^-24 of a tile's largest value and 2^-25 of a weight at its power is rounded away)."""
    c, q, lens = make([500, 77], [new, new], 8, 2, 128, 16, seed=5, spread=spread)
    q = (q.double() * 2.0 ** (-spread)).to(torch.bfloat16) if spread > 8 else q * 2.0 ** -6
    if spread <= 8:
        check(c, q, [new, new], lens)
        return
    out, lse, ws = run(c, q, [new, new], lens)
    o, z, bound, z_bound = attention(c, q, [new, new], lens, True, 0)
    assert bp.get_status(ws) == 0 and torch.isfinite(out).all()
    first = 0
    for s, n in enumerate(lens):
        from _fp8 import keys_of
        top = keys_of(c, "v", s, n).abs().amax((0, 2)).repeat_interleave(4)  # of a head
        rows = slice(first, first + new)
        assert ((out[rows].double() - o[rows]).abs() <= bound[rows] + 2.0 ** -20 * top[None, :, None]).all()
        first += new
    assert ((lse.double() - z).abs() <= z_bound).all()


@pytest.mark.parametrize("exponent", [0, 1, 60, 135, 180, 200])
def test_extreme_scales(exponent):
    c, q, lens = make([300], [20], 4, 1, 128, 64)
    c["v_scale"].fill_(exponent)
    c["k_scale"].fill_(max(1, 240 - exponent) if exponent > 100 else 120)
    q = (q.double() * 2.0 ** (-exponent if exponent < 1 else min(0, exponent - 120))).to(torch.bfloat16)
    out, lse, ws = run(c, q, [20], lens)
    o, z, bound, z_bound = attention(c, q, [20], lens, True, 0)
    tiny = 2.0 ** -133  # bf16's least number: what lies under it is rounded away
    # (below 2^-112 the values' power is not lowered any more, and they lose bits)
    assert ((out.double() - o).abs() <= bound + tiny + (2.0 ** -130 if exponent < 15 else 0)).all()
    assert ((lse.double() - z).abs() <= z_bound).all()


@pytest.mark.parametrize("new", [16, 200])
@pytest.mark.parametrize("where", ["key", "value", "query"])
def test_what_is_no_number_is_seen_by_its_rows_alone(new, where):
    c, q, lens = make([100, 40], [new, new], 8, 2, 128, 16, seed=7)
    page = c["page"]
    for key, head in ((100 + new // 2, 0), (3, 1)) if where != "query" else ():
        row = int(c["table"][0, key // page]) * page + key % page
        c[where[0]].view(torch.uint8)[row, head, 77] = 0x7f if head else 0xff
    if where == "query":
        q[5, 3, 100], q[7, 2, 0] = math.nan, math.inf
    out, _ = check(c, q, [new, new], lens)
    assert torch.isnan(out).any() and torch.isfinite(out[new:]).all()
    if where != "query":
        assert torch.isfinite(out[:new // 2, :4]).all()
        check(c, q, [new, new], lens, window=16)


def test_a_score_that_overflows():
    c, q, lens = make([60], [4], 2, 2, 64, 16)
    c["k_scale"].fill_(250)
    q[1] = q[1] * 1e30
    out, lse, _ = run(c, q, [4], lens)
    assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()


@pytest.mark.parametrize("new", [8, 100])
def test_strided_queries_scale_and_reuse(new):
    """Views of a packed projection, a softmax scale of its own, one workspace for calls of both kernels in turn."""
    c, q, lens = make([333, 90], [new, new], 8, 2, 128, 64, seed=2)
    packed = torch.randn(2 * new, 12, 128, device="cuda").to(torch.bfloat16)
    packed[:, :8] = q
    ws = workspace([new, new], q, 2)
    a, _ = check(c, packed[:, :8], [new, new], lens, scale=0.02, ws=ws)
    for most in (100, 100, 31 if new < 31 else 100):
        b, _ = check(c, q, [new, new], lens, scale=0.02, ws=ws, most=max(most, new))
        if most > 31 or new > 31:
            continue
        assert torch.equal(a, b)


def test_same_results_every_time():
    c, q, lens = make([5000, 3, 800], [16, 16, 16], 32, 8, 128, 64, seed=4)
    a, la, ws = run(c, q, [16] * 3, lens)
    for _ in range(5):
        b, lb, _ = run(c, q, [16] * 3, lens, ws=ws)
        assert torch.equal(a, b) and torch.equal(la, lb)


def test_graph_replayed_over_other_lengths():
    """Captured with bounds, replayed over other lengths and on another stream than the one it was captured on."""
    news = [16, 5]
    c, q, lens = make([600, 300], news, 8, 2, 128, 64, seed=6)
    cu_q, cu_kv = offsets(news), offsets(lens)
    out, ws = torch.empty_like(q), workspace(news, q, 2)
    call = lambda: bp.chunk_attention_paged_fp8(q, c["k"], c["k_scale"], c["v"], c["v_scale"], cu_q, cu_kv, c["table"], 64, 31,  # noqa: E731
                                                640, out=out, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for part in (lens, [200, 305], [16, 5], [130, 40]):
        cu_kv.copy_(offsets(part))
        graph.replay()
        torch.cuda.synchronize()
        o, _, bound, _ = attention(c, q, news, part, True, 0)
        assert ((out.double() - o).abs() <= bound).all() and bp.get_status(ws) == 0


def test_two_calls_at_once():
    made = [make([700, 20], [n, n], 8, 2, 128, 16, seed=n) for n in (8, 90)]
    streams = [torch.cuda.Stream() for _ in made]
    spaces = [workspace([q.shape[0] // 2] * 2, q, 2) for _, q, _ in made]
    wanted = [run(c, q, [q.shape[0] // 2] * 2, lens)[0] for c, q, lens in made]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, (c, q, lens) in enumerate(made):
            with torch.cuda.stream(streams[i]):
                got[i].append(run(c, q, [q.shape[0] // 2] * 2, lens, ws=spaces[i])[0])
    torch.cuda.synchronize()
    for want, outs in zip(wanted, got):
        assert all(torch.equal(want, o) for o in outs)


def test_what_the_device_refuses():
    """A page outside the pool, a sequence past its table row or the bounds, a scale of 255: reported, and nothing else broken."""
    c, q, lens = make([100, 50], [4, 4], 8, 2, 128, 16)
    ws = workspace([4, 4], q, 2)

    def status(change):
        d = dict(c, **{k: v.clone() for k, v in c.items() if torch.is_tensor(v)})
        change(d)
        run(d, q, [4, 4], lens, ws=ws)
        return bp.get_status(ws)

    assert status(lambda d: None) == 0
    for bad in (-1, 1 << 20):
        assert status(lambda d: d["table"][0].__setitem__(2, bad)) == 6
    for name in ("k_scale", "v_scale"):
        assert status(lambda d: d[name][c["table"][1, 0].long()].__setitem__(1, 255) or d[name].__setitem__((int(c["table"][1, 0]), 1), 255)) == 6
    out, _, _ = run(c, q, [4, 4], lens, ws=ws, most=4)
    assert bp.get_status(ws) == 0
    bp.chunk_attention_paged_fp8(q, c["k"], c["k_scale"], c["v"], c["v_scale"], offsets([4, 4]), offsets(lens), c["table"], 16, 4, 60,
                                 ws=ws)
    assert bp.get_status(ws) == 6
    check(c, q, [4, 4], lens, ws=ws)


def test_no_sequences_and_no_tokens():
    c, q, lens = make([100], [4], 8, 2, 128, 16)
    o, _ = bp.chunk_attention_paged_fp8(q[:0], c["k"], c["k_scale"], c["v"], c["v_scale"], offsets([0]), offsets([100]), c["table"], 16, 1, 100)
    assert o.shape == (0, 8, 128)


@pytest.mark.parametrize("new", [16, 100])
def test_a_cache_past_4_gib(new):
    """Pages at the far end of pools of 4.6 GB each: append and attention by 64-bit offsets."""
    hkv, dim, page = 8, 128, 64
    pages = (4600 << 20) // (hkv * dim * page)
    c = dict(page=page)
    for name in "kv":
        c[name] = torch.empty(pages * page, hkv, dim, dtype=torch.uint8, device="cuda")
        c[name + "_scale"] = torch.full((pages, hkv), 120, dtype=torch.uint8, device="cuda")
    c["table"] = torch.tensor([[pages - 1, 5, pages - 2, pages - 7]], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(9)
    rows = torch.randn(200, 2 * hkv, dim, generator=g).to(torch.bfloat16).cuda()
    ws = bp.workspace(256, "cuda")
    bp.kv_append_fp8(c["k"], c["k_scale"], c["v"], c["v_scale"], rows[:, :hkv], rows[:, hkv:], offsets([200]), offsets([200]), c["table"],
                     page, ws=ws)
    assert bp.get_status(ws) == 0
    small = dict(page=page, table=torch.arange(4, dtype=torch.int32, device="cuda")[None])
    for name in "kv":
        at = (c["table"][0].long()[:, None] * page + torch.arange(page, device="cuda")).flatten()
        small[name], small[name + "_scale"] = c[name][at].clone(), c[name + "_scale"][c["table"][0].long()].clone()
        near = rows[:, :hkv] if name == "k" else rows[:, hkv:]
        value = small[name].view(torch.float8_e4m3fn)[:200].float() * torch.exp2(small[name + "_scale"].float() - 127).repeat_interleave(page, 0)[:200, :, None]
        # (a code is off by half a step, 2^-4 of it, or by 2^-10 of a scale that takes the page's largest number below 448)
        assert ((value - near.float()).abs() <= 2.0 ** -4 * near.float().abs() + 2.0 ** -10 * 2.0 ** -6).all()
    q = torch.randn(new, 32, dim, generator=g).to(torch.bfloat16).cuda()
    far, _, _ = run(c, q, [new], [200])
    assert torch.equal(far, run(small, q, [new], [200])[0])


@pytest.mark.parametrize("new", [1, 20, 120])
@pytest.mark.parametrize("hkv,dim", [(2, 128), (1, 64)])
def test_maxima_that_grow(new, hkv, dim):
    """A row's scores rise or fall from one tile of 128 keys to the next, by less and by more than a maximum may be outgrown; the rows
    of a warp differ, so that some move for the others' sake."""
    c, q, lens = make([1900], [new], 4 * hkv, hkv, dim, 64, seed=5, spread=6)
    g = torch.Generator().manual_seed(6)
    keys = torch.arange(lens[0])
    at = (c["table"][0].cpu().long()[keys // 64] * 64 + keys % 64).cuda()
    k = 0.5 * torch.randn(lens[0], hkv, dim, generator=g)
    k[:, :, 0] = (keys // 128 + 1).float()[:, None]  # (up to 16: e4m3 numbers)
    c["k"].view(torch.uint8)[at] = k.to(torch.float8_e4m3fn).view(torch.uint8).cuda()
    c["k_scale"].fill_(127)
    steps = torch.tensor([3.0, -3.0, 9.0, 9.9, -9.0, 11.0, -11.0, 40.0, 0.0, -40.0, 5.0])  # of a tile, in powers of two
    row = torch.arange(q.shape[0] * q.shape[1]).view(q.shape[0], q.shape[1])
    q[:, :, 0] = (steps[row % len(steps)] * math.sqrt(dim) * math.log(2)).to(torch.bfloat16).cuda()
    check(c, q, [new], lens)
    check(c, q, [new], lens, window=700)
