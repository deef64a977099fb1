"""chunk_attention_paged_fp8 over values whose pages' scales lie far apart: a row is off by what the keys that it sees allow, whatever
lies in pages that are hidden from it."""
import math

import pytest
import torch

import paper_2606_31315_gb300 as bp
from _fp8 import attention, keys_of, random_cache

pytestmark = pytest.mark.gpu


def offsets(lengths):
    return torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


def exponents(c, s, n):
    """The values' exponents of keys 0 .. n - 1 of sequence s: [n, heads]."""
    j = torch.arange(n, device="cuda")
    return c["v_scale"][c["table"][s].long()[j // c["page"]]].double() - 127


def allowance(c, q, news, lens, causal, window):
    """What a row may be off by beyond `attention`'s bound, whose 11 bits of a weight fp16 has down to its least step: a weight times
    its page's scale is off by 2^-29 of the row's largest such product at most (2^-25, half of fp16's least step, where the
    largest is 2^4 at least), for each key that the row sees, times a code of at most 448; and a value by 448 2^-25 of 2^-60 of the
    sequence's largest scale (what its scale is below that is multiplied into it in fp16: off by 2^-25 down to 2^-24, and 0 from 2^-25 on,
    which fp16 does not have).  [tokens, heads]"""
    hkv, out, first = c["k"].shape[1], torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda"), 0
    for s, (b, n) in enumerate(zip(news, lens)):
        k, e = keys_of(c, "k", s, n).nan_to_num(), exponents(c, s, n)
        pos, j = torch.arange(n - b, n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
        seen = (j <= pos) if causal else torch.ones(b, n, dtype=torch.bool, device="cuda")
        if window:
            seen = seen & (j > pos - window)
        for h in range(q.shape[1]):
            kv = h // (q.shape[1] // hkv)
            x = torch.where(seen, q[first:first + b, h].double() @ k[:, kv].T * q.shape[2] ** -0.5, -math.inf)
            products = torch.softmax(x, 1) * torch.pow(2.0, e[:, kv])
            out[first:first + b, h] = n * 2.0 ** -29 * 448 * products.amax(1) + 448 * 2.0 ** -85 * torch.pow(2.0, e[:, kv].max())
        first += b
    return out


def check(c, q, news, lens, causal=True, window=0):
    hkv = c["k"].shape[1]
    ws = bp.workspace(bp.chunk_attention_workspace_size(len(news), len(q), q.shape[1], hkv, q.shape[2]), "cuda")
    out, lse = torch.full(q.shape, 7.0, device="cuda", dtype=torch.bfloat16), torch.full(q.shape[:2], 7.0, device="cuda")
    bp.chunk_attention_paged_fp8(q, c["k"], c["k_scale"], c["v"], c["v_scale"], offsets(news), offsets(lens), c["table"], c["page"],
                                 max(news), max(lens), mask=bp.MASK_CAUSAL if causal else bp.MASK_BIDIR, window=window, out=out,
                                 lse=lse, ws=ws)
    assert bp.get_status(ws) == 0
    o, z, bound, z_bound = attention(c, q, news, lens, causal, window)
    off = (out.double() - o).abs()
    # (bf16's least number is 2^-133: what lies under it is rounded away)
    over = float((off / (bound + allowance(c, q, news, lens, causal, window)[..., None] + 2.0 ** -133)).max())
    z_over = float(((lse.double() - z).abs() / z_bound).max())
    assert over <= 1 and z_over <= 1, (over, z_over)
    return out, o


def make(ctxs, news, hkv, dim, page, seed, exps=None):
    """4 query heads a KV head; the values' exponents random in 120 - exps .. 120 + exps."""
    g = torch.Generator().manual_seed(seed)
    lens = [c + n for c, n in zip(ctxs, news)]
    c = random_cache(g, lens, hkv, dim, page)
    if exps:
        c["v_scale"] = (120 + torch.randint(-exps, exps + 1, c["v_scale"].shape, generator=g)).to(torch.uint8).cuda()
    return c, torch.randn(sum(news), 4 * hkv, dim, generator=g).to(torch.bfloat16).cuda(), lens


def set_pages(c, s, pages, exponent):
    c["v_scale"][c["table"][s, pages].long()] = exponent


NEWS = [[1, 1, 1], [16, 9, 20], [200, 30, 130]]  # (20: block kernel; 200: both streams, and tiles of one)


@pytest.mark.parametrize("news", NEWS)
@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("exps", [12, 40, 100])
def test_scales_far_apart(news, page, dim, exps):
    c, q, lens = make([700, 0, 333], news, 2, dim, page, 21, exps)
    check(c, q, news, lens)


@pytest.mark.parametrize("new", [24, 100])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("far", [20, 40, 110])
def test_large_values_behind_a_row_cost_it_nothing(new, dim, far):
    """Rows in pages of small values, with pages of values 2^far as large after them: in the same tile of 128 keys, and in a later
    one.  The rows before are as exact as if those were not there."""
    for ctx in (30, 120, 250):
        c, q, lens = make([ctx], [new], 2, dim, 16, 22)
        small = (ctx + new // 2) // 16  # of the pages, the rows of whose keys see small values alone
        set_pages(c, 0, slice(0, small), 127 - far // 2)
        set_pages(c, 0, slice(small, None), 127 + far - far // 2)
        out, o = check(c, q, [new], lens)
        before = max(0, small * 16 - ctx)
        assert before > 0 and o[:before].abs().max() < 448 * 2.0 ** -(far // 2)
        if far > 60:  # (that far below the largest scale the values themselves lose bits)
            continue
        # (the bound of `attention`, and the allowance with the largest weight as large as it can be: 1)
        _, _, bound, _ = attention(c, q, [new], lens, True, 0)
        floor = lens[0] * 2.0 ** -29 * 448 * 2.0 ** -(far // 2)
        assert ((out[:before].double() - o[:before]).abs() <= bound[:before] + floor).all()


@pytest.mark.parametrize("new", [1, 24, 100])
def test_large_values_before_a_window(new):
    """Pages that the window has left behind, of values 2^50 as large as those in it, some in its first tile."""
    c, q, lens = make([500], [new], 2, 128, 16, 23)
    set_pages(c, 0, slice(0, (500 - 70) // 16), 127 + 25)
    set_pages(c, 0, slice((500 - 70) // 16, None), 127 - 25)
    out, o = check(c, q, [new], lens, window=64)
    check(c, q, [new], lens, causal=False, window=64)
    assert o.abs().max() < 448 * 2.0 ** -25 and (out != 0).any(-1).all()


@pytest.mark.parametrize("new", [1, 24, 100])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("first", [False, True])
def test_pages_of_zeros_keep_their_weights(new, page, first):
    """As the append leaves them: every code 0, the least scale, 2^-126.  Their keys count in the sum all the same."""
    c, q, lens = make([900], [new], 2, 128, page, 24)
    n = -(-lens[0] // page)
    zeros = torch.arange(0, n // 2) if first else torch.arange(1, n, 3)
    at = c["table"][0, zeros].long()
    c["v_scale"][at] = 1
    rows = (at[:, None] * page + torch.arange(page, device="cuda")).flatten()
    c["v"].view(torch.uint8)[rows] = 0
    check(c, q, [new], lens)


@pytest.mark.parametrize("new", [1, 24, 100])
@pytest.mark.parametrize("low,high", [(0, 2), (1, 254), (250, 254), (100, 101)])
def test_the_ends_of_the_scales(new, low, high):
    """Every other page at either exponent; values of at most 2^-3 where they would leave bf16's range otherwise."""
    c, q, lens = make([400], [new], 2, 64, 16, 25)
    c["v_scale"][0::2], c["v_scale"][1::2] = low, high
    if high > 240:
        c["v"] = torch.where(torch.isnan(c["v"].float()), math.nan, c["v"].float() * 2.0 ** -12).to(torch.float8_e4m3fn)
    check(c, q, [new], lens)


@pytest.mark.parametrize("new", [1, 24, 100])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("power", [4, 12, 16])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_scores(new, dim, power, sign):
    """Scores of up to 2^22 with one key far above (or, all of them negative, far less below 0 than) the others: its value is the
    output, and its score the log-sum-exp."""
    c, q, lens = make([700], [new], 2, dim, 16, 26, 6)
    first = int(c["table"][0, 0]) * 16
    k = torch.zeros(c["k"].shape, device="cuda")
    k[:, :, 0] = 1.0 if sign > 0 else 448.0
    k[first, :, 0] = 448.0 if sign > 0 else 1.0
    c["k"] = k.to(torch.float8_e4m3fn)
    c["k_scale"].fill_(127)
    q.zero_()
    q[:, :, 0] = sign * 2.0 ** power
    ws = bp.workspace(bp.chunk_attention_workspace_size(1, new, 8, 2, dim), "cuda")
    out, lse = bp.chunk_attention_paged_fp8(q, c["k"], c["k_scale"], c["v"], c["v_scale"], offsets([new]), offsets(lens), c["table"], 16,
                                            new, lens[0], lse=torch.empty(q.shape[:2], device="cuda"), ws=ws)
    # (bf16 numbers, but for torch's powers of two in 64 bits, which need not be exact; what the others weigh: 800 2^-447 at most)
    wanted = keys_of(c, "v", 0, 1)[0].repeat_interleave(4, 0).to(torch.bfloat16)
    assert bp.get_status(ws) == 0 and torch.equal(out, wanted.expand_as(out))
    # (a product of three fp32 numbers, one of them rounded before)
    score = sign * 2.0 ** power * (448.0 if sign > 0 else 1.0) * dim ** -0.5
    assert ((lse.double() - score).abs() <= 2.0 ** -21 * abs(score) + 2.0 ** -20).all()


@pytest.mark.parametrize("new", [1, 31, 200])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("exps", [3, 40])
def test_long_contexts_cut_and_merged(new, page, exps):
    """Parts of a row from several CTAs, each with powers of its own."""
    c, q, lens = make([9000, 4000], [new, new], 2, 128, page, 27, exps)
    check(c, q, [new, new], lens)
    check(c, q, [new, new], lens, window=3000)


@pytest.mark.parametrize("new", [1, 24, 100])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("exponent,power", [(0, 115), (1, 114), (254, -130), (250, -126)])
def test_the_ends_of_the_keys_scales(new, page, exponent, power):
    """Keys of 2^(exponent - 127) times a code, queries of 2^power: scores of an ordinary size."""
    c, q, lens = make([300], [new], 2, 64, page, 28)
    c["k_scale"].fill_(exponent)
    q = torch.ldexp(q.double().cpu(), torch.tensor(power)).to(torch.bfloat16).cuda()
    check(c, q, [new], lens)
