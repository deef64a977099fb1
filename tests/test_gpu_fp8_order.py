"""What the warps of the attention over a cache in 8 bits hand to one another: scales, row maxima and sums that differ from job to job,
so that one taken before it is there, or from another job, shows as a wrong power of two."""
import pytest
import torch

import paper_2606_31315_gb300 as bp
from _fp8 import attention, random_cache

pytestmark = pytest.mark.gpu


def offsets(lengths):
    return torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


def make(ctxs, news, hq, hkv, dim, page, seed, spread):
    g = torch.Generator().manual_seed(seed)
    lens = [c + n for c, n in zip(ctxs, news)]
    c = random_cache(g, lens, hkv, dim, page, spread)
    # (rows of sizes from 2^-6 to 2: what one row says of its size is not another's)
    size = torch.pow(2.0, torch.randint(-6, 2, (sum(news), hq, 1), generator=g).float())
    q = (torch.randn(sum(news), hq, dim, generator=g) * size).to(torch.bfloat16).cuda()
    return c, q, lens


def check(c, q, news, lens, times=3, cold=()):
    """The call, some times over, against 64 bits; `cold`: tensors that are not in L2 when it begins, the others are."""
    hkv = c["k"].shape[1]
    ws = bp.workspace(bp.chunk_attention_workspace_size(len(news), len(q), q.shape[1], hkv, q.shape[2]), "cuda")
    o, z, bound, z_bound = attention(c, q, news, lens, True, 0)
    # (`bound` is of what fp16 holds in 11 bits.  A weight times 2^5 at least, where the row's largest is 1 at least, is off by half of
    # fp16's least step, 2^-25: 2^-30 of the row's sum for each of its keys, times a value of at most 448 2^(b - 127).  Rows whose
    # scores are hundreds apart have columns with nothing else)
    most = torch.pow(2.0, c["v_scale"].double().amax(0) - 127).repeat_interleave(q.shape[1] // hkv)
    bound = bound + max(lens) * 2.0 ** -30 * 448 * most[None, :, None]
    cu_q, cu_kv = offsets(news), offsets(lens)
    flush = torch.empty(64 << 20, device="cuda")
    for _ in range(times):
        if cold:
            flush.zero_()
            for name, x in c.items():
                if torch.is_tensor(x) and name not in cold:
                    x.view(torch.uint8).sum()
        out, lse = torch.full(q.shape, 7.0, device="cuda", dtype=torch.bfloat16), torch.full(q.shape[:2], 7.0, device="cuda")
        bp.chunk_attention_paged_fp8(q, c["k"], c["k_scale"], c["v"], c["v_scale"], cu_q, cu_kv, c["table"], c["page"], max(news),
                                     max(lens), out=out, lse=lse, ws=ws)
        assert bp.get_status(ws) == 0
        over, z_over = float(((out.double() - o).abs() / bound).max()), float(((lse.double() - z).abs() / z_bound).max())
        assert over <= 1 and z_over <= 1, (over, z_over)


@pytest.mark.parametrize("new", [1, 16, 100])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dim", [64, 128])
def test_scales_of_values_that_come_late(new, page, dim):
    """The values' scales come from memory, all else from L2: they may be the last to be there."""
    ctxs = [3 + 97 * s % 1500 for s in range(24)]
    c, q, lens = make(ctxs, [new] * 24, 8, 2, dim, page, 11, 6)
    check(c, q, [new] * 24, lens, cold=("v_scale", "v"))


@pytest.mark.parametrize("hq,hkv,dim", [(32, 8, 128), (8, 8, 64), (12, 4, 128)])
@pytest.mark.parametrize("more", [1, 9, 30])
def test_tiles_of_one_stream_among_others(hq, hkv, dim, more):
    """Many work tiles to a CTA, by turns of both streams and of one, which both streams then share: the rows' maxima and sums of
    those lie where the others' queries are."""
    tile = 2 * (128 * hkv // hq)
    news = [tile + more if s % 3 else more for s in range(60)]
    c, q, lens = make([17 * s % 300 for s in range(60)], news, hq, hkv, dim, 32, 12, 3)
    check(c, q, news, lens)


@pytest.mark.parametrize("hq,hkv,dim", [(32, 8, 128), (8, 2, 64), (12, 12, 128)])
def test_blocks_of_a_single_key_tile(hq, hkv, dim):
    """Jobs that are over after one tile, many to a CTA: a row's sum is there while its queries' size is still handed on."""
    news = [1 + s % 16 for s in range(200)]
    c, q, lens = make([11 * s % 112 for s in range(200)], news, hq, hkv, dim, 16, 13, 3)
    check(c, q, news, lens)


@pytest.mark.parametrize("hkv,dim", [(2, 128), (4, 64)])
def test_chunks_of_a_single_key_tile(hkv, dim):
    """The same of tiles that two streams share, in the kernel for longer chunks."""
    news = [1 + s % 20 for s in range(199)] + [70]
    c, q, lens = make([11 * s % 100 for s in range(200)], news, 4 * hkv, hkv, dim, 16, 14, 3)
    check(c, q, news, lens)
