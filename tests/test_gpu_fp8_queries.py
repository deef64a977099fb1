"""What chunk_attention_paged_fp8 keeps of its queries: elements from 2^-9 of their row's largest on are exact, smaller ones off by 2^-16
of that at most."""
import math

import pytest
import torch

import paper_2606_31315_gb300 as bp
from _fp8 import attention, keys_of, random_cache

pytestmark = pytest.mark.gpu


def offsets(lengths):
    return torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


def run(c, q, news, lens, window=0):
    hkv = c["k"].shape[1]
    ws = bp.workspace(bp.chunk_attention_workspace_size(len(news), len(q), q.shape[1], hkv, q.shape[2]), "cuda")
    out, lse = bp.chunk_attention_paged_fp8(q, c["k"], c["k_scale"], c["v"], c["v_scale"], offsets(news), offsets(lens), c["table"],
                                            c["page"], max(news), max(lens), window=window, lse=torch.empty(q.shape[:2], device="cuda"), ws=ws)
    assert bp.get_status(ws) == 0
    return out, lse


@pytest.mark.parametrize("news", [[128], [16] * 8])  # (both kernels)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bits", [8, 9, 14, 40])
def test_elements_one_by_one(news, dim, bits):
    """Rows that see one key each, which has one element: the log-sum-exp is the query's element there times it.  Rows of a page
    are of its size, from 2^-90 to 2^90, and their keys the other way round: scores are to be below 2^22."""
    g = torch.Generator().manual_seed(31)
    c = random_cache(g, news, 2, dim, 16)
    sizes = torch.randint(-90, 91, (8,), generator=g)
    k = torch.zeros(c["k"].shape, device="cuda")
    q = torch.pow(2.0, -bits * torch.rand(128, 8, dim, generator=g)) * (torch.randint(0, 2, (128, 8, dim), generator=g) * 2 - 1)
    q = torch.ldexp(q, sizes.repeat_interleave(16)[:, None, None]).to(torch.bfloat16).cuda()
    channel, first = torch.randint(0, dim, (128,), generator=g), 0
    for s, n in enumerate(news):
        for i in range(n):
            page = int(c["table"][s, i // 16])
            k[page * 16 + i % 16, :, channel[first + i]] = 448.0
            c["k_scale"][page] = 127 - int(sizes[(first + i) // 16])
        first += n
    c["k"] = k.to(torch.float8_e4m3fn)
    _, lse = run(c, q, news, news, window=1)
    x = torch.ldexp(q.double(), -sizes.repeat_interleave(16)[:, None, None].cuda())
    element, size = x[torch.arange(128), :, channel.cuda()], x.abs().amax(2)
    scale = 448 * dim ** -0.5
    off = (lse.double() - scale * element).abs()
    # (fp32: a factor of three roundings and the way through powers of two; 2^-20 of a score near 0 in the log-sum-exp)
    exact = 2.0 ** -21 * scale * element.abs() + 2.0 ** -20
    held = element.abs() >= 2.0 ** -9 * size
    assert (off <= exact)[held].all() and (off <= exact + 2.0 ** -16 * scale * size)[~held].all()
    assert held.all() or bits > 8


@pytest.mark.parametrize("new", [1, 24, 100])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("times", [1, 6, 10, 16])
def test_a_large_element_that_meets_no_key(new, dim, times):
    """One element of every row 2^times as large as the others, where the keys are 0: the others alone make the scores."""
    g = torch.Generator().manual_seed(32)
    c = random_cache(g, [300 + new], 2, dim, 16)
    k = c["k"].float()
    k[:, :, 5] = torch.where(torch.isnan(k[:, :, 5]), math.nan, 0.0)
    c["k"] = k.to(torch.float8_e4m3fn)
    q = torch.randn(new, 8, dim, generator=g).to(torch.bfloat16).cuda()
    q[:, :, 5] = 2.0 ** times
    out, lse = run(c, q, [new], [300 + new])
    o, z, bound, z_bound = attention(c, q, [new], [300 + new], True, 0)
    # a score is off by 2^-16 of the row's largest element for each element of a key, a weight by twice as much
    keys = keys_of(c, "k", 0, 300 + new).abs().sum(2).amax(0).repeat_interleave(4)
    most = keys_of(c, "v", 0, 300 + new).abs().amax((0, 2)).repeat_interleave(4)
    off = 2.0 ** -16 * q.double().abs().amax(2) * keys * dim ** -0.5
    assert ((out.double() - o).abs() <= bound + ((2 * off).exp() - 1)[..., None] * most[None, :, None]).all()
    assert ((lse.double() - z).abs() <= z_bound + off).all()


@pytest.mark.parametrize("new", [1, 24, 100])
def test_the_least_and_the_largest_queries(new):
    """Rows of numbers below 2^-119, whose power is not raised any further, of zeros, and next to the largest."""
    g = torch.Generator().manual_seed(33)
    c = random_cache(g, [200 + new], 2, 64, 16)
    q = torch.randn(new, 8, 64, generator=g).to(torch.bfloat16).cuda()
    for times, shift in ((2.0 ** -126, 0), (0.0, 0), (2.0 ** 100, -110), (2.0 ** -110, 100)):
        d = dict(c, k_scale=(c["k_scale"].int() + shift).clamp(0, 254).to(torch.uint8))
        x = (q.double() * times).to(torch.bfloat16)
        out, lse = run(d, x, [new], [200 + new])
        o, z, bound, z_bound = attention(d, x, [new], [200 + new], True, 0)
        assert ((out.double() - o).abs() <= bound).all() and ((lse.double() - z).abs() <= z_bound).all()
