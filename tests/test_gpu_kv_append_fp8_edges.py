"""kv_append_fp8 where its arguments are at their limits: what is reported is not written, and all else is as by its definition."""
import numpy as np
import pytest
import torch

import paper_2606_31315_gb300 as bp
from _fp8 import Append, random_cache

pytestmark = pytest.mark.gpu


def offsets(lengths, first=0):
    return torch.tensor(first + np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32), dtype=torch.int32, device="cuda")


def make(ctxs, news, page, seed, rows=None, dtype=torch.bfloat16):
    """Two heads of 64; room for the contexts and what is new."""
    g = torch.Generator().manual_seed(seed)
    c = random_cache(g, [a + n for a, n in zip(ctxs, news)], 2, 64, page)
    x = torch.randn(rows or sum(news), 4, 64, generator=g).to(dtype).cuda()
    return c, x[:, :2], x[:, 2:]


def after(c, name, x, ctxs, news, skip=lambda s, t: False, first=0):
    """(codes, scales) by the definition, of rows [first, ...) and without those of sequence s that begin at token t and are to be skipped."""
    ref, at = Append(c[name].view(torch.uint8).cpu().numpy(), c[name + "_scale"].cpu().numpy(), c["page"]), first
    for s, (held, n) in enumerate(zip(ctxs, news)):
        t = 0
        while t < n:
            some = min(c["page"] - (held + t) % c["page"], n - t)
            if not skip(s, t):
                ref(x[at + t:at + t + some].float().cpu().numpy(), held + t, c["table"][s].cpu().numpy())
            t += some
        at += n
    return ref.codes, ref.scale


def same(c, name, codes, scale):
    got = c[name].view(torch.uint8).cpu().numpy()
    assert ((got == codes) | ((got & 127 == 127) & (codes & 127 == 127))).all()
    np.testing.assert_array_equal(c[name + "_scale"].cpu().numpy(), scale)


@pytest.mark.parametrize("new", [3, 40])  # (a warp's unit, and the whole block's)
@pytest.mark.parametrize("page", [16, 64])
def test_a_page_at_a_scale_of_255(new, page):
    """No power of two: that page's head is reported and left, its other head, K or V, and all other pages are written."""
    ctxs, news = [page + 5, 7], [new, new]
    c, k, v = make(ctxs, news, page, 41)
    bad = int(c["table"][0, 1])
    c["k_scale"][bad, 1] = 255
    before = {m: (c[m].view(torch.uint8).cpu().numpy().copy(), c[m + "_scale"].cpu().numpy().copy()) for m in "kv"}
    wanted = {m: after(c, m, x, ctxs, news) for m, x in (("k", k), ("v", v))}
    rows = slice(bad * page, bad * page + page)
    wanted["k"][0][rows, 1], wanted["k"][1][bad, 1] = before["k"][0][rows, 1], 255
    ws = bp.workspace(256, "cuda")
    bp.kv_append_fp8(c["k"], c["k_scale"], c["v"], c["v_scale"], k, v, offsets(news), offsets([a + n for a, n in zip(ctxs, news)]),
                     c["table"], page, ws=ws)
    assert bp.get_status(ws) == 6
    for m in "kv":
        same(c, m, *wanted[m])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("first", [1, 21, 150])
def test_rows_before_the_first_sequence(dtype, page, first):
    """Offsets that begin inside the rows, as for a part of a batch: the rows before are no one's, and those behind."""
    ctxs, news = [200, 30, 5], [90, 1, 17]
    c, k, v = make(ctxs, news, page, 42, first + sum(news) + 70, dtype)
    wanted = {m: after(c, m, x, ctxs, news, first=first) for m, x in (("k", k), ("v", v))}
    ws = bp.workspace(256, "cuda")
    bp.kv_append_fp8(c["k"], c["k_scale"], c["v"], c["v_scale"], k, v, offsets(news, first),
                     offsets([a + n for a, n in zip(ctxs, news)], 7), c["table"], page, ws=ws)
    assert bp.get_status(ws) == 0
    for m in "kv":
        same(c, m, *wanted[m])


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("keys", [0, 1, 16, 50, 99])
def test_fewer_keys_than_new_rows(page, keys):
    """The rows before key 0 are reported and not written; the others are, as the attention reads them."""
    news, lens = [100, 6], [keys, 20]
    c, k, v = make([0, 14], [100, 6], page, 43)
    wanted = {}
    for m, x in (("k", k), ("v", v)):
        ref = Append(c[m].view(torch.uint8).cpu().numpy(), c[m + "_scale"].cpu().numpy(), page)
        ref(x[100 - keys:100].float().cpu().numpy(), 0, c["table"][0].cpu().numpy())
        ref(x[100:].float().cpu().numpy(), 14, c["table"][1].cpu().numpy())
        wanted[m] = (ref.codes, ref.scale)
    ws = bp.workspace(256, "cuda")
    bp.kv_append_fp8(c["k"], c["k_scale"], c["v"], c["v_scale"], k, v, offsets(news), offsets(lens), c["table"], page, ws=ws)
    assert bp.get_status(ws) == 6
    for m in "kv":
        same(c, m, *wanted[m])
