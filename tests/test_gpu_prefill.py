"""The prefill operators against plain forms in 64 bits: norms and rotation of queries and keys, the same on the way into
a paged cache, and attention of chunks of new tokens over it.

Tolerances are per element and derived from what the kernels round (u = 2^-8, the unit roundoff of bf16's 8 bits,
e = 2^-24 that of fp32):
  norm and rotation   fp32 throughout: the mean of squares, its root, two products and a rotation of two products and a
                      sum stay within 16 e of |a| + |b|, the pair's sizes after the norm; a bf16 output adds u of itself
  attention           a weight is rounded to bf16 (u), its exponent carries the fp32 error of a product of 128 terms
                      (below 5e-4 for these inputs: 128 e times |q| |k| scale < 35, doubled for weight and sum), and
                      the output is rounded (u): (u + 1e-3) sum_j p_j |v_j| + u |o|; log-sum-exp within 5e-4
"""
import math

import numpy as np
import pytest
import torch

import paper_2606_31315_gb300 as bp

pytestmark = pytest.mark.gpu

U, E = 2.0 ** -8, 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    bp.build()
    bp.load()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _offsets(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")


def _table(positions, rotary):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * 1e4 ** (
        -torch.arange(rotary // 2, dtype=torch.float64) / max(1, rotary // 2))
    return torch.cat([angle.cos(), angle.sin()], 1).float().cuda()


def _turned(x, weight, table, pos, interleaved, eps):
    """(the exact result, |a| + |b| of every element's pair) in 64 bits."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    r = 0 if table is None else table.shape[1]
    if r == 0:
        return x, x.abs()
    row = table[pos.long()].double()[:, None]
    c, s = row[..., :r // 2], row[..., r // 2:]
    i = torch.arange(r // 2, device="cuda")
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
    a, b = x[..., ia], x[..., ib]
    out, size = x.clone(), x.abs()
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return out, size


def _near_turned(got, ref):
    out, size = ref
    tol = 16 * E * size + (U * out.abs() * 1.001 if got.dtype == torch.bfloat16 else 0.0)
    err = (got.double() - out).abs()
    assert torch.all(err <= tol + 1e-37), float((err - tol).max())


TURNS = [  # head_dim, rotary_dim, interleaved, norm
    (128, 128, False, True), (128, 64, False, True), (128, 128, True, True), (64, 64, False, True), (64, 32, True, False),
    (96, 96, False, True), (80, 16, False, True), (256, 128, False, True), (16, 16, True, True), (128, 0, False, True),
    (8, 0, False, False)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,rotary,interleaved,norm", TURNS)
@pytest.mark.parametrize("tokens,hq,hkv", [(1, 32, 8), (7, 5, 1), (1500, 6, 2)])
def test_norm_and_rotation(dtype, dim, rotary, interleaved, norm, tokens, hq, hkv):
    g = _gen(tokens + dim)
    q = torch.randn(tokens, hq, dim, device="cuda", generator=g).to(dtype)
    k = (3 * torch.randn(tokens, hkv, dim, device="cuda", generator=g)).to(dtype)
    q[0, 0] = 0  # a head of zeros: eps keeps its norm finite
    qw, kw = [(1 + torch.randn(dim, device="cuda", generator=g)).to(dtype) if norm else None for _ in range(2)]
    table = _table(500, rotary) if rotary else None
    pos = torch.randint(0, 500, (tokens,), device="cuda", generator=g).to(torch.int32)
    ws = bp.workspace(256, "cuda")
    qo, ko = bp.qk_norm_rope(q, k, table, pos, q_weight=qw, k_weight=kw, interleaved=interleaved, eps=1e-5, ws=ws)
    assert bp.get_status(ws) == 0
    _near_turned(qo, _turned(q, qw, table, pos, interleaved, 1e-5))
    _near_turned(ko, _turned(k, kw, table, pos, interleaved, 1e-5))


def test_norm_and_rotation_of_views_and_in_place():
    """Views of a packed projection, queries alone, keys alone, and outputs over the inputs."""
    g = _gen(1)
    packed = torch.randn(37, 12, 128, device="cuda", generator=g).to(torch.bfloat16)
    q, k = packed[:, :8], packed[:, 8:10]
    w = (1 + 0.1 * torch.randn(128, device="cuda", generator=g)).to(torch.bfloat16)
    table, pos = _table(64, 128), torch.arange(37, device="cuda", dtype=torch.int32)
    rq, rk = _turned(q, w, table, pos, False, 1e-6), _turned(k, w, table, pos, False, 1e-6)
    ws = bp.workspace(256, "cuda")
    qo, none = bp.qk_norm_rope(q, None, table, pos, q_weight=w, ws=ws)
    assert none is None
    _near_turned(qo, rq)
    none, ko = bp.qk_norm_rope(None, k, table, pos, k_weight=w, ws=ws)
    assert none is None
    _near_turned(ko, rk)
    rest = packed[:, 10:].clone()
    bp.qk_norm_rope(q, k, table, pos, q_weight=w, k_weight=w, q_out=q, k_out=k, ws=ws)
    _near_turned(packed[:, :8], rq)
    _near_turned(packed[:, 8:10], rk)
    assert torch.equal(packed[:, 10:], rest) and bp.get_status(ws) == 0


def test_a_position_outside_the_table_is_reported():
    x = torch.ones(3, 2, 64, device="cuda")
    out = torch.full_like(x, 7.0)
    ws = bp.workspace(256, "cuda")
    table = _table(10, 64)
    bp.qk_norm_rope(x, None, table, torch.tensor([0, 10, -1], dtype=torch.int32, device="cuda"), q_out=out, ws=ws)
    assert bp.get_status(ws) == bp._binding.BP_ERR_DEVICE_FLAG
    assert torch.all(out[1:] == 7.0) and torch.all(out[0] != 7.0)


def _paged(lens, page, hkv, dim, dtype, g, held):
    """A pool whose rows are not numbers, but for the first held[s] keys of every sequence; a table of shuffled pages."""
    need = [-(-n // page) for n in lens]
    order = torch.randperm(sum(need) + 2, generator=torch.Generator().manual_seed(page)).to(torch.int32)
    table = torch.full((len(lens), max(1, max(need))), -5, dtype=torch.int32)  # entries no sequence uses
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    table = table.cuda()
    rows = (sum(need) + 2) * page
    caches = [torch.full((rows, hkv, dim), math.nan, device="cuda", dtype=dtype) for _ in range(2)]
    keys = []
    for s, n in enumerate(lens):
        j = torch.arange(n, device="cuda")
        r = table[s].long()[j // page] * page + j % page
        keys.append(r)
        for c in caches:
            c[r[:held[s]]] = torch.randn(held[s], hkv, dim, device="cuda", generator=g).to(dtype)
    return caches, table, keys


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ctx,new", [((0,), (1,)), ((5, 100, 0, 33, 63), (3, 1, 70, 0, 1)), ((40,) * 45, (2, 0, 1) * 15),
                                     ((1000, 7), (600, 400))])
@pytest.mark.parametrize("page,packed", [(16, True), (64, False)])
def test_append(dtype, ctx, new, page, packed):
    """Keys normed and rotated, values as they are, each at its key's place and nothing else touched; the queries; rows of
    padding behind the last sequence left out."""
    g = _gen(len(ctx))
    hq, hkv, dim, pad = 4, 2, 64, 3
    total = sum(new)
    (kc, vc), table, keys = _paged([c + n for c, n in zip(ctx, new)], page, hkv, dim, dtype, g, ctx)
    qkv = torch.randn(total + pad, hq + 2 * hkv, dim, device="cuda", generator=g).to(dtype)
    kw = (1 + 0.1 * torch.randn(dim, device="cuda", generator=g)).to(dtype)
    tab = _table(max(c + n for c, n in zip(ctx, new)), 32)
    q, k, v = qkv.split([hq, hkv, hkv], 1)
    rows = torch.cat([r[c:] for r, c in zip(keys, ctx)])
    pos = torch.cat([torch.arange(c, c + n, device="cuda") for c, n in zip(ctx, new)])
    want_k, want_v = kc.clone(), vc.clone()
    want_v[rows] = v[:total]
    ws = bp.workspace(256, "cuda")
    qo = torch.full((total + pad, hq, dim), 7.0, device="cuda", dtype=dtype)
    given = qkv if packed else (q.contiguous(), k.contiguous(), v.contiguous())
    got = bp.qkv_append(given, kc, vc, _offsets(new), _offsets([c + n for c, n in zip(ctx, new)]), table, page, tab,
                        k_weight=kw, q_out=qo, ws=ws)
    assert bp.get_status(ws) == 0 and got is qo
    _near_turned(qo[:total], _turned(q[:total], None, tab, pos, False, 1e-6))
    assert torch.all(qo[total:] == 7.0)
    _near_turned(kc[rows], _turned(k[:total], kw, tab, pos, False, 1e-6))
    want_k[rows] = kc[rows]
    bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
    assert torch.equal(kc.view(bits), want_k.view(bits)) and torch.equal(vc.view(bits), want_v.view(bits))


def test_append_of_keys_alone_at_given_positions():
    g = _gen(2)
    (kc, vc), table, keys = _paged([20], 16, 2, 128, torch.bfloat16, g, [15])
    k, v = [torch.randn(5, 2, 128, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)]
    pos = torch.tensor([9, 3, 0, 4, 7], dtype=torch.int32, device="cuda")
    tab = _table(10, 128)
    ws = bp.workspace(256, "cuda")
    assert bp.qkv_append((None, k, v), kc, vc, _offsets([5]), _offsets([20]), table, 16, tab, positions=pos, interleaved=True,
                         ws=ws) is None
    assert bp.get_status(ws) == 0
    _near_turned(kc[keys[0][15:]], _turned(k, None, tab, pos, True, 1e-6))
    assert torch.equal(vc[keys[0][15:]], v)


def test_append_without_a_place_is_reported():
    """A page id outside the pool and a key past the table: reported, not written; the other sequence's tokens are."""
    g = _gen(3)
    (kc, vc), table, keys = _paged([16, 32], 16, 1, 64, torch.float32, g, [15, 30])
    table[0, 0] = 99
    k, v = [torch.randn(4, 1, 64, device="cuda", generator=g) for _ in range(2)]
    before = kc.clone()
    ws = bp.workspace(256, "cuda")
    # sequence 0: one token on page 99; sequence 1: key 31 has a place, keys 32 and 33 lie past its two pages
    bp.qkv_append((None, k, v), kc, vc, _offsets([1, 3]), _offsets([16, 34]), table, 16, None, ws=ws)
    assert bp.get_status(ws) == bp._binding.BP_ERR_DEVICE_FLAG
    before[keys[1][31]] = k[1]
    assert torch.equal(kc.view(torch.int32), before.view(torch.int32))


def _attend(q, kc, vc, rows, causal, window, scale):
    """One sequence in 64 bits: o, the sums of p |v|, the log-sum-exp; rows without a key give 0 and -inf."""
    b, hq, d = q.shape
    n, hkv = len(rows), kc.shape[1]
    k, v = [c[rows].double().repeat_interleave(hq // hkv, 1) for c in (kc, vc)]
    x = torch.einsum("ihd,jhd->hij", q.double(), k) * scale
    p, j = torch.arange(n - b, n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    hidden = torch.zeros(b, n, dtype=torch.bool, device="cuda")
    if causal:
        hidden |= j > p
    if window:
        hidden |= j <= p - window
    x.masked_fill_(hidden, -math.inf)
    z = torch.logsumexp(x, 2) if n else torch.full((hq, b), -math.inf, dtype=torch.float64, device="cuda")
    w = torch.exp(x - z[..., None].nan_to_num(neginf=0.0))
    return torch.einsum("hij,jhd->ihd", w, v), torch.einsum("hij,jhd->ihd", w, v.abs()), z.T


def _check_chunk(ctx, new, hq=8, hkv=2, dim=128, page=16, causal=True, window=0, scale=0.0, seed=0, stride=None):
    g = _gen(seed)
    lens = [c + n for c, n in zip(ctx, new)]
    (kc, vc), table, keys = _paged(lens, page, hkv, dim, torch.bfloat16, g, lens)
    total = sum(new)
    wide = torch.randn(total, stride or hq, dim, device="cuda", generator=g).mul_(1.5).to(torch.bfloat16)
    q = wide[:, :hq]
    lse = torch.full((total, hq), 7.0, device="cuda")
    out = torch.full((total, hq, dim), 7.0, device="cuda", dtype=torch.bfloat16)
    ws = bp.workspace(bp.chunk_attention_workspace_size(len(new), total, hq, hkv, dim), "cuda")
    bp.chunk_attention_paged(q, kc, vc, _offsets(new), _offsets(lens), table, page, max(new), max(1, max(lens)),
                             mask=bp.MASK_CAUSAL if causal else bp.MASK_BIDIR, window=window, softmax_scale=scale, out=out,
                             lse=lse, ws=ws)
    assert bp.get_status(ws) == 0
    at = 0
    for c, n, r in zip(ctx, new, keys):
        if n:
            o, size, z = _attend(q[at:at + n], kc, vc, r, causal, window, scale or dim ** -0.5)
            err = (out[at:at + n].double() - o).abs()
            tol = (U + 1e-3) * size + U * o.abs()
            assert torch.all(err <= tol + 1e-30), (c, n, float((err - tol).max()))
            got = lse[at:at + n].double()
            assert torch.equal(torch.isinf(z), torch.isinf(got))
            assert float((got - z).nan_to_num(0.0, 0.0, 0.0).abs().max()) <= 5e-4
        at += n
    return out


@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("ctx,new", [
    ((0,), (1,)), ((0,), (2,)), ((15,), (1,)), ((127,), (1,)), ((128,), (1,)), ((2047,), (1,)), ((0,), (63,)),
    ((0,), (128,)), ((0,), (129,)), ((700,), (300,)), ((5, 0, 1000, 31, 64), (1, 200, 33, 0, 17)), ((3000,), (70,)),
    ((0,) * 40, (1, 2, 3, 50) * 10)])
def test_chunk_lengths(dim, ctx, new):
    _check_chunk(ctx, new, dim=dim)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (6, 2), (10, 2), (7, 1), (32, 8), (16, 1), (128, 1), (100, 1)])
@pytest.mark.parametrize("dim,page", [(128, 64), (64, 16)])
def test_chunk_heads(hq, hkv, dim, page):
    _check_chunk((130, 17, 4), (70, 1, 140), hq=hq, hkv=hkv, dim=dim, page=page, seed=hq)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 1024])
def test_chunk_pages(page):
    _check_chunk((200, 0, 511), (77, 300, 1), page=page, seed=page)


@pytest.mark.parametrize("window", [1, 2, 100, 128, 129, 700, 5000])
@pytest.mark.parametrize("causal", [True, False])
def test_chunk_windows(window, causal):
    _check_chunk((900, 0, 300), (200, 500, 1), causal=causal, window=window, seed=window)


@pytest.mark.parametrize("dim", [128, 64])
def test_chunk_sees_everything(dim):
    _check_chunk((0, 100, 1000), (130, 1, 64), causal=False, dim=dim)


def test_chunk_scale_and_stride():
    _check_chunk((300, 0), (90, 40), scale=0.3, stride=13)


@pytest.mark.parametrize("causal", [True, False])
def test_rows_without_keys(causal):
    """More new tokens than keys: the first rows see nothing and are 0, with a log-sum-exp of -inf."""
    _check_chunk((-50, 0, -3, -200, 100), (80, 5, 3, 500, 2), causal=causal)
    _check_chunk((-50, 10), (80, 70), causal=causal, window=20)


def test_long_split_and_repeats():
    """A context cut over all CTAs; the same call gives the same bits again, and once more on another stream."""
    ctx, new = (20000, 3, 9000), (40, 5, 1)
    a = _check_chunk(ctx, new, hq=4, hkv=1, page=64)
    b = _check_chunk(ctx, new, hq=4, hkv=1, page=64)
    assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = _check_chunk(ctx, new, hq=4, hkv=1, page=64)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, c)


def test_scores_of_any_size():
    """Rows whose maxima grow from tile to tile, and scores far below 0: the running maximum is followed."""
    g = _gen(9)
    n, hkv, dim = 1200, 1, 128
    (kc, vc), table, keys = _paged([n], 64, hkv, dim, torch.bfloat16, g, [n])
    ramp = torch.linspace(-60, 60, n, device="cuda")
    kc[keys[0]] = 0
    kc[keys[0], 0, 0] = ramp.to(torch.bfloat16)
    q = torch.zeros(64, 2, dim, device="cuda", dtype=torch.bfloat16)
    q[:, 0, 0], q[:, 1, 0] = 30.0, -30.0
    ws = bp.workspace(bp.chunk_attention_workspace_size(1, 64, 2, 1, dim), "cuda")
    out, _ = bp.chunk_attention_paged(q, kc, vc, _offsets([64]), _offsets([n]), table, 64, 64, n, softmax_scale=1.0, ws=ws)
    assert bp.get_status(ws) == 0
    o, size, _ = _attend(q, kc, vc, keys[0], True, 0, 1.0)
    assert torch.all((out.double() - o).abs() <= (U + 1e-3) * size + U * o.abs() + 1e-30)


def test_a_bad_page_is_reported():
    g = _gen(4)
    (kc, vc), table, _ = _paged([300], 16, 1, 64, torch.bfloat16, g, [300])
    table[0, 3] = 10 ** 6
    q = torch.randn(4, 2, 64, device="cuda", generator=g).to(torch.bfloat16)
    ws = bp.workspace(bp.chunk_attention_workspace_size(1, 4, 2, 1, 64), "cuda")
    bp.chunk_attention_paged(q, kc, vc, _offsets([4]), _offsets([300]), table, 16, 4, 300, ws=ws)
    assert bp.get_status(ws) == bp._binding.BP_ERR_DEVICE_FLAG


@pytest.mark.parametrize("max_q, max_kv", [(63, 1200), (64, 1199), (1, 300), (64, 1200), (1000, 1216)])
def test_a_sequence_past_the_bounds_is_reported(max_q, max_kv):
    """The merge is sized by the bounds, so a longer sequence than they say must not pass unnoticed."""
    g = _gen(12)
    (kc, vc), table, _ = _paged([900, 1200], 64, 1, 64, torch.bfloat16, g, [900, 1200])
    q = torch.randn(65, 2, 64, device="cuda", generator=g).to(torch.bfloat16)
    ws = bp.workspace(bp.chunk_attention_workspace_size(2, 65, 2, 1, 64), "cuda")
    bp.chunk_attention_paged(q, kc, vc, _offsets([1, 64]), _offsets([900, 1200]), table, 64, max_q, max_kv, ws=ws)
    assert bp.get_status(ws) == (0 if max_q >= 64 and max_kv >= 1200 else bp._binding.BP_ERR_DEVICE_FLAG)


def test_empty_calls():
    z = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    ws = bp.workspace(bp.chunk_attention_workspace_size(1, 0, 2, 1, 64), "cuda")
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    o, _ = bp.chunk_attention_paged(z(0, 2, 64), z(16, 1, 64), z(16, 1, 64), _offsets([0]), _offsets([5]), table, 16, 0, 5, ws=ws)
    assert o.shape == (0, 2, 64)
    assert bp.qk_norm_rope(z(0, 2, 64), z(0, 1, 64), _table(4, 64), torch.zeros(0, dtype=torch.int32, device="cuda"))[0].shape == (0, 2, 64)
    assert bp.qkv_append(z(0, 4, 64), z(16, 1, 64), z(16, 1, 64), _offsets([0]), _offsets([5]), table, 16, None).shape == (0, 2, 64)


def test_more_tokens_than_a_grid_has_rows():
    """Half a million tokens: blocks take more than one group of tokens."""
    g = _gen(11)
    t = 65535 * 8 + 1003
    q = torch.randn(t, 1, 16, device="cuda", generator=g)
    pos = torch.randint(0, 50, (t,), device="cuda", generator=g).to(torch.int32)
    table = _table(50, 16)
    ws = bp.workspace(256, "cuda")
    out, _ = bp.qk_norm_rope(q, None, table, pos, ws=ws)
    assert bp.get_status(ws) == 0
    _near_turned(out, _turned(q, None, table, pos, False, 1e-6))


def test_offsets_beyond_32_bits():
    """Pages whose rows lie more than 2^31 elements into their pool, by append and attention."""
    g = _gen(12)
    hkv, dim, page, ctx, new = 8, 128, 64, 100, 60
    rows = (2 ** 31 // (hkv * dim) // page + 40) * page
    kc, vc = [torch.empty(rows, hkv, dim, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    table = torch.tensor([[rows // page - 1, 1, rows // page - 30]], dtype=torch.int32, device="cuda")
    j = torch.arange(ctx + new, device="cuda")
    at = table[0].long()[j // page] * page + j % page
    for c in (kc, vc):
        c[at[:ctx]] = torch.randn(ctx, hkv, dim, device="cuda", generator=g).to(torch.bfloat16)
    qkv = torch.randn(new, 16 + 2 * hkv, dim, device="cuda", generator=g).to(torch.bfloat16)
    ws = bp.workspace(bp.chunk_attention_workspace_size(1, new, 16, hkv, dim), "cuda")
    q = bp.qkv_append(qkv, kc, vc, _offsets([new]), _offsets([ctx + new]), table, page, None, ws=ws)
    assert torch.equal(q, qkv[:, :16]) and torch.equal(kc[at[ctx:]], qkv[:, 16:24]) and torch.equal(vc[at[ctx:]], qkv[:, 24:])
    o, _ = bp.chunk_attention_paged(q, kc, vc, _offsets([new]), _offsets([ctx + new]), table, page, new, ctx + new, ws=ws)
    assert bp.get_status(ws) == 0
    ref, size, _ = _attend(q, kc, vc, at, True, 0, dim ** -0.5)
    assert torch.all((o.double() - ref).abs() <= (U + 1e-3) * size + U * ref.abs() + 1e-30)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 400])
def test_a_window_over_everything(window):
    """Wider than every context: the same bits as without one, rows without keys among them."""
    args = dict(ctx=(-50, 200, 0), new=(80, 150, 300), causal=False)
    assert torch.equal(_check_chunk(**args, window=window), _check_chunk(**args))


def test_batch_does_not_matter():
    """Many sequences (more than one round of the plan), and rows of other sequences that are not numbers."""
    ctx, new = tuple(range(0, 1400, 20)), (1, 3, 40, 0, 2) * 14
    _check_chunk(ctx, new, hq=4, hkv=1, dim=64)
    g = _gen(5)
    (kc, vc), table, keys = _paged([70, 30], 16, 1, 64, torch.bfloat16, g, [70, 30])
    q = torch.randn(25, 2, 64, device="cuda", generator=g).to(torch.bfloat16)
    q[20:] = math.nan  # the second sequence's
    ws = bp.workspace(bp.chunk_attention_workspace_size(2, 25, 2, 1, 64), "cuda")
    o, _ = bp.chunk_attention_paged(q, kc, vc, _offsets([20, 5]), _offsets([70, 30]), table, 16, 20, 70, ws=ws)
    ref, size, _ = _attend(q[:20], kc, vc, keys[0], True, 0, 0.125)
    assert torch.all((o[:20].double() - ref).abs() <= (U + 1e-3) * size + U * ref.abs() + 1e-30) and torch.isnan(o[20:].float()).all()


def test_example_runs():
    """The example's prompts give the same rows in chunks as at once, and its block the same as a chunk, up to the
    rounding of two layers' bf16 activations (a few roundings of 2^-9 on average each: below 2e-2 of a row's size)."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "chunked_prefill.py")
    spec = importlib.util.spec_from_file_location("chunked_prefill", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    off, near, finite = example.main()
    assert off < 2e-2 and near < 2e-2 and finite


@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("ctx", [100, 6000])
def test_what_is_no_number_shows(ctx, new, dim):
    """A NaN in a query or in a key that a row sees, and a score past fp32, make that row NaN in o and in the log-sum-exp,
    whether its keys are one CTA's (100) or cut among many (6000); the rows that see none of it keep their bits."""
    g = _gen(ctx + new)
    n, hq = ctx + new, 4
    (kc, vc), table, keys = _paged([n], 64, 1, dim, torch.bfloat16, g, [n])
    q = torch.randn(new, hq, dim, device="cuda", generator=g).to(torch.bfloat16)
    ws = bp.workspace(bp.chunk_attention_workspace_size(1, new, hq, 1, dim), "cuda")

    def attend(q, k):
        lse = torch.full((new, hq), 7.0, device="cuda")
        o, _ = bp.chunk_attention_paged(q, k, vc, _offsets([new]), _offsets([n]), table, 64, new, n, lse=lse, ws=ws)
        assert bp.get_status(ws) == 0
        return o, lse

    def is_lost(got, lost):
        o, lse = got
        assert torch.isnan(o[lost].float()).all() and torch.isnan(lse[lost]).all()
        assert torch.equal(o[~lost], clean[0][~lost]) and torch.equal(lse[~lost], clean[1][~lost])

    clean = attend(q, kc)
    assert torch.isfinite(clean[0].float()).all() and torch.isfinite(clean[1]).all()
    lost = torch.zeros(new, hq, dtype=torch.bool, device="cuda")
    lost[new // 2, 2] = True
    bad_q = q.clone()
    bad_q[lost] = math.nan
    is_lost(attend(bad_q, kc), lost)
    for key in (0, ctx // 2, ctx + new // 2, n - 1):
        bad_k = kc.clone()
        bad_k[keys[0][key], 0, 5] = math.nan
        lost = (torch.arange(ctx, n, device="cuda") >= key)[:, None].expand(new, hq)
        is_lost(attend(q, bad_k), lost)
    # 1e30 times 1e30 in one score; all others stay below 1e32
    bad_q, bad_k = q.clone(), kc.clone()
    bad_q[0, 1] = 0
    bad_q[0, 1, 0] = 1e30
    bad_k[keys[0][ctx // 2]] = 0
    bad_k[keys[0][ctx // 2], 0, 0] = 1e30
    o, lse = attend(bad_q, bad_k)
    assert torch.isnan(o[0, 1].float()).all() and not torch.isfinite(lse[0, 1])


def test_calls_on_a_stream_of_their_own():
    """stream= with nothing else given, while the current stream is busy and its free memory is written to right after each
    call: the same bits as with outputs and workspaces of the caller's."""
    g = _gen(31)
    n, hq, hkv, dim = 3000, 8, 2, 128
    (kc, vc), table, _ = _paged([n], 64, hkv, dim, torch.bfloat16, g, [n])
    q = torch.randn(40, hq, dim, device="cuda", generator=g).to(torch.bfloat16)
    tab, pos, cu, cu_kv = _table(n, dim), torch.arange(40, device="cuda", dtype=torch.int32), _offsets([40]), _offsets([n])
    want_o, _ = bp.chunk_attention_paged(q, kc, vc, cu, cu_kv, table, 64, 40, n)
    want_q, want_k = bp.qk_norm_rope(q, q[:, :2], tab, pos)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)  # about 10 ms on the current stream
    got_o, _ = bp.chunk_attention_paged(q, kc, vc, cu, cu_kv, table, 64, 40, n, stream=side)
    got_q, got_k = bp.qk_norm_rope(q, q[:, :2], tab, pos, stream=side)
    taken = [torch.full((bp.chunk_attention_workspace_size(1, 40, hq, hkv, dim),), 255, device="cuda", dtype=torch.uint8) for _ in range(3)]
    side.synchronize()
    got = [x.clone() for x in (got_o, got_q, got_k)]
    torch.cuda.synchronize()
    assert len(taken) == 3 and all(torch.equal(a, b) for a, b in zip(got, (want_o, want_q, want_k)))


@pytest.mark.parametrize("first", [0, 3])
def test_rows_past_the_call_are_not_written(first):
    """Offsets that name more rows than the call has (a batch that grew past the room of a replayed call): reported, that
    sequence left out, nothing written behind the outputs, the others computed."""
    g = _gen(13)
    lens, new, total, hq, dim = [700, 3000], [4, 8], 8, 2, 64
    (kc, vc), table, keys = _paged(lens, 64, 1, dim, torch.bfloat16, g, lens)
    q = torch.randn(total, hq, dim, device="cuda", generator=g).to(torch.bfloat16)
    out, lse = torch.full((40, hq, dim), 7.0, device="cuda", dtype=torch.bfloat16), torch.full((40, hq), 7.0, device="cuda")
    ws = bp.workspace(bp.chunk_attention_workspace_size(2, total, hq, 1, dim), "cuda")
    cu = _offsets(new) + first
    bp.chunk_attention_paged(q, kc, vc, cu, _offsets(lens), table, 64, 8, 3000, out=out[:total], lse=lse[:total], ws=ws)
    assert bp.get_status(ws) == bp._binding.BP_ERR_DEVICE_FLAG
    rows = slice(first, first + new[0])
    ref, size, _ = _attend(q[rows], kc, vc, keys[0], True, 0, dim ** -0.5)
    assert torch.all((out[rows].double() - ref).abs() <= (U + 1e-3) * size + U * ref.abs() + 1e-30)
    for x in (out, lse):
        assert torch.all(x[:first] == 7.0) and torch.all(x[first + new[0]:] == 7.0)
    bp.chunk_attention_paged(q, kc, vc, cu + 100, _offsets(lens), table, 64, 8, 3000, out=out[:total], lse=lse[:total], ws=ws)
    assert bp.get_status(ws) == bp._binding.BP_ERR_DEVICE_FLAG and torch.all(out[total:] == 7.0)
    bp.chunk_attention_paged(q, kc, vc, cu - first - 1, _offsets(lens), table, 64, 8, 3000, out=out[:total], lse=lse[:total], ws=ws)
    assert bp.get_status(ws) == bp._binding.BP_ERR_DEVICE_FLAG and torch.all(out[total:] == 7.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("hq,hkv", [(32, 8), (5, 1), (0, 3)])
@pytest.mark.parametrize("ctx,new,at", [((0,), (1,), False), ((5, 100, 0, 33, 63), (3, 1, 70, 0, 1), True), ((1000, 7), (600, 400), False)])
def test_append_of_whole_heads_in_halves(dtype, dim, hq, hkv, ctx, new, at):
    """The usual form (the whole head turned in halves, both norms weighted), packed and in tensors of their own: queries,
    keys and values against 64 bits, at the keys' numbers and at given positions; nothing else of the pool touched."""
    g = _gen(dim + hq)
    total, page = sum(new), 16
    qkv = (2 * torch.randn(total, hq + 2 * hkv, dim, device="cuda", generator=g)).to(dtype)
    q, k, v = qkv.split([hq, hkv, hkv], 1)
    qw, kw = [(1 + 0.3 * torch.randn(dim, device="cuda", generator=g)).to(dtype) for _ in range(2)]
    lens = [c + n for c, n in zip(ctx, new)]
    tab = _table(2000, dim)
    pos = torch.cat([torch.arange(c, c + n, device="cuda") for c, n in zip(ctx, new)])
    if at:
        pos = torch.randint(0, 2000, (total,), device="cuda", generator=g)
    bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
    for given in (qkv, (q if hq else None, k.contiguous(), v)):
        (kc, vc), table, keys = _paged(lens, page, hkv, dim, dtype, g, ctx)
        rows = torch.cat([r[c:] for r, c in zip(keys, ctx)])
        want_k, want_v = kc.clone(), vc.clone()
        want_v[rows] = v
        ws = bp.workspace(256, "cuda")
        qo = bp.qkv_append(given, kc, vc, _offsets(new), _offsets(lens), table, page, tab,
                           positions=pos.to(torch.int32) if at else None, q_weight=qw, k_weight=kw, eps=1e-5, ws=ws)
        assert bp.get_status(ws) == 0
        if hq:
            _near_turned(qo, _turned(q, qw, tab, pos, False, 1e-5))
        _near_turned(kc[rows], _turned(k, kw, tab, pos, False, 1e-5))
        want_k[rows] = kc[rows]
        assert torch.equal(kc.view(bits), want_k.view(bits)) and torch.equal(vc.view(bits), want_v.view(bits))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (6, 2), (10, 2), (7, 1), (32, 8), (16, 1), (128, 1), (100, 1)])
@pytest.mark.parametrize("dim,page", [(128, 64), (64, 16)])
@pytest.mark.parametrize("new", [(70, 1, 140), (1, 1, 1)])
def test_chunk_heads_of_cut_contexts(hq, hkv, dim, page, new):
    """Contexts that are cut among CTAs: both forms of the merge, with any number of heads and tokens a tile."""
    _check_chunk((6000, 17, 2500), new, hq=hq, hkv=hkv, dim=dim, page=page, seed=hq)


def test_a_graph_replays_with_other_lengths():
    """Norm and rotation, append and attention captured once, with room for 300 tokens of 3 sequences, and replayed over
    other lengths, pages and values: every call reads them from the device."""
    g = _gen(21)
    room, hq, hkv, dim, page, most = 300, 8, 2, 128, 64, 5000
    per = most // page + 1
    qkv = torch.zeros(room, hq + 2 * hkv, dim, device="cuda", dtype=torch.bfloat16)
    kc, vc = [torch.zeros(3 * per * page, hkv, dim, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    w = [(1 + 0.1 * torch.randn(dim, device="cuda", generator=g)).to(torch.bfloat16) for _ in range(2)]
    tab = _table(most, dim)
    cu_new, cu_kv = [torch.zeros(4, dtype=torch.int32, device="cuda") for _ in range(2)]
    table = torch.zeros(3, per, dtype=torch.int32, device="cuda")
    pos = torch.zeros(room, dtype=torch.int32, device="cuda")
    q = torch.empty(room, hq, dim, device="cuda", dtype=torch.bfloat16)
    q2, o = torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty(room, hq, device="cuda")
    small, ws = bp.workspace(256, "cuda"), bp.workspace(bp.chunk_attention_workspace_size(3, room, hq, hkv, dim), "cuda")

    def step():
        bp.qkv_append(qkv, kc, vc, cu_new, cu_kv, table, page, tab, q_weight=w[0], k_weight=w[1], q_out=q, ws=small)
        bp.qk_norm_rope(qkv[:, :hq], None, tab, pos, q_weight=w[0], q_out=q2, ws=small)
        bp.chunk_attention_paged(q, kc, vc, cu_new, cu_kv, table, page, room, most, out=o, lse=lse, ws=ws)

    step()  # nothing to do: no sequence has a token
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for ctx, new in (((4000, 0, 70), (1, 200, 1)), ((10, 4900, 0), (100, 100, 100)), ((0, 0, 3000), (0, 0, 1)), ((4000, 0, 70), (1, 200, 1))):
        lens, total = [c + n for c, n in zip(ctx, new)], sum(new)
        order = torch.randperm(3 * per, device="cuda", generator=g).to(torch.int32).view(3, per)
        qkv.copy_(torch.randn(qkv.shape, device="cuda", generator=g))
        for c in (kc, vc):
            c.copy_(torch.randn(c.shape, device="cuda", generator=g))
        table.copy_(order)
        cu_new.copy_(_offsets(new))
        cu_kv.copy_(_offsets(lens))
        here = torch.cat([torch.arange(c, c + n, device="cuda") for c, n in zip(ctx, new)])
        pos[:total] = here
        for t in (q, o, lse):
            t.fill_(7.0)
        graph.replay()
        assert bp.get_status(small) == 0 and bp.get_status(ws) == 0
        _near_turned(q[:total], _turned(qkv[:total, :hq], w[0], tab, here, False, 1e-6))
        assert torch.equal(q2[:total], q[:total])
        assert torch.all(q[total:] == 7.0) and torch.all(o[total:] == 7.0) and torch.all(lse[total:] == 7.0)
        at = 0
        for s, (c, n) in enumerate(zip(ctx, new)):
            if n:
                j = torch.arange(c + n, device="cuda")
                rows = order[s].long()[j // page] * page + j % page
                _near_turned(kc[rows[c:]], _turned(qkv[at:at + n, hq:hq + hkv], w[1], tab, j[c:], False, 1e-6))
                assert torch.equal(vc[rows[c:]], qkv[at:at + n, hq + hkv:])
                ref, size, z = _attend(q[at:at + n], kc, vc, rows, True, 0, dim ** -0.5)
                err = (o[at:at + n].double() - ref).abs()
                assert torch.all(err <= (U + 1e-3) * size + U * ref.abs() + 1e-30)
                assert float((lse[at:at + n].double() - z).abs().max()) <= 5e-4
            at += n
