"""Prefill over a paged KV cache: what carries a prompt, or a chunk of one, from a layer's projections to its attention.

Three operators, each in a plain form (elementary torch operations in 32 bits, rounded once at the end) and as the
package's entry point:

  rope    every head's query and key normed (root mean square) and rotated to its position in one pass
  append  the same on the packed output of a layer's projection, the keys and values going to their pages
  chunk   attention of chunks of new tokens, of one token to a whole prompt, over the pages

Sizes are those of the package's workloads (32 query / 8 KV heads of 128; contexts of 256 to 32768 keys; pages of 16
and 64) and the ranges around them.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
MOST_PAIRS = 60_000_000  # padded (query, key) pairs of a drawn case at 32 heads


def _rope(name, tokens, **more):
    """tokens: drawn from a batch's rows; their positions lie anywhere below ctx."""
    case = dict(kind="rope", tokens=tokens, ctx=32768, dtype="bf16", hq=32, hkv=8, dim=128, rotary=128, interleaved=False,
                norm=True)
    case.update(more)
    return dict(case, name=name) if name else case


def _append(name, seqs, ctx, new, **more):
    """ctx and new are every sequence's keys in the cache and new tokens; mixed: see _lengths."""
    case = dict(kind="append", seqs=seqs, ctx=ctx, new=new, mixed=False, dtype="bf16", hq=32, hkv=8, dim=128, rotary=128,
                interleaved=False, norm=True, page=64, shape_seed=3)
    case.update(more)
    return dict(case, name=name) if name else case


def _chunk(name, seqs, ctx, new, **more):
    case = dict(kind="chunk", seqs=seqs, ctx=ctx, new=new, mixed=False, hq=32, hkv=8, dim=128, causal=True, window=0,
                lse=False, page=64, shape_seed=3)
    case.update(more)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest call: one request decodes one token
        _rope("rope_1", 1),
        # a verify pass's queries and keys: 8 requests' blocks of 16
        _rope("rope_128", 128),
        # a prefill batch of whole prompts, an odd number of tokens
        _rope("rope_16381", 16381),
        # an fp32 model with small heads, of which the front half turns, in neighbouring pairs
        _rope("rope_f32_1000", 1000, dtype="f32", hq=4, hkv=2, dim=64, rotary=32, interleaved=True, ctx=2048),
        # a decoding batch: one token of each of 32 requests
        _append("append_32x1", 32, 4096, 1),
        # a serving batch: a quarter of the requests bring a chunk of their prompt, the others decode
        _append("append_mixed_32", 32, 4096, 1000, mixed=True, page=16),
        # the chunk of a long prompt
        _append("append_1x8192", 1, 8192, 8192),
        # one request decodes one token over a chat-length context
        _chunk("chunk_1x1_2048", 1, 2048, 1, lse=True),
        # a serving batch: prompt chunks and decoding requests in one call
        _chunk("chunk_mixed_16", 16, 4096, 500, mixed=True, page=16),
        # small heads over a sliding window, 4 prompts of an odd length
        _chunk("chunk_window_4x2001", 4, 0, 2001, hq=8, hkv=2, dim=64, window=1024),
        # a whole prompt at once
        _chunk("chunk_1x8192", 1, 0, 8192),
        # a chunk of a long document, the largest call
        _chunk("chunk_2048_of_32768", 1, 32768 - 2048, 2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rope", "rope", "append", "append", "chunk", "chunk", "chunk", "chunk"))
    seed = rng.randrange(1 << 20)
    dim = rng.choice((64, 128, 128))
    heads = dict(zip(("hq", "hkv"), rng.choice(((32, 8), (32, 8), (8, 2), (8, 8), (4, 2), (12, 4), (10, 2)))))
    turn = dict(dtype=rng.choice(("bf16", "bf16", "f32")), rotary=rng.choice((dim, dim, dim // 2)),
                interleaved=rng.random() < 0.3, norm=rng.random() < 0.8, dim=dim, **heads)
    if kind == "rope":
        return _rope("", _log_int(rng, 1, 16384), ctx=_log_int(rng, 256, 32768), **turn)
    seqs = _log_int(rng, 1, 32)
    ctx = _log_int(rng, 0.6, 32768)
    mixed = seqs > 3 and rng.random() < 0.6
    page = rng.choice((16, 64, 128))
    if kind == "append":
        ctx = min(ctx, 65536 // seqs)
        return _append("", seqs, ctx, _log_int(rng, 1, max(2, 8192 // seqs)), mixed=mixed, page=page, shape_seed=seed, **turn)
    ctx = min(ctx, 262144 // seqs)
    budget = MOST_PAIRS * 32 // (heads["hq"] * seqs)
    most = int((math.sqrt(ctx * ctx + 4 * budget) - ctx) / 2)  # new * (ctx + new) within the budget
    return _chunk("", seqs, ctx, _log_int(rng, 1, max(2, min(8192, most))), mixed=mixed, page=page, shape_seed=seed, dim=dim,
                  causal=rng.random() < 0.85, window=rng.choice((0, 0, 0, _log_int(rng, 16, 4096))),
                  lse=rng.random() < 0.4, **heads)


# --------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """Every sequence's keys before the call and its new tokens.  mixed: the contexts lie in [ctx / 16, ctx], a quarter
    of the sequences brings half of `new` to all of it, the others one token."""
    n, ctx, new = case["seqs"], case["ctx"], case["new"]
    if not case["mixed"]:
        return [ctx] * n, [new] * n
    g = np.random.default_rng(case["shape_seed"])
    ctxs = g.integers(ctx // 16, ctx, size=n, endpoint=True).tolist()
    news = g.integers((new + 1) // 2, new, size=n, endpoint=True)
    news[g.permutation(n)[(n + 3) // 4:]] = 1
    return ctxs, news.tolist()


def _offsets(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32), device="cuda")


def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _turning(case, g, ctx):
    """A table of cosines and sines for every position, and the norms' weights."""
    half = case["rotary"] // 2
    angle = torch.arange(ctx, dtype=torch.float64, device="cuda")[:, None] * 1e6 ** (
        -torch.arange(half, dtype=torch.float64, device="cuda") / half)
    w = [(1 + 0.2 * torch.randn(case["dim"], device="cuda", generator=g)).to(_dtype(case)) for _ in range(2)]
    return dict(table=torch.cat([angle.cos(), angle.sin()], 1).float(), interleaved=case["interleaved"],
                q_weight=w[0] if case["norm"] else None, k_weight=w[1] if case["norm"] else None)


def _paging(case, ctxs, news, seed):
    """A block table over a pool of pages, the sequences' pages in shuffled order, and the pool's rows."""
    page = case["page"]
    need = [-(-(c + n) // page) for c, n in zip(ctxs, news)]
    order = np.random.default_rng(seed).permutation(sum(need)).astype(np.int32)
    table = np.zeros((len(need), max(need)), dtype=np.int32)
    for i, part in enumerate(np.split(order, np.cumsum(need)[:-1])):
        table[i, :len(part)] = part
    return dict(pages=torch.from_numpy(table).cuda(), page=page, cu_new=_offsets(news),
                cu_kv=_offsets([c + n for c, n in zip(ctxs, news)]), max_new=max(news),
                max_kv=max(c + n for c, n in zip(ctxs, news))), sum(need) * page


def prepare(case, seed):
    """Projections are N(0, 1), their queries a little wider, so that a row's attention favours some keys.  Rows of the
    pool that no key has yet are not numbers: memory that nothing has written."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    hq, hkv, dim, dtype = case["hq"], case["hkv"], case["dim"], _dtype(case)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    if case["kind"] == "rope":
        t = case["tokens"]
        return dict(_turning(case, g, case["ctx"]), kind="rope", q=randn(t, hq, dim).to(dtype), k=randn(t, hkv, dim).to(dtype),
                    pos=torch.randint(0, case["ctx"], (t,), device="cuda", generator=g).to(torch.int32))
    ctxs, news = _lengths(case)
    s, rows = _paging(case, ctxs, news, seed)
    s["kind"] = case["kind"]
    held = torch.zeros(rows, dtype=torch.bool, device="cuda")
    at = torch.arange(s["max_kv"], device="cuda")
    full = _rows_of(s, at)
    len_kv, len_new = s["cu_kv"].diff().long(), s["cu_new"].diff().long()
    if case["kind"] == "append":
        s.update(_turning(case, g, s["max_kv"]), qkv=randn(sum(news), hq + 2 * hkv, dim).to(dtype), hkv=hkv)
        len_kv = len_kv - len_new
    held[full[at < len_kv[:, None]]] = True
    for name in ("k_cache", "v_cache"):
        s[name] = randn(rows, hkv, dim).masked_fill_(~held[:, None, None], math.nan).to(dtype)
    if case["kind"] == "chunk":
        s.update(q=(1.5 * randn(sum(news), hq, dim)).to(dtype), causal=case["causal"], window=case["window"], lse=case["lse"])
    return s


def _rows_of(s, at):
    """The pool rows of every sequence's keys `at`: [sequences, len(at)]."""
    return s["pages"].long()[:, at // s["page"]] * s["page"] + at % s["page"]


# --------------------------------------------------------------------------------------------- the plain forms
def _plain_turn(x, weight, s, pos):
    x = x.float()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    half = s["table"].shape[1] // 2
    row = s["table"][pos.long()][:, None, :]
    c, t = row[..., :half], row[..., half:]
    turn, rest = x[..., :2 * half], x[..., 2 * half:]
    if s["interleaved"]:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turn = torch.stack([a * c - b * t, b * c + a * t], -1).flatten(-2)
    else:
        a, b = turn[..., :half], turn[..., half:]
        turn = torch.cat([a * c - b * t, b * c + a * t], -1)
    return torch.cat([turn, rest], -1)


def _plain_rope(s):
    return (_plain_turn(s["q"], s["q_weight"], s, s["pos"]).to(s["q"].dtype),
            _plain_turn(s["k"], s["k_weight"], s, s["pos"]).to(s["k"].dtype))


def _plain_append(s):
    qkv, hkv = s["qkv"], s["hkv"]
    hq = qkv.shape[1] - 2 * hkv
    t = torch.arange(qkv.shape[0], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["cu_new"], t, right=True) - 1
    pos = (s["cu_kv"].diff() - s["cu_new"].diff() - s["cu_new"][:-1])[seq] + t
    row = s["pages"][seq, pos // s["page"]].long() * s["page"] + pos % s["page"]
    s["k_cache"][row] = _plain_turn(qkv[:, hq:hq + hkv], s["k_weight"], s, pos).to(qkv.dtype)
    s["v_cache"][row] = qkv[:, hq + hkv:]
    return _plain_turn(qkv[:, :hq], s["q_weight"], s, pos).to(qkv.dtype), s["k_cache"], s["v_cache"]


def _plain_chunk(s):
    """The sequences padded to the longest: scores of every (query, key) pair, the hidden ones struck out."""
    q, hkv, dim = s["q"], s["k_cache"].shape[1], s["q"].shape[2]
    group, n, m = q.shape[1] // hkv, s["max_kv"], s["max_new"]
    at, i = torch.arange(n, device="cuda"), torch.arange(m, device="cuda")
    len_kv, len_new = s["cu_kv"].diff()[:, None], s["cu_new"].diff()[:, None]
    there, real = at < len_kv, i < len_new
    rows = _rows_of(s, at)
    k = s["k_cache"][rows].float().masked_fill(~there[..., None, None], 0.0)
    v = s["v_cache"][rows].float().masked_fill(~there[..., None, None], 0.0)
    t = (s["cu_new"][:-1, None] + i).clamp(max=len(q) - 1).long()
    qq = q[t].float().view(-1, m, hkv, group, dim).permute(0, 2, 3, 1, 4).reshape(-1, hkv, group * m, dim)
    score = torch.matmul(qq, k.permute(0, 2, 3, 1)).mul_(1 / math.sqrt(dim)).view(-1, hkv, group, m, n)
    pos = (len_kv - len_new + i)[..., None]
    seen = there[:, None, :].expand(-1, m, -1)
    if s["causal"]:
        seen = seen & (at <= pos)
    if s["window"]:
        seen = seen & (at > pos - s["window"])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = score.sum(-1, keepdim=True)
    o = torch.matmul(score.view(-1, hkv, group * m, n), v.permute(0, 2, 1, 3)).view(-1, hkv, group, m, dim)
    o = (o / total.masked_fill(total == 0, 1.0)).permute(0, 3, 1, 2, 4).reshape(-1, m, hkv * group, dim)[real]
    if not s["lse"]:
        return o.to(q.dtype)
    return o.to(q.dtype), (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(-1, m, hkv * group)[real]


# --------------------------------------------------------------------------------------------- the package's operators
def _own_rope(s):
    import paper_2606_31315_gb300 as bp

    if "ws" not in s:
        s.update(ws=bp.workspace(256, "cuda"), q_out=torch.empty_like(s["q"]), k_out=torch.empty_like(s["k"]))
    return bp.qk_norm_rope(s["q"], s["k"], s["table"], s["pos"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                           interleaved=s["interleaved"], eps=EPS, q_out=s["q_out"], k_out=s["k_out"], ws=s["ws"])


def _own_append(s):
    import paper_2606_31315_gb300 as bp

    qkv = s["qkv"]
    if "ws" not in s:
        s.update(ws=bp.workspace(256, "cuda"), q_out=torch.empty_like(qkv[:, :qkv.shape[1] - 2 * s["hkv"]]).contiguous())
    q = bp.qkv_append(qkv, s["k_cache"], s["v_cache"], s["cu_new"], s["cu_kv"], s["pages"], s["page"], s["table"],
                      q_weight=s["q_weight"], k_weight=s["k_weight"], interleaved=s["interleaved"], eps=EPS,
                      q_out=s["q_out"], ws=s["ws"])
    return q, s["k_cache"], s["v_cache"]


def _own_chunk(s):
    import paper_2606_31315_gb300 as bp

    q = s["q"]
    if "ws" not in s:
        s.update(out=torch.empty_like(q), lse_out=torch.empty(q.shape[:2], device="cuda") if s["lse"] else None,
                 ws=bp.workspace(bp.chunk_attention_workspace_size(s["cu_new"].numel() - 1, q.shape[0], q.shape[1],
                                                                   s["k_cache"].shape[1], q.shape[2]), "cuda"))
    o, lse = bp.chunk_attention_paged(q, s["k_cache"], s["v_cache"], s["cu_new"], s["cu_kv"], s["pages"], s["page"],
                                      s["max_new"], s["max_kv"], mask=bp.MASK_CAUSAL if s["causal"] else bp.MASK_BIDIR,
                                      window=s["window"], out=s["out"], lse=s["lse_out"], ws=s["ws"])
    return (o, lse) if s["lse"] else o


_PLAIN = dict(rope=_plain_rope, append=_plain_append, chunk=_plain_chunk)
_OWN = dict(rope=_own_rope, append=_own_append, chunk=_own_chunk)


def run(state):
    return (_OWN if own else _PLAIN)[state["kind"]](state)


# --------------------------------------------------------------------------------------------- in 64 bits
def _exact_turn(x, weight, s, pos):
    """Every pair of a head as a complex number, times the unit number of its angle."""
    x = x.double()
    if weight is not None:
        x = x * weight.double() * ((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS) ** -0.5
    r = s["table"].shape[1]
    unit = torch.view_as_complex(s["table"][pos.long()].double().view(-1, 1, 2, r // 2).transpose(2, 3).contiguous())
    pairs = x[..., :r].reshape(*x.shape[:-1], *((r // 2, 2) if s["interleaved"] else (2, r // 2)))
    if not s["interleaved"]:
        pairs = pairs.transpose(-1, -2)
    turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * unit)
    if not s["interleaved"]:
        turned = turned.transpose(-1, -2)
    out = x.clone()
    out[..., :r] = turned.reshape(*x.shape[:-1], r)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return _exact_turn(s["q"], s["q_weight"], s, s["pos"]), _exact_turn(s["k"], s["k_weight"], s, s["pos"])
    ctxs, news = _lengths(case)
    keys = [_rows_of(s, torch.arange(c + n, device="cuda"))[i] for i, (c, n) in enumerate(zip(ctxs, news))]
    if case["kind"] == "append":
        hq, hkv = case["hq"], case["hkv"]
        pos = torch.cat([torch.arange(c, c + n, device="cuda") for c, n in zip(ctxs, news)])
        row = torch.cat([r[c:] for c, r in zip(ctxs, keys)])
        q, k, v = s["qkv"].split([hq, hkv, hkv], 1)
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        kc[row], vc[row] = _exact_turn(k, s["k_weight"], s, pos), v.double()
        return _exact_turn(q, s["q_weight"], s, pos), kc, vc
    out, lses, first = [], [], 0
    for c, n, rows in zip(ctxs, news, keys):
        p, j = torch.arange(c, c + n, device="cuda")[:, None], torch.arange(c + n, device="cuda")[None, :]
        hidden = (j > p) if case["causal"] else torch.zeros(n, c + n, dtype=torch.bool, device="cuda")
        if case["window"]:
            hidden = hidden | (p - j >= case["window"])
        o, z = [], []
        for h in range(case["hq"]):
            kv = h // (case["hq"] // case["hkv"])
            x = s["q"][first:first + n, h].double() @ s["k_cache"][rows, kv].double().T / case["dim"] ** 0.5
            x[hidden] = -math.inf
            z.append(torch.logsumexp(x, 1))
            o.append(torch.exp(x - z[-1][:, None]) @ s["v_cache"][rows, kv].double())
        out.append(torch.stack(o, 1))
        lses.append(torch.stack(z, 1))
        first += n
    return (torch.cat(out), torch.cat(lses)) if case["lse"] else torch.cat(out)


# --------------------------------------------------------------------------------------------- what a pass has to do
def work(case):
    e = 4 if case.get("dtype") == "f32" else 2
    hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
    if case["kind"] == "chunk":
        ctxs, news = _lengths(case)
        pairs = keys = 0
        for c, n in zip(ctxs, news):
            p = np.arange(c, c + n, dtype=np.int64)
            hi = p + 1 if case["causal"] else np.full(n, c + n)
            lo = np.maximum(0, p + 1 - case["window"]) if case["window"] else np.zeros(n, dtype=np.int64)
            pairs += int((hi - lo).sum())
            keys += int(hi[-1] - lo[0])
        return {"bytes": e * dim * (2 * sum(news) * hq + 2 * keys * hkv) + (4 * sum(news) * hq if case["lse"] else 0),
                "flops": 4 * pairs * hq * dim}
    tokens = case["tokens"] if case["kind"] == "rope" else sum(_lengths(case)[1])
    turned = tokens * (hq + hkv)
    copied = tokens * hkv if case["kind"] == "append" else 0
    # every element read and written, its table row and position read; squares, sums, a scale and a weight for each
    # element, and a rotation of two products and a sum
    return {"bytes": 2 * e * dim * (turned + copied) + 4 * tokens * (case["rotary"] + 1),
            "flops": turned * (4 * dim * case["norm"] + 3 * case["rotary"])}
