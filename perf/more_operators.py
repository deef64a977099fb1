"""A paged KV cache held in 8 bits: its pages given out, filled and read.

Three operators, each in a plain form (elementary torch operations in 32 bits, rounded once at the end; whole numbers as
they are) and as the package's entry point:

  pages   a step's pages: sequences grow and shrink, the pages of a pool's free list go to the block table and back, and
          every new token gets its position and its slot in the pool
  append  new keys and values to their pages in e4m3, with a power of two as the scale of each page and head
  attend  attention of chunks of new tokens, of one token to a whole prompt, over such pages

Sizes are those of the package's workloads (32 query / 8 KV heads of 128; contexts of 256 to 32768 keys; blocks of 16 and
31; pages of 16 and 64) and the ranges around them.
"""
import math

import numpy as np
import torch

own = False

MOST_PAIRS = 60_000_000  # padded (query, key) pairs of a drawn case at 32 heads


def _pages(name, seqs, ctx, new, **more):
    """ctx and new as in _lengths; of `leave` sequences one ends, and its pages go back."""
    case = dict(kind="pages", seqs=seqs, ctx=ctx, new=new, mixed=False, leave=0, page=64, shape_seed=3)
    case.update(more)
    return dict(case, name=name) if name else case


def _append(name, seqs, ctx, new, **more):
    """ctx and new are every sequence's keys in the cache and new tokens; mixed: see _lengths."""
    case = dict(kind="append", seqs=seqs, ctx=ctx, new=new, mixed=False, dtype="bf16", hq=32, hkv=8, dim=128, page=64,
                shape_seed=3)
    case.update(more)
    return dict(case, name=name) if name else case


def _attend(name, seqs, ctx, new, **more):
    case = dict(kind="attend", seqs=seqs, ctx=ctx, new=new, mixed=False, hq=32, hkv=8, dim=128, causal=True, window=0,
                lse=False, page=64, shape_seed=3)
    case.update(more)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest call: one request decodes one token
        _pages("pages_1", 1, 2048, 1),
        # a verify pass's blocks of 16 for a batch of 256 requests, some of which end
        _pages("pages_block_256", 256, 4096, 16, mixed=False, leave=20, page=16),
        # a scheduler's step: prompts come in next to decoding requests, and some requests end
        _pages("pages_admit_1024", 1024, 4096, 2000, mixed=True, leave=16),
        # one decoded token
        _append("append_1x1", 1, 2048, 1),
        # a verify pass's blocks, most of which begin inside a page
        _append("append_32x16", 32, 4091, 16),
        # an fp32 model with small heads, a few prompts of an odd length
        _append("append_f32_5x333", 5, 77, 333, dtype="f32", hq=4, hkv=2, dim=64, page=16),
        # the chunk of a long prompt
        _append("append_1x8192", 1, 8192, 8192),
        # one request decodes one token over a chat-length context
        _attend("attend_1x1_2048", 1, 2048, 1, lse=True),
        # a serving batch: prompt chunks and decoding requests in one call
        _attend("attend_mixed_16", 16, 4096, 500, mixed=True, page=16),
        # small heads over a sliding window, 4 prompts of an odd length
        _attend("attend_window_4x2001", 4, 0, 2001, hq=8, hkv=2, dim=64, window=1024),
        # the verify pass of 8 long-context requests, blocks of 31
        _attend("attend_verify_8x31_32768", 8, 32768, 31, lse=True),
        # a whole prompt at once
        _attend("attend_1x8192", 1, 0, 8192),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("pages", "pages", "append", "append", "attend", "attend", "attend", "attend"))
    seed = rng.randrange(1 << 20)
    page = rng.choice((16, 64, 128))
    if kind == "pages":
        seqs = _log_int(rng, 1, 2048)
        mixed = seqs > 3 and rng.random() < 0.5
        return _pages("", seqs, min(_log_int(rng, 0.6, 32768), (1 << 22) // seqs), _log_int(rng, 1, max(2, min(4096, 262144 // seqs))),
                      mixed=mixed, leave=rng.choice((0, 2, 7, 16)) if seqs > 1 else 0, page=page, shape_seed=seed)
    heads = dict(zip(("hq", "hkv"), rng.choice(((32, 8), (32, 8), (8, 2), (8, 8), (4, 2), (12, 4), (10, 2)))))
    dim = rng.choice((64, 128, 128))
    seqs = _log_int(rng, 1, 32)
    ctx = _log_int(rng, 0.6, 32768)
    mixed = seqs > 3 and rng.random() < 0.6
    if kind == "append":
        ctx = min(ctx, 65536 // seqs)
        return _append("", seqs, ctx, _log_int(rng, 1, max(2, 8192 // seqs)), mixed=mixed, page=page, shape_seed=seed,
                       dtype=rng.choice(("bf16", "bf16", "f32")), dim=dim, **heads)
    ctx = min(ctx, 262144 // seqs)
    budget = MOST_PAIRS * 32 // (heads["hq"] * seqs)
    most = int((math.sqrt(ctx * ctx + 4 * budget) - ctx) / 2)  # new * (ctx + new) within the budget
    return _attend("", seqs, ctx, _log_int(rng, 1, max(2, min(8192, most))), mixed=mixed, page=page, shape_seed=seed, dim=dim,
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


def _step(case):
    """Every sequence's keys before and after a step of the scheduler: its new tokens more, or none where it ends."""
    ctxs, news = _lengths(case)
    ends = (np.random.default_rng(case["shape_seed"] + 1).integers(0, case["leave"], size=len(ctxs)) == 0 if case["leave"]
            else np.zeros(len(ctxs), dtype=bool))
    return ctxs, [0 if e else c + n for c, n, e in zip(ctxs, news, ends)]


def _int32(values):
    return torch.tensor(np.asarray(values, dtype=np.int32), device="cuda")


def _offsets(lengths):
    return _int32(np.concatenate([[0], np.cumsum(lengths)]))


def _paging(case, held, need, seed):
    """A block table over a pool of pages, the sequences' pages in shuffled order, and the number of pages; of a
    sequence's `need` places the first `held` are in the table, the others' pages come last in the order."""
    order = np.random.default_rng(seed).permutation(int(sum(need))).astype(np.int32)
    table = np.zeros((len(need), max(1, max(need))), dtype=np.int32)
    for i, part in enumerate(np.split(order[:int(sum(held))], np.cumsum(held)[:-1])):
        table[i, :len(part)] = part
    return table, order[int(sum(held)):]


def _two_to(e):
    """2^e in 32 bits for whole numbers e, by its bits (a library's power need not be exact)."""
    return ((e.to(torch.int32).clamp(-126, 127) + 127) << 23).view(torch.float32)


def _quantised(x, there):
    """[pages, page, heads, dim] in e4m3 with a power of two a page and head, as a cache holds it: its biased exponent is
    the least with no value above 448.  What is not `there` is not a number: memory that nothing has written."""
    top = (x.abs() * there).amax((1, 3), keepdim=True)
    frac, e = torch.frexp(top / 448)
    e = (torch.where(frac == 0.5, e - 1, e) + 127).clamp(1, 254)
    e = torch.where(top == 0, torch.ones_like(e), e)
    q = (x * _two_to(127 - e)).masked_fill_(~there, math.nan).to(torch.float8_e4m3fn)
    return q.flatten(0, 1), e[:, 0, :, 0].to(torch.uint8)


def prepare(case, seed):
    """Projections are N(0, 1) with a width of their own for every head, their queries a little wider, so that a row's
    attention favours some keys; the pool holds them as an earlier append left them."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    page = case["page"]
    up = lambda lengths: [-(-n // page) for n in lengths]  # noqa: E731
    if case["kind"] == "pages":
        before, after = _step(case)
        held, most = up(before), [max(a, b) for a, b in zip(up(before), up(after))]
        table, free = _paging(case, held, most, seed)
        spare = np.arange(len(free) + sum(held), 8 + len(free) + sum(held) * 9 // 8, dtype=np.int32)
        free = np.concatenate([free, np.random.default_rng(seed + 1).permutation(spare)])
        pool = np.full(sum(held) + len(free), -1, dtype=np.int32)
        pool[:len(free)] = free
        return dict(kind="pages", page=page, table=_int32(table), free=_int32(pool), num_free=_int32([len(free)]),
                    before=_int32(before), after=_int32(after), total=sum(max(0, a - b) for a, b in zip(after, before)))
    hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
    ctxs, news = _lengths(case)
    ends = [c + n for c, n in zip(ctxs, news)]
    table, _ = _paging(case, up(ends), up(ends), seed)
    s = dict(kind=case["kind"], page=page, pages=_int32(table), cu_new=_offsets(news), cu_kv=_offsets(ends),
             max_new=max(news), max_kv=max(ends))
    rows = sum(up(ends)) * page

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    width = torch.exp(0.5 * randn(2, hkv, 1))
    there = torch.zeros(rows, dtype=torch.bool, device="cuda")
    at = torch.arange(s["max_kv"], device="cuda")
    held = s["cu_kv"].diff() - (s["cu_new"].diff() if case["kind"] == "append" else 0)
    there[_rows_of(s, at)[at < held[:, None]]] = True
    for i, name in enumerate(("k", "v")):
        s[name + "_cache"], s[name + "_scale"] = _quantised((width[i] * randn(rows, hkv, dim)).view(-1, page, hkv, dim),
                                                            there.view(-1, page, 1, 1))
    t = sum(news)
    if case["kind"] == "attend":
        return dict(s, q=(1.5 * randn(t, hq, dim)).bfloat16(), causal=case["causal"], window=case["window"], lse=case["lse"])
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    # the keys come out of a rotation, the values from a layer's packed projection
    packed = randn(t, hq + 2 * hkv, dim)
    packed[:, hq + hkv:] *= width[1]
    return dict(s, k=(width[0] * randn(t, hkv, dim)).to(dtype), v=packed.to(dtype)[:, hq + hkv:])


def _rows_of(s, at):
    """The pool rows of every sequence's keys `at`: [sequences, len(at)]."""
    return s["pages"].long()[:, at // s["page"]] * s["page"] + at % s["page"]


# --------------------------------------------------------------------------------------------- the plain forms
def _prefix(x):
    return torch.cat([x.new_zeros(1), x.cumsum(0)]).to(torch.int32)


def _plain_update(s, old, new, total):
    """What is given back goes to the front of what can be taken; the rest of that is the free list from its end."""
    table, free, page = s["table"], s["free"], s["page"]
    held, need = (old + page - 1) // page, (new + page - 1) // page
    j = torch.arange(table.shape[1], device="cuda", dtype=torch.int32)
    give = ((j >= need[:, None]) & (j < held[:, None])).flatten()
    take = ((j >= held[:, None]) & (j < need[:, None])).flatten()
    back = free.new_zeros(len(free) + 1)
    back[torch.where(give, give.cumsum(0) - 1, len(free))] = table.flatten()
    given, taken, at, nf = give.sum(), take.sum(), take.cumsum(0) - 1, s["num_free"]
    missing = (taken - given - nf).clamp(min=0)
    ok = missing == 0
    page_id = torch.where(at < given, back[at.clamp(0, len(free) - 1)], free[(nf - 1 - (at - given)).clamp(0, len(free) - 1)])
    table.copy_(torch.where(take & ok, page_id, table.flatten()).view_as(table))
    i = torch.arange(len(free), device="cuda")
    left = ok & (i >= nf) & (i < nf + given - taken)
    free.copy_(torch.where(left, back[(given - 1 - (i - nf)).clamp(0, len(free) - 1)], free))
    s["num_free"].copy_(torch.where(ok, nf + given - taken, nf))
    cu_new = _prefix((new - old).clamp(min=0) * ok)
    cu_kv = _prefix(torch.where(ok, new, old))
    t = torch.arange(total, device="cuda", dtype=torch.int32)
    seq = (torch.searchsorted(cu_new, t, right=True) - 1).clamp(max=len(old) - 1)
    pos = old[seq] + t - cu_new[seq]
    real = t < cu_new[-1]
    slot = table[seq, (pos // page).clamp(0, table.shape[1] - 1)].long() * page + pos % page
    return torch.where(real, pos, -1), torch.where(real, slot, -1), cu_new, cu_kv, missing.to(torch.int32)


def _plain_pages(s):
    """The step's pages, then back to what was held before (the step is cancelled)."""
    got = _plain_update(s, s["before"], s["after"], s["total"])
    back = _plain_update(s, s["after"], s["before"], 0)
    return *got, back[3], back[4], s["table"], s["free"], s["num_free"]


def _plain_append(s):
    """The first page of every sequence is rescaled where the new keys need a larger scale than it has."""
    page, hkv = s["page"], s["k"].shape[1]
    begin = s["cu_kv"].diff() - s["cu_new"].diff()
    t = torch.arange(s["k"].shape[0], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["cu_new"], t, right=True) - 1
    pos = (begin - s["cu_new"][:-1])[seq] + t
    to = s["pages"][seq, pos // page].long()
    first = s["pages"].gather(1, (begin // page).long()[:, None])[:, 0].long()
    i = torch.arange(page, device="cuda")
    rows, old = first[:, None] * page + i, (i < (begin % page)[:, None])[..., None, None]
    for name in ("k", "v"):
        cache, scale, x = s[name + "_cache"].view(torch.uint8), s[name + "_scale"], s[name].float()
        fine = torch.isfinite(x)
        top = torch.zeros(scale.shape, device="cuda").index_reduce_(0, to, torch.where(fine, x.abs(), 0.0).amax(-1), "amax")
        frac, e = torch.frexp(top / 448)
        e = torch.where(top == 0, 1, (torch.where(frac == 0.5, e - 1, e) + 127).clamp(1, 254))
        was = scale[first].to(torch.int32)
        grown = torch.where(old[:, 0, 0], torch.maximum(was, e[first]), e[first])
        held = cache[rows]
        moved = (held.view(torch.float8_e4m3fn).float() * _two_to(was - grown)[:, None, :, None]).to(torch.float8_e4m3fn)
        cache[rows] = torch.where(old, moved.view(torch.uint8), held)
        e[first] = grown
        y = torch.where(fine, x, math.nan) * _two_to(127 - e)[to][..., None]
        cache[to * page + pos % page] = y.to(torch.float8_e4m3fn).view(torch.uint8)
        scale[to] = e[to].to(torch.uint8)
    return s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"]


def _values(s, name, rows):
    scale = _two_to(s[name + "_scale"].to(torch.int32) - 127)[rows // s["page"]]
    return s[name + "_cache"].view(torch.uint8)[rows].view(torch.float8_e4m3fn).float() * scale[..., None]


def _plain_attend(s):
    """The sequences padded to the longest: scores of every (query, key) pair, the hidden ones struck out."""
    q, hkv, dim = s["q"], s["k_cache"].shape[1], s["q"].shape[2]
    group, n, m = q.shape[1] // hkv, s["max_kv"], s["max_new"]
    at, i = torch.arange(n, device="cuda"), torch.arange(m, device="cuda")
    len_kv, len_new = s["cu_kv"].diff()[:, None], s["cu_new"].diff()[:, None]
    there, real = at < len_kv, i < len_new
    rows = _rows_of(s, at)
    k = _values(s, "k", rows).masked_fill(~there[..., None, None], 0.0)
    v = _values(s, "v", rows).masked_fill(~there[..., None, None], 0.0)
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
def _own_pages(s):
    import paper_2606_31315_gb300 as bp

    if "ws" not in s:
        n = len(s["before"])
        new = lambda k, dtype=torch.int32: torch.empty(k, device="cuda", dtype=dtype)  # noqa: E731
        s.update(ws=bp.workspace(256, "cuda"), out=(new(s["total"]), new(s["total"], torch.int64), new(n + 1), new(n + 1), new(1)),
                 back=(None, None, None, new(n + 1), new(1)))
    got = bp.pages_update(s["table"], s["before"], s["after"], s["free"], s["num_free"], s["page"], s["total"], *s["out"], ws=s["ws"])
    back = bp.pages_update(s["table"], s["after"], s["before"], s["free"], s["num_free"], s["page"], None, *s["back"], ws=s["ws"])
    return *got, back[3], back[4], s["table"], s["free"], s["num_free"]


def _own_append(s):
    import paper_2606_31315_gb300 as bp

    if "ws" not in s:
        s["ws"] = bp.workspace(256, "cuda")
    bp.kv_append_fp8(s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"], s["k"], s["v"], s["cu_new"], s["cu_kv"],
                     s["pages"], s["page"], ws=s["ws"])
    return s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"]


def _own_attend(s):
    import paper_2606_31315_gb300 as bp

    q, hkv = s["q"], s["k_cache"].shape[1]
    if "ws" not in s:
        s.update(ws=bp.workspace(bp.chunk_attention_workspace_size(len(s["cu_new"]) - 1, len(q), q.shape[1], hkv, q.shape[2]), "cuda"),
                 out=torch.empty_like(q), lse_out=torch.empty(q.shape[:2], device="cuda") if s["lse"] else None)
    o, lse = bp.chunk_attention_paged_fp8(q, s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"], s["cu_new"], s["cu_kv"],
                                          s["pages"], s["page"], s["max_new"], s["max_kv"],
                                          mask=bp.MASK_CAUSAL if s["causal"] else bp.MASK_BIDIR, window=s["window"],
                                          out=s["out"], lse=s["lse_out"], ws=s["ws"])
    return (o, lse) if s["lse"] else o


_PLAIN = dict(pages=_plain_pages, append=_plain_append, attend=_plain_attend)
_OWN = dict(pages=_own_pages, append=_own_append, attend=_own_attend)


def run(state):
    return (_OWN if own else _PLAIN)[state["kind"]](state)


# --------------------------------------------------------------------------------------------- in 64 bits
def _power(e):
    """2^e in 64 bits for whole numbers e, by its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _value_of(codes):
    """What an e4m3 code stands for, by its bits."""
    codes = codes.long()
    e, m = codes >> 3 & 15, (codes & 7).double()
    x = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * _power(e - 10))
    return torch.where(codes & 127 == 127, math.nan, torch.where(codes > 127, -x, x))


def _nearest(x):
    """The e4m3 value nearest to each x of at most 448, the even one of two."""
    step = _power((x.abs().clamp(min=2.0 ** -6).view(torch.int64) >> 52) - 1023 - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    if case["kind"] == "pages":
        return None  # whole numbers
    s = prepare(case, seed)
    ctxs, news = _lengths(case)
    page, hkv = case["page"], case["hkv"]
    keys = [_rows_of(s, torch.arange(c + n, device="cuda"))[i] for i, (c, n) in enumerate(zip(ctxs, news))]
    if case["kind"] == "append":
        out = []
        for name in ("k", "v"):
            codes = _value_of(s[name + "_cache"].view(torch.uint8))
            scale = s[name + "_scale"].long()
            first = 0
            for c, n, rows in zip(ctxs, news, keys):
                x = s[name][first:first + n].double()
                first += n
                for lo in range(c // page * page, c + n, page):
                    a, b = max(lo, c), min(lo + page, c + n)
                    part, p = x[a - c:b - c], rows[a] // page
                    top = part.abs().amax((0, 2))
                    e = (top.view(torch.int64) >> 52) - 1023 - 8 + 127  # 448 is 1.75 times 2^8
                    e += top > 448 * _power(e - 127)
                    if a > lo:
                        e = torch.maximum(e, scale[p])
                        codes[rows[lo:a]] = _nearest(codes[rows[lo:a]] * _power(scale[p] - e)[:, None])
                    codes[rows[a:b]] = _nearest(part * _power(127 - e)[:, None])
                    scale[p] = e
            out += [codes, None]
        return tuple(out)
    value = {name: _value_of(s[name + "_cache"].view(torch.uint8)) * _power(s[name + "_scale"].long() - 127)
             .repeat_interleave(page, 0)[..., None] for name in ("k", "v")}
    out, lses, first = [], [], 0
    for c, n, rows in zip(ctxs, news, keys):
        p, j = torch.arange(c, c + n, device="cuda")[:, None], torch.arange(c + n, device="cuda")[None, :]
        hidden = (j > p) if case["causal"] else torch.zeros(n, c + n, dtype=torch.bool, device="cuda")
        if case["window"]:
            hidden = hidden | (p - j >= case["window"])
        o, z = [], []
        for h in range(case["hq"]):
            kv = h // (case["hq"] // hkv)
            x = s["q"][first:first + n, h].double() @ value["k"][rows, kv].T / case["dim"] ** 0.5
            x[hidden] = -math.inf
            z.append(torch.logsumexp(x, 1))
            o.append(torch.exp(x - z[-1][:, None]) @ value["v"][rows, kv])
        out.append(torch.stack(o, 1))
        lses.append(torch.stack(z, 1))
        first += n
    return (torch.cat(out), torch.cat(lses)) if case["lse"] else torch.cat(out)


# --------------------------------------------------------------------------------------------- what a pass has to do
def work(case):
    page = case["page"]
    if case["kind"] == "pages":
        before, after = (np.asarray(x, dtype=np.int64) for x in _step(case))
        moved = int(np.abs(-(-after // page) + before // -page).sum())
        tokens = int(np.maximum(after - before, 0).sum())
        # twice (the step and back): the lengths read, offsets written, a page's number read in one place and written in
        # another; once a position and a slot for every token; a division a length, page and token
        return {"bytes": 2 * (8 + 4) * len(before) + 4 * len(before) + 2 * 8 * moved + 12 * tokens,
                "flops": 4 * len(before) + 2 * moved + 2 * tokens}
    hkv, dim = case["hkv"], case["dim"]
    ctxs, news = _lengths(case)
    if case["kind"] == "append":
        e = 4 if case["dtype"] == "f32" else 2
        values = 2 * sum(news) * hkv * dim
        touched = sum(-(-(c + n) // page) - c // page for c, n in zip(ctxs, news))
        # every value read, compared, scaled and rounded, written in one byte; the scale of every page and head
        return {"bytes": (e + 1) * values + 2 * 2 * touched * hkv, "flops": 3 * values}
    hq = case["hq"]
    pairs = keys = pages = 0
    for c, n in zip(ctxs, news):
        p = np.arange(c, c + n, dtype=np.int64)
        hi = p + 1 if case["causal"] else np.full(n, c + n)
        lo = np.maximum(0, p + 1 - case["window"]) if case["window"] else np.zeros(n, dtype=np.int64)
        pairs += int((hi - lo).sum())
        keys += int(hi[-1] - lo[0])
        pages += int(-(-hi[-1] // page) - lo[0] // page)
    return {"bytes": 2 * dim * 2 * sum(news) * hq + 2 * keys * hkv * dim + 2 * pages * hkv + (4 * sum(news) * hq if case["lse"] else 0),
            "flops": 4 * pairs * hq * dim}
