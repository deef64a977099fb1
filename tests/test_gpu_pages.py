"""pages_update against its definition, in Python: tables, list and places have to be equal; and the operators of the cache in 8
bits together, as a loop of verify steps uses them."""
import numpy as np
import pytest
import torch

import paper_2606_31315_gb300 as bp
from _fp8 import Append, attention

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


class Pages:
    """The operator by its definition."""

    def __init__(self, table, free, num_free, page):
        self.table, self.free, self.num_free, self.page = table.copy(), free.copy(), num_free, page

    def __call__(self, old, new, total):
        up = lambda n: -(-n // self.page)  # noqa: E731
        back = [self.table[s, j] for s, (a, b) in enumerate(zip(old, new)) for j in range(up(b), up(a))]
        wants = [(s, j) for s, (a, b) in enumerate(zip(old, new)) for j in range(up(a), up(b))]
        missing = max(0, len(wants) - len(back) - self.num_free)
        if missing:
            return np.full(total, -1), np.full(total, -1), np.zeros(len(old) + 1), np.concatenate([[0], np.cumsum(old)]), missing
        stack = list(self.free[:self.num_free]) + back[::-1]
        for s, j in wants:
            self.table[s, j] = stack.pop()
        self.free[:len(stack)], self.num_free = stack, len(stack)
        pos = [p for a, b in zip(old, new) for p in range(a, b)]
        slot = [int(self.table[s, p // self.page]) * self.page + p % self.page for s, (a, b) in enumerate(zip(old, new)) for p in range(a, b)]
        pad = [-1] * (total - len(pos))
        grown = [max(0, b - a) for a, b in zip(old, new)]
        return np.array(pos + pad), np.array(slot + pad), np.concatenate([[0], np.cumsum(grown)]), np.concatenate([[0], np.cumsum(new)]), 0


def setup(lens, page, per, spare, seed=0):
    g = np.random.default_rng(seed)
    need = [-(-n // page) for n in lens]
    ids = g.permutation(sum(need) + spare).astype(np.int32)
    table = np.full((len(lens), per), -5, dtype=np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = ids[at:at + n]
        at += n
    free = np.full(len(ids), -7, dtype=np.int32)
    free[:spare] = ids[at:]
    return table, free, spare


def step(state, old, new, ref, total=None, ws=None):
    grown = sum(max(0, b - a) for a, b in zip(old, new))
    total = grown if total is None else total
    table, free, num = state
    got = bp.pages_update(table, i32(old), i32(new), free, num, ref.page, total, ws=ws)
    wanted = ref(old, new, total)
    for x, y in zip(got, wanted):
        np.testing.assert_array_equal(x.cpu().numpy(), np.atleast_1d(y))
    np.testing.assert_array_equal(table.cpu().numpy(), ref.table)
    assert int(num) == ref.num_free
    np.testing.assert_array_equal(free.cpu().numpy()[:ref.num_free], ref.free[:ref.num_free])


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("seqs", [1, 3, 31, 33, 513, 2000])
def test_random_steps(seqs, page):
    """Steps of growth, rollbacks, ends and new prompts; padded outputs."""
    g = np.random.default_rng(seqs)
    lens = g.integers(0, 300, seqs).tolist()
    per = 800 // page + 1
    t, f, n = setup(lens, page, per, 3 * seqs * (200 // page + 1), seed=seqs)
    ref, state, ws = Pages(t, f, n, page), (i32(t), i32(f), i32([n])), bp.workspace(256, "cuda")
    for k in range(6):
        kind = g.integers(0, 4, seqs)
        new = [0 if a == 0 else max(0, l - int(g.integers(0, 40))) if a == 1 else l if a == 2 else min(800, l + int(g.integers(1, 200)))
               for a, l in zip(kind, lens)]
        short = sum(-(-b // page) for b in new) - sum(-(-a // page) for a in lens) > int(state[2])
        step(state, lens, new, ref, total=None if k % 2 else sum(max(0, b - a) for a, b in zip(lens, new)) + 37, ws=ws)
        lens = lens if short else new
    assert bp.get_status(ws) == 0


def test_giving_back_restores_the_list():
    lens, page = [5, 100, 64, 0, 17], 16
    t, f, n = setup(lens, page, 20, 40)
    ref, state = Pages(t, f, n, page), (i32(t), i32(f), i32([n]))
    new = [200, 0, 64, 33, 160]
    step(state, lens, new, ref)
    step(state, new, lens, ref, total=200)
    assert torch.equal(state[1], i32(f)) and int(state[2]) == n
    for s, l in enumerate(lens):
        assert torch.equal(state[0][s, :-(-l // page)], i32(t[s, :-(-l // page)]))


def test_too_few_pages_change_nothing():
    lens, page = [10, 33], 16
    t, f, n = setup(lens, page, 10, 2)
    ref, state, ws = Pages(t, f, n, page), (i32(t), i32(f), i32([n])), bp.workspace(256, "cuda")
    step(state, lens, [100, 33], ref, total=120, ws=ws)   # 6 wanted, 2 there
    step(state, lens, [100, 0], ref, ws=ws)               # 6 wanted, 2 + 3 there
    step(state, lens, [80, 0], ref, ws=ws)                # 4 wanted
    assert bp.get_status(ws) == 0


def test_outputs_that_are_not_wanted_and_tables_with_views():
    lens, page = [10, 33], 16
    t, f, n = setup(lens, page, 10, 8)
    ref, (table, free, num) = Pages(t, f, n, page), (i32(t), i32(f), i32([n]))
    got = bp.pages_update(table, i32(lens), i32([50, 40]), free, num, page, None)
    wanted = ref(lens, [50, 40], 47)
    assert got[0] is None and got[1] is None and int(got[4]) == 0
    np.testing.assert_array_equal(got[3].cpu().numpy(), wanted[3])
    np.testing.assert_array_equal(table.cpu().numpy(), ref.table)


@pytest.mark.parametrize("old,new,num", [([-1, 5], [5, 5], 4), ([5, 5], [-3, 5], 4), ([5, 5], [5, 161], 4), ([5, 161], [5, 5], 4),
                                         ([5, 5], [5, 5], -1), ([5, 5], [5, 5], 100), ([100, 5], [0, 5], 6), ([5, 5], [90, 5], 4)])
def test_refused_by_the_device(old, new, num):
    """Lengths below 0 or past a row, a list that cannot be, more tokens than there is room for: nothing changes."""
    t, f, _ = setup([5, 5], 16, 10, 8)
    table, free, count, ws = i32(t), i32(f), i32([num]), bp.workspace(256, "cuda")
    got = bp.pages_update(table, i32(old), i32(new), free, count, 16, 84 if new == [90, 5] else 200, ws=ws)
    assert bp.get_status(ws) == 6
    assert torch.equal(table, i32(t)) and torch.equal(free, i32(f)) and int(count) == num
    assert (got[0] == -1).all() and (got[1] == -1).all() and (got[2] == 0).all()


def test_the_largest_number_of_sequences():
    seqs = 16384
    t, f, n = setup([1] * seqs, 16, 3, seqs)
    ref, state = Pages(t, f, n, 16), (i32(t), i32(f), i32([n]))
    step(state, [1] * seqs, [17 if s % 2 else 0 for s in range(seqs)], ref)


def test_a_loop_of_verify_steps():
    """What a step of a serving loop does, captured once and replayed: pages for the block, queries and keys normed and rotated,
    the append, attention over the pages, the commit's new lengths, the dropped tokens' pages given back.  The cache and the
    outputs as by their definitions in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(1)
    hq, hkv, dim, page, block, seqs = 8, 2, 128, 16, 6, 3
    start, per = [0, 13, 40], 12
    t, f, n = setup(start, page, per, 20)
    pages = Pages(t, f, n, page)
    table, free, num = i32(t), i32(f), i32([n])
    rows = len(f) * page
    cache = dict(table=table, page=page)
    for name in "kv":
        cache[name] = torch.full((rows, hkv, dim), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        cache[name + "_scale"] = torch.full((len(f), hkv), 120, dtype=torch.uint8, device="cuda")
    small = [bp.workspace(256, "cuda") for _ in range(4)]
    held, grown = i32(start), i32([0] * seqs)
    # the contexts before the loop
    x = torch.randn(sum(start), 2 * hkv, dim, device="cuda", generator=g).to(torch.bfloat16)
    bp.kv_append_fp8(cache["k"], cache["k_scale"], cache["v"], cache["v_scale"], x[:, :hkv], x[:, hkv:],
                     i32([0, *np.cumsum(start)]), i32([0, *np.cumsum(start)]), table, page, ws=small[1])
    angle = torch.arange(per * page, device="cuda")[:, None] * torch.linspace(1.0, 0.01, dim // 2, device="cuda")
    turn = torch.cat([angle.cos(), angle.sin()], 1)
    packed = torch.zeros(seqs * block, hq + 2 * hkv, dim, device="cuda", dtype=torch.bfloat16)
    accepted, tokens = i32([0] * seqs), i32([0] * (seqs * block))
    cu_draft = i32(np.arange(seqs + 1) * (block - 1))
    pos, slots, cu_new, cu_kv, missing = (torch.empty(seqs * block, dtype=torch.int32, device="cuda"),
                                          torch.empty(seqs * block, dtype=torch.int64, device="cuda"), i32([0] * (seqs + 1)),
                                          i32([0] * (seqs + 1)), i32([0]))
    q = torch.empty(seqs * block, hq, dim, device="cuda", dtype=torch.bfloat16)
    k = torch.empty(seqs * block, hkv, dim, device="cuda", dtype=torch.bfloat16)
    out = torch.empty_like(q)
    ws = bp.workspace(bp.chunk_attention_workspace_size(seqs, seqs * block, hq, hkv, dim), "cuda")
    next_kv = i32([0] * (seqs + 1))

    def one():
        grown.copy_(held + block)
        bp.pages_update(table, held, grown, free, num, page, seqs * block, pos, slots, cu_new, cu_kv, missing, ws=small[0])
        bp.qk_norm_rope(packed[:, :hq], packed[:, hq:hq + hkv], turn, pos, q_out=q, k_out=k, ws=small[2])
        bp.kv_append_fp8(cache["k"], cache["k_scale"], cache["v"], cache["v_scale"], k, packed[:, hq + hkv:], cu_new, cu_kv, table,
                         page, ws=small[1])
        bp.chunk_attention_paged_fp8(q, cache["k"], cache["k_scale"], cache["v"], cache["v_scale"], cu_new, cu_kv, table, page, block,
                                     per * page, out=out, ws=ws)
        bp.verify_commit(held, accepted, tokens, cu_draft, per * page, cu_kv_next=next_kv, ws=small[3])
        bp.pages_update(table, grown, held, free, num, page, None, cu_new=i32_a, cu_kv=i32_b, missing=i32_c, ws=small[0])

    i32_a, i32_b, i32_c = i32([0] * (seqs + 1)), i32([0] * (seqs + 1)), i32([0])
    keep = [x.clone() for x in (table, free, num, held, *(cache[m].view(torch.uint8) for m in "kv"), cache["k_scale"], cache["v_scale"])]
    one()  # warm
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        one()
    for x, y in zip((table, free, num, held, *(cache[m].view(torch.uint8) for m in "kv"), cache["k_scale"], cache["v_scale"]), keep):
        x.copy_(y)
    lens = list(start)
    refs = {m: Append(cache[m].view(torch.uint8).cpu().numpy(), cache[m + "_scale"].cpu().numpy(), page) for m in "kv"}
    rng = np.random.default_rng(2)
    for _ in range(7):
        packed.copy_(torch.randn(packed.shape, device="cuda", generator=g))
        took = rng.integers(0, block, seqs)
        accepted.copy_(i32(took))
        graph.replay()
        torch.cuda.synchronize()
        new = [n + block for n in lens]
        wanted = pages(lens, new, seqs * block)
        np.testing.assert_array_equal(pos.cpu().numpy(), wanted[0])
        np.testing.assert_array_equal(slots.cpu().numpy(), wanted[1])
        for m, x in (("k", k), ("v", packed[:, hq + hkv:])):
            for s in range(seqs):
                refs[m](x[s * block:(s + 1) * block].float().cpu().numpy(), lens[s], pages.table[s])
        for m in "kv":
            np.testing.assert_array_equal(cache[m].view(torch.uint8).cpu().numpy(), refs[m].codes)
            np.testing.assert_array_equal(cache[m + "_scale"].cpu().numpy(), refs[m].scale)
        o, _, bound, _ = attention(dict(cache, table=i32(pages.table)), q, [block] * seqs, new, True, 0)
        assert ((out.double() - o).abs() <= bound).all()
        after = [n + 1 + int(a) for n, a in zip(lens, took)]
        pages(new, after, 0)
        lens = after
        np.testing.assert_array_equal(table.cpu().numpy(), pages.table)
        assert held.tolist() == lens and int(num) == pages.num_free
    assert all(bp.get_status(w) == 0 for w in (*small, ws)) and int(missing) == 0
