"""What pages_update refuses on the device that tests/test_gpu_pages.py does not have, and the steps that do not take place."""
import numpy as np
import pytest
import torch

import paper_2606_31315_gb300 as bp

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


@pytest.mark.parametrize("room", [0, 5, 6])
def test_more_new_tokens_than_there_is_room_for(room):
    """Room for none is room too: 6 new tokens are one too many for 5, and six too many for 0, which is the default."""
    table, free, count, ws = i32([[3, 9]]), i32([0, 1, 2, 4] + [0] * 6), i32([4]), bp.workspace(256, "cuda")
    keep = [x.clone() for x in (table, free, count)]
    got = bp.pages_update(table, i32([14]), i32([20]), free, count, 16, *([room] if room else []), ws=ws)
    fits = room == 6
    assert bp.get_status(ws) == (0 if fits else 6)
    assert got[0].tolist() == (list(range(14, 20)) if fits else [-1] * room) and got[2].tolist() == ([0, 6] if fits else [0, 0])
    assert got[3].tolist() == [0, 20 if fits else 14] and int(got[4]) == 0
    if fits:
        assert table.tolist() == [[3, 4]] and int(count) == 3
    else:
        assert all(torch.equal(x, y) for x, y in zip((table, free, count), keep))


def test_no_new_tokens_and_no_room():
    """Sequences that shrink or stay need none."""
    table, free, count, ws = i32([[3, 9], [1, 0]]), i32([2, 4] + [0] * 8), i32([2]), bp.workspace(256, "cuda")
    got = bp.pages_update(table, i32([20, 5]), i32([3, 5]), free, count, 16, ws=ws)
    assert bp.get_status(ws) == 0 and int(count) == 3 and free[:3].tolist() == [2, 4, 9]
    assert got[0].numel() == 0 and got[2].tolist() == [0, 0, 0] and got[3].tolist() == [0, 3, 8]


@pytest.mark.parametrize("seqs", [1, 127, 128, 129, 513, 3000, 16384])
def test_too_few_pages_for_many_sequences(seqs):
    """Nothing changes: the offsets are those of the old lengths, of all sequences."""
    g = np.random.default_rng(seqs)
    old = g.integers(0, 33, seqs)
    new = np.where(g.integers(0, 4, seqs) == 0, 0, old + 16)
    need = lambda x: -(-x // 16)  # noqa: E731
    held = need(old)
    table = np.full((seqs, 4), -5, dtype=np.int32)
    table[np.arange(4)[None] < held[:, None]] = np.arange(held.sum())
    wanted, back = np.maximum(need(new) - held, 0).sum(), np.maximum(held - need(new), 0).sum()
    spare = max(0, int(wanted - back) - 1)
    pool = np.zeros(held.sum() + spare + 9, dtype=np.int32)
    pool[:spare] = held.sum() + np.arange(spare)
    state = [i32(table), i32(pool), i32([spare])]
    keep = [x.clone() for x in state]
    ws = bp.workspace(256, "cuda")
    if wanted - back <= spare:  # (one sequence that ends, or needs a page that is there)
        new = old + 32
        wanted, back = (need(new) - held).sum(), 0
    got = bp.pages_update(state[0], i32(old), i32(new), state[1], state[2], 16, 40, ws=ws)
    if np.maximum(new - old, 0).sum() > 40:  # (more than there is room for: refused before the pages are counted)
        assert bp.get_status(ws) == 6 and int(got[4]) == 0
        got = bp.pages_update(state[0], i32(old), i32(new), state[1], state[2], 16, None, ws=ws)
    assert bp.get_status(ws) == 0 and int(got[4]) == wanted - back - spare
    assert (got[2] == 0).all() and got[3].tolist() == [0, *np.cumsum(old).tolist()]
    assert all(torch.equal(x, y) for x, y in zip(state, keep))
