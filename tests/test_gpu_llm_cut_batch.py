"""A step whose token batch is longer than its list of slots: requests whose rows do not all have a slot are left for a later step."""
import pytest
import torch

import paper_2505_20932_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I4 = torch.int32


def _ints(v):
    return torch.tensor(v, dtype=I4, device=DEV)


def _step(old, new, free, n_free, table, cap):
    slots = torch.full((cap,), -77, dtype=torch.int64, device=DEV)
    start, lens, left = (torch.full((n,), -77, dtype=I4, device=DEV) for n in (len(old) + 1, len(old), 1))
    P.llm_kv_assign_pages(_ints(old), _ints(new), 16, free, _ints([n_free]), table, slots, start, lens, left)
    return slots.tolist(), start.tolist(), lens.tolist(), left.item()


@pytest.mark.parametrize("cap", [46, 45, 44, 25, 24, 5, 4, 1])
def test_requests_without_all_their_slots_wait(cap):
    old, new = [0, 16, 3, 0, 30], [5, 0, 20, 0, 20]                    # rows 0 .. 4, none, 5 .. 24, none, 25 .. 44
    free = torch.arange(40, dtype=I4, device=DEV)
    table = torch.full((5, 4), -1, dtype=I4, device=DEV)
    table[1, 0], table[2, 0], table[4, 0], table[4, 1] = 100, 101, 102, 103
    before = table.clone()
    slots, start, lens, left = _step(old, new, free, 40, table, cap)
    got = [i for i in range(5) if new[i] == 0 or start[i + 1] <= cap]
    assert start == [0, 5, 5, 25, 25, 45]
    assert lens == [old[i] + new[i] if i in got else old[i] for i in range(5)]
    need = [-(-(old[i] + new[i]) // 16) - -(-old[i] // 16) for i in range(5)]
    assert left == 40 - sum(need[i] for i in got)
    for i in range(5):
        rows = slots[start[i]:start[i + 1]]
        if i in got:
            want = [int(table[i, (old[i] + j) // 16]) * 16 + (old[i] + j) % 16 for j in range(new[i])]
            assert rows == want and all(s >= 0 for s in rows)
        else:
            assert all(s == -1 for s in rows) and torch.equal(table[i], before[i])
    # the rest, in a step of its own
    if len(got) < 5:
        later = [0 if i in got else new[i] for i in range(5)]
        _, _, lens, left = _step(lens, later, free, left, table, sum(later))
        assert lens == [o + n for o, n in zip(old, new)] and left == 40 - sum(need)


def test_no_list_of_slots_reserves_pages():
    table = torch.full((2, 4), -1, dtype=I4, device=DEV)
    free = torch.arange(9, dtype=I4, device=DEV)
    slots, start, lens, left = _step([0, 20], [40, 1], free, 9, table, 0)
    assert slots == [] and start == [0, 40, 41] and lens == [40, 21] and left == 6 and table[0].tolist() == [8, 7, 6, -1]
