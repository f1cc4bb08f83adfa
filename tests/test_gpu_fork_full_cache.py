"""Rows that change places in a cache whose ring has no page left: what a caller can do before, and after, a call in which rows got none."""
import random

import pytest
import torch

from tests.test_gpu_page_fork import check, i32
from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu


def beams(B, p, seed):
    """Rows of a few full pages and a part of one, some full ones shared; the ring is empty."""
    rng = random.Random(seed)
    n, table, seq = 0, [], []
    for b in range(B):
        m = rng.randint(1, 5) * p + rng.randint(1, p - 1)
        shared = rng.randint(0, min(m, seq[b - 1]) // p) if b else 0
        mine = (table[b - 1][:shared] if b else []) + list(range(n, n + -(-m // p) - shared))
        n += -(-m // p) - shared
        table.append(mine + [-1] * (7 - len(mine)))
        seq.append(m)
    from_ = [rng.randrange(B) for _ in range(B)]
    return table, seq, from_, n


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B", [4, 40, 1100])
def test_pages_of_rows_that_nobody_comes_from_are_given_back_by_a_call_before(ac, B, in_place):  # noqa: F811
    p = 8
    for seed in range(3):
        table, seq, from_, n = beams(B, p, seed)
        ring = [-1] * n
        direct = check(ac, table, seq, from_, ring, 0, 0, 1, p, 4, "f32", in_place)
        assert -1 in direct[1] or from_ == sorted(set(from_))
        used = set(from_)
        t, s, r, state = check(ac, table, seq, [b if b in used else -1 for b in range(B)], ring, 0, 0, 1, p, 4, "f32", True)
        assert state[1] >= B - len(used)      # a page at least of each: as many as there are copies
        t, s, r, state = check(ac, t, s, from_, r, *state, 1, p, 4, "f32", in_place)
        assert s == [seq[f] for f in from_]


@pytest.mark.parametrize("B", [30, 1100])
def test_outputs_of_their_own_leave_the_inputs_to_go_on_from(ac, B):  # noqa: F811
    """Tables, lengths, the ring's entries in use and pages that rows hold are what they were, also where rows got no page."""
    p, H, D = 8, 1, 4
    table, seq, from_, n = beams(B, p, 5)
    n += 3
    ring = [n - 3, n - 2, n - 1] + [-1] * (n - 3)
    first = n - 2                                    # (the ring's entries go over its end)
    ring = [ring[(i - first) % n] for i in range(n)]
    held = torch.tensor(sorted({q for r in table for q in r if q >= 0}), device="cuda")
    k, v = (torch.randn(n, H, p, D, device="cuda") for _ in range(2))
    t, s, state, r, f = i32(table), i32(seq), i32([first, 3]), i32(ring), i32(from_)
    ws = torch.empty(ac.attncache_page_fork_workspace_bytes(B, 7, n), dtype=torch.uint8, device="cuda")
    keep = [x.clone() for x in (t, s, state, r, k, v)]

    def fork(source):
        out = [torch.full_like(x, -9) for x in (t, s, state)]
        ac.attncache_page_fork(source, s, state, r, t, *out, k, v, ws)
        return out

    assert (fork(f)[1] == -1).sum() == B - len(set(from_)) - 3 > 0
    inuse = [(first + i) % n for i in range(3)]
    assert torch.equal(t, keep[0]) and torch.equal(s, keep[1]) and torch.equal(state, keep[2]) and torch.equal(r[inuse], keep[3][inuse])
    assert torch.equal(k[held], keep[4][held]) and torch.equal(v[held], keep[5][held])
    # from the same inputs: first what nobody goes on with, then all rows, each of which holds what its source held
    used = set(from_)
    t, s, state = fork(i32([b if b in used else -1 for b in range(B)]))
    t, s, state = fork(f)
    assert s.tolist() == [seq[x] for x in from_]
    rows = t.tolist()
    for b in range(0, B, 1 + B // 50):
        for j in range(seq[from_[b]]):
            q = table[from_[b]][j // p]
            assert torch.equal(k[rows[b][j // p], :, j % p], keep[4][q, :, j % p]) and torch.equal(v[rows[b][j // p], :, j % p], keep[5][q, :, j % p])
