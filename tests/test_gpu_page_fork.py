"""Rows of a cache that become other rows, against the same kept by hand: tables, the ring, lengths and every place of the pages."""
import random

import pytest
import torch

from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def fork(table, seq, from_, ring, first, count, p, n, sinks, window):
    """-> table rows of the new entries, lengths, ring, state, moves (from page, to page, tokens)."""
    B, width = len(seq), len(table[0])
    held = lambda t: -(-t // p)  # noqa: E731
    seq = [min(max(s, 0), width * p) for s in seq]
    rows, lens, moves, queue = [], [], [], 0
    for b, s in enumerate(from_):
        if not 0 <= s < B:
            rows.append([])
            lens.append(0)
            continue
        m, mine = seq[s], table[s][:held(seq[s])]
        keeper = s if from_[s] == s else from_.index(s)
        if m % p and keeper != b:
            queue += 1
            if queue > count:
                rows.append([])
                lens.append(-1)
                continue
            fresh = ring[(first + queue - 1) % n]
            moves.append((mine[-1], fresh, m % p))
            mine = mine[:-1] + [fresh]
        rows.append([-1 if window and (j + 1) * p <= m - window and j * p >= sinks else q for j, q in enumerate(mine)])
        lens.append(m)
    ok = lambda q: 0 <= q < n  # noqa: E731
    had = {q for t, s in zip(table, seq) for q in t[:held(s)] if ok(q)}
    gone = sorted(had - {q for r in rows for q in r if ok(q)})
    out = ring[:]
    for i, q in enumerate(gone):
        out[(first + count + i) % n] = q
    return rows, lens, out, [(first + len(moves)) % n, count - len(moves) + len(gone)], moves


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def call(ac, table, seq, from_, ring, state, k, v, in_place, **kw):  # noqa: F811
    """One call on copies: what came back."""
    t = [i32(x) for x in (table, seq, state)]
    out = t if in_place else [torch.full_like(x, -99) for x in t]
    r, f = i32(ring), i32(from_)
    ws = torch.full((ac.attncache_page_fork_workspace_bytes(*t[0].shape, len(ring)) // 4 + 1,), -1, dtype=torch.int32, device="cuda")
    ac.attncache_page_fork(f, t[1], t[2], r, t[0], out[0], out[1], out[2], k, v, ws[:-1], **kw)
    assert ws[-1] == -1 and f.tolist() == from_
    return out[0].tolist(), out[1].tolist(), r.tolist(), out[2].tolist()


def check(ac, table, seq, from_, ring, first, count, H, p, D, dt, in_place, sinks=0, window=0, apart=0):  # noqa: F811
    n = len(ring)
    size = H * p * D + apart
    g = torch.Generator(device="cuda").manual_seed(n + p)
    k, v = (torch.randn(n, size, generator=g, device="cuda").to(DT[dt]) for _ in range(2))
    k0, v0 = k.clone(), v.clone()
    view = lambda t: t.as_strided((n, H, p, D), (size, p * D, D, 1))  # noqa: E731
    rows, lens, ring_, state, moves = fork(table, seq, from_, ring, first, count, p, n, sinks, window)
    got = call(ac, table, seq, from_, ring, [first, count], view(k), view(v), in_place, sinks=sinks, window=window)
    keep = table if in_place else [[-99] * len(t) for t in table]
    assert got[0] == [r + t[len(r):] for r, t in zip(rows, keep)]
    assert got[1:] == (lens, ring_, state)
    for a, b, m in moves:
        view(k0)[b, :, :m], view(v0)[b, :, :m] = view(k0)[a, :, :m], view(v0)[a, :, :m]
    assert torch.equal(k, k0) and torch.equal(v, v0)
    return got


def cache(rng, B, p, hi, share=0.5, spare=20):
    """Rows that share some full pages; a ring of the others."""
    width = -(-hi // p) + 1
    n = B * width + spare
    pages = list(range(n))
    rng.shuffle(pages)
    table, seq = [], []
    for b in range(B):
        m = rng.choice([0, 1, p, hi, rng.randint(0, hi)])
        held = -(-m // p)
        row = []
        if b and rng.random() < share:
            of = rng.randrange(b)
            row = table[of][:min(seq[of] // p, m // p)]
        row = row + [pages.pop() for _ in range(held - len(row))]
        table.append(row + [-1] * (width - held))
        seq.append(m)
    first = rng.randrange(n)
    ring = [-1] * n
    for i, q in enumerate(pages):
        ring[(first + i) % n] = q
    return table, seq, ring, first, len(pages)


# rows, page size, most tokens: one workgroup's work, and more rows, entries or pages than that
PLACES = [(1, 16, 40), (2, 1, 9), (7, 4, 50), (33, 16, 300), (64, 10, 1000), (300, 16, 100), (1024, 8, 100), (1500, 8, 40), (5, 128, 2000), (4, 1, 5000)]
TYPES = [(1, 64, "bf16", 0), (8, 128, "bf16", 64), (128, 64, "bf16", 0), (3, 33, "f32", 0), (2, 199, "f32", 5), (5, 256, "f32", 4), (1, 1, "f32", 0)]
# rows, page size, pages of a row, pages
LARGE = [(3000, 4, 3, 4000), (9, 16, 2000, 20000), (5, 4, 10, 70000)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,p,hi", PLACES)
def test_rows_change_places(ac, B, p, hi, in_place):  # noqa: F811
    for seed in range(3):
        rng = random.Random(B + seed)
        table, seq, ring, first, count = cache(rng, B, p, hi)
        from_ = [rng.choice([b, rng.randrange(B), rng.randrange(B), -1]) for b in range(B)]
        check(ac, table, seq, from_, ring, first, count, 2, p, 4, "f32", in_place)


@pytest.mark.parametrize("H,D,dt,apart", TYPES)
def test_types_and_strides(ac, H, D, dt, apart):  # noqa: F811
    rng = random.Random(D)
    table, seq, ring, first, count = cache(rng, 12, 16, 100)
    from_ = [rng.randrange(12) for _ in range(12)]
    check(ac, table, seq, from_, ring, first, count, H, 16, D, dt, False, apart=apart)


def test_many_answers_to_one_prompt_and_many_copies(ac):  # noqa: F811
    rng = random.Random(0)
    for B, p, m in ((256, 16, 1003), (3000, 4, 7)):
        table, seq, ring, first, count = cache(rng, 1, p, m, spare=B + 5)
        held = -(-m // p)
        table = [ring_pages(ring, first, held) + [-1]] + [[-1] * (held + 1) for _ in range(B - 1)]
        first, count = (first + held) % len(ring), count - held
        got = check(ac, table, [m] + [0] * (B - 1), [0] * B, ring, first, count, 1, p, 64, "bf16", False)
        assert got[1] == [m] * B


def ring_pages(ring, first, k):
    return [ring[(first + i) % len(ring)] for i in range(k)]


@pytest.mark.parametrize("in_place", [False, True])
def test_a_ring_that_runs_out(ac, in_place):  # noqa: F811
    """Rows that get no page hold nothing, in order; a page given back serves the next call."""
    p, seq = 4, [6, 0, 0, 0, 8]
    table = [[0, 1, -1], [-1] * 3, [-1] * 3, [-1] * 3, [2, 3, -1]]
    for count in (0, 1, 2, 5):
        ring = [9, 8, 7, 6, 5] + [-1] * 5
        got = check(ac, table, seq, [0, 0, 0, 0, -1], ring, 0, count, 1, p, 4, "f32", in_place)
        assert got[1] == [6] + [6 if i < count else -1 for i in range(3)] + [0]
        assert got[3] == [min(3, count), count - min(3, count) + 2]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,p,width,n", LARGE)
@pytest.mark.parametrize("dt,D", [("bf16", 64), ("f32", 33)])
def test_more_than_a_workgroup_plans(ac, B, p, width, n, dt, D, in_place):  # noqa: F811
    rng = random.Random(B)
    pages = list(range(n))
    rng.shuffle(pages)
    seq = [rng.choice([0, 3, width * p, rng.randint(0, width * p)]) if b < 7 else rng.randint(0, 3) for b in range(B)]
    table = [[pages.pop() for _ in range(-(-m // p))] for m in seq]
    table = [t + [-1] * (width - len(t)) for t in table]
    ring = [-1] * n
    for i, q in enumerate(pages):
        ring[(n - 5 + i) % n] = q
    from_ = [rng.choice([b, rng.randrange(min(B, 7)), -1]) for b in range(B)]
    check(ac, table, seq, from_, ring, n - 5, len(pages), 1, p, D, dt, in_place)


def test_one_row_or_page_more_than_a_workgroup_and_a_word(ac):  # noqa: F811
    for B, spare in ((1023, 0), (1024, 31), (1025, 1), (2049, 33)):
        rng = random.Random(B)
        table, seq, ring, first, count = cache(rng, B, 4, 9, share=0.7, spare=spare)
        count = min(count, B // 4)
        from_ = [rng.randrange(B) if rng.random() < 0.8 else -1 for _ in range(B)]
        check(ac, table, seq, from_, ring, first, count, 1, 4, 4, "f32", B % 2 == 0)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("sinks,window", [(0, 1), (4, 30), (5, 30), (16, 64), (100, 7), (0, 2 ** 31 - 1), (2 ** 31 - 1, 1)])
def test_pages_that_a_window_leaves_behind(ac, sinks, window, in_place):  # noqa: F811
    rng = random.Random(window)
    table, seq, ring, first, count = cache(rng, 20, 8, 200)
    same = list(range(20))
    got = check(ac, table, seq, same, ring, first, count, 1, 8, 4, "f32", in_place, sinks=sinks, window=window)
    # again, from the result, with entries that are gone
    from_ = [rng.randrange(20) for _ in range(20)]
    if in_place:
        check(ac, got[0], got[1], from_, got[2], *got[3], 1, 8, 4, "f32", in_place, sinks=sinks, window=max(1, window // 2))


@pytest.mark.parametrize("in_place", [False, True])
def test_rows_and_pages_out_of_range(ac, in_place):  # noqa: F811
    """Sources outside the batch end a row, pages outside the cache are nobody's, lengths are clamped."""
    p, n = 4, 40
    table = [[0, 40, 2, 3], [4, -5, 2 ** 31 - 1, -1], [8, 9, 10, 11], [-1] * 4]
    ring = list(range(12, 32)) + [-1] * 20
    for from_, seq in (([1, 0, 2, 2], [14, 10, 99, -3]), ([7, -9, 2 ** 31 - 1, -2 ** 31], [16, 10, 13, 5]), ([3, 3, 3, 3], [16, 10, 13, 0])):
        n_rows = fork(table, seq, from_, ring, 0, 20, p, n, 0, 0)
        if any(not (0 <= a < n and 0 <= b < n) for a, b, _ in n_rows[4]):
            # the page in which a row ends is not there: nothing is copied
            t = call(ac, table, seq, from_, ring, [0, 20], *(torch.zeros(n, 1, p, 4, device="cuda") for _ in range(2)), in_place)
            assert t[1:] == (n_rows[1], n_rows[2], n_rows[3])
        else:
            check(ac, table, seq, from_, ring, 0, 20, 1, p, 4, "f32", in_place)


@pytest.mark.parametrize("state,n", [([-3, 5], 9), ([100, 4], 9), ([4, 99], 9), ([2, -1], 9)])
def test_a_ring_with_odd_numbers(ac, state, n):  # noqa: F811
    """First entry modulo the ring, number within it."""
    ring = [(5 + i) % n for i in range(n)]
    table, seq = [[0, 1], [2, 3]], [3, 4]
    first, count = state[0] % n, min(max(state[1], 0), n)
    k, v = (torch.randn(n, 1, 2, 4, device="cuda") for _ in range(2))
    rows, lens, ring_, st, _ = fork(table, seq, [0, 0], ring, first, count, 2, n, 0, 0)
    got = call(ac, table, seq, [0, 0], ring, state, k, v, False)
    assert got[1:] == (lens, ring_, [st[0], min(st[1], n)])


def test_beams_step_by_step_in_a_graph(ac):  # noqa: F811
    """Plan, fork, plan, ... of beams: replayed in place, each step compared with the one kept by hand."""
    B, p, n, width, H, D = 6, 4, 200, 20, 2, 8
    rng = random.Random(3)
    table, seq, ring, state = torch.full((B, width), -1, dtype=torch.int32, device="cuda"), i32([0] * B), i32(list(range(n))), i32([0, n])
    k, v = (torch.randn(n, H, p, D, device="cuda") for _ in range(2))
    from_, new, added, slot = i32([0] * B), i32([1] * B), i32([0] * B), torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    rows_k = torch.randn(B, H, 1, D, device="cuda")
    ws = torch.empty(ac.attncache_page_fork_workspace_bytes(B, width, n), dtype=torch.uint8, device="cuda")

    def step():
        ac.attncache_page_plan(seq, new, state, ring, table, seq, added, state, slot, page_size=p)
        ac.attncache_page_append(rows_k, rows_k, slot, k, v)
        ac.attncache_page_fork(from_, seq, state, ring, table, table, seq, state, k, v, ws)

    from_.copy_(i32(list(range(B))))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    held = [[rows_k[b].clone()] for b in range(B)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(25):
        order = [rng.randrange(B) for _ in range(B)]
        from_.copy_(i32(order))
        rows_k.copy_(torch.randn(B, H, 1, D, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        held = [held[b] + [rows_k[b].clone()] for b in range(B)]
        held = [list(held[b]) for b in order]
        assert seq.tolist() == [len(x) for x in held]
        t = table.tolist()
        for b, rows in enumerate(held):
            for j, row in enumerate(rows):
                assert torch.equal(k[t[b][j // p], :, j % p], row[:, 0]) and torch.equal(v[t[b][j // p], :, j % p], row[:, 0])
        used = {q for b in range(B) for q in t[b][:-(-seq[b].item() // p)]}
        first, count = state.tolist()
        free = [ring[(first + x) % n].item() for x in range(count)]
        assert len(set(free)) == count == n - len(used) and not used & set(free)
