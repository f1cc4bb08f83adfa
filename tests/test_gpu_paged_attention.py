"""Attention of one new token over pages, against plain attention in 64 bits.  What no request's token lies in is NaN: unused
pages, places behind a request's last token, the workspace."""
import pytest
import torch

from tests import generation as gen
from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Cache:
    """Requests of the given lengths in a cache of shuffled pages; ``more``: elements between pages."""

    def __init__(self, lens, Hkv, D, dt, page, seed, more=0, spare=3, width=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        held = [-(-n // page) for n in lens]
        n = sum(held) + spare
        size = Hkv * page * D + more
        self.k, self.v = (torch.full((n, size), float("nan"), device="cuda", dtype=DT[dt]).as_strided(
            (n, Hkv, page, D), (size, page * D, D, 1)) for _ in range(2))
        order = torch.randperm(n, generator=torch.Generator().manual_seed(seed)).tolist()
        width = max(max(held), 1) if width is None else width
        self.table = torch.full((len(lens), width), -1, dtype=torch.int32)
        self.rows = []
        for b, (m, q) in enumerate(zip(lens, held)):
            mine = [order.pop() for _ in range(q)]
            self.table[b, :q] = torch.tensor(mine, dtype=torch.int32)
            kv = [torch.randn(Hkv, m, D, generator=g, device="cuda").to(DT[dt]) for _ in range(2)]
            self.rows.append(kv)
            for j, p in enumerate(mine):
                c = min(page, m - j * page)
                for to, rows in zip((self.k, self.v), kv):
                    to[p, :, :c] = rows[:, j * page:j * page + c]
        self.table = self.table.cuda()
        self.len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.gen = g

    def call(self, ac, Q, **kw):  # noqa: F811
        B, Hq, D = Q.shape
        room = torch.full((B + 1, Hq, D), 7.0, dtype=Q.dtype, device="cuda")
        ws = torch.full((ac.attention_paged_workspace_bytes(B, Hq, self.k.shape[1], D) // 4,), float("nan"), device="cuda")
        ac.attention_paged(Q, self.k, self.v, self.table, self.len, room[:B], ws, **kw)
        assert (room[B] == 7.0).all()
        return room[:B]

    def check(self, O, Q, some=None, scale=None):
        g = Q.shape[1] // self.k.shape[1]
        for b in range(Q.shape[0]) if some is None else some:
            for h, (k, v) in enumerate(zip(*self.rows[b])):
                rows = slice(h * g, (h + 1) * g)
                gen.check(O[b, rows], *gen.attend(Q[b, rows], k, v, scale))


def _case(ac, lens, Hq, Hkv, D, dt, page, **kw):  # noqa: F811
    c = Cache(lens, Hkv, D, dt, page, sum(lens) + D, **kw)
    Q = torch.randn(len(lens), Hq, D, generator=c.gen, device="cuda").to(DT[dt])
    O = c.call(ac, Q)
    some = None if len(lens) <= 40 else sorted({0, 1, 2, len(lens) // 2, len(lens) - 2, len(lens) - 1})
    c.check(O, Q, some)
    return c, Q, O


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 0, 127, 128, 129, 300]


PAGES = [1, 7, 16, 32, 48, 128]
TYPES = [(64, "bf16"), (128, "bf16"), (64, "f32"), (128, "f32"), (1, "f32"), (33, "f32"), (80, "f32"), (199, "f32"), (256, "f32")]
HEADS = [(1, 1), (5, 1), (12, 12), (32, 8), (16, 1), (17, 1), (33, 1), (40, 2), (64, 1)]
RAGGED = [[1], [5000], [70001], [3] * 300, [40] * 700 + [9000], [9000] + [0] * 200, [0] * 130 + [77],
          [100, 20000, 5, 5, 5, 17, 3000], [513] * 64]
RAGGED_TYPES = [(4, 1, 128, "bf16"), (8, 8, 64, "bf16"), (3, 3, 128, "f32")]
# tables of many pages: runs of blocks over all requests.  Rows of several blocks of 16, odd dimensions, lengths of zero between others,
# more requests than lanes
RUNS = [([70, 0, 4000, 31, 0, 0, 1, 2500], 40, 2, 64, "bf16", 16), ([3001, 64, 65], 17, 1, 128, "bf16", 7),
        ([2100] * 9 + [0] * 70 + [33] * 60 + [5000], 24, 8, 128, "bf16", 48), ([40] * 701 + [9000], 8, 8, 128, "bf16", 16),
        ([9000, 1] * 40, 2, 2, 64, "bf16", 128), ([2049], 64, 1, 64, "bf16", 1), ([1500, 0, 40, 1100], 6, 2, 80, "f32", 10),
        ([1030, 16, 17, 0, 2000], 20, 1, 33, "f32", 16), ([1200] * 30 + [5] * 90, 2, 1, 199, "f32", 7), ([1025, 3], 33, 1, 256, "f32", 32),
        ([30] * 200 + [1700] * 3, 4, 4, 64, "f32", 16), ([2000, 70], 3, 3, 3, "f32", 5),
        ([1030] + [3] * 350, 4, 2, 64, "f32", 16), ([1030] + [3] * 350, 4, 2, 256, "f32", 16), ([1030] + [3] * 100, 4, 2, 256, "f32", 16), ([8000, 1, 700], 12, 4, 128, "f32", 64)]


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("D,dt", TYPES)
def test_lengths_around_blocks_and_pages(ac, page, D, dt):  # noqa: F811
    _case(ac, EDGES, 6, 2, D, dt, page)


@pytest.mark.parametrize("D,dt", TYPES)
def test_many_short_requests(ac, D, dt):  # noqa: F811
    _case(ac, EDGES * 5, 6, 2, D, dt, 16)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_head_layouts(ac, Hq, Hkv, dt):  # noqa: F811
    _case(ac, [70, 1, 600, 33], Hq, Hkv, 64, dt, 16)


@pytest.mark.parametrize("lens", RAGGED, ids=lambda x: f"{len(x)}x{max(x)}")
@pytest.mark.parametrize("Hq,Hkv,D,dt", RAGGED_TYPES)
def test_ragged_batches(ac, lens, Hq, Hkv, D, dt):  # noqa: F811
    _case(ac, lens, Hq, Hkv, D, dt, 16)


@pytest.mark.parametrize("case", RUNS, ids=lambda c: f"{len(c[0])}x{max(c[0])}-" + "-".join(map(str, c[1:])))
def test_runs_over_many_units(ac, case):  # noqa: F811
    lens, Hq, Hkv, D, dt, page = case
    c, Q, O = _case(ac, lens, Hq, Hkv, D, dt, page)
    # every row: a few at a time against one product in 64 bits, or that nothing was left as it was
    assert O.isfinite().all() and (O != 7.0).any(-1).all()
    assert (O[c.len == 0] == 0).all()


@pytest.mark.parametrize("seed", range(16))
def test_drawn_batches(ac, seed):  # noqa: F811
    import random
    rng = random.Random(seed)
    Hkv = rng.choice([1, 2, 3, 8])
    Hq = Hkv * rng.choice([1, 2, 4, 5, 19])
    D, dt = rng.choice([(64, "bf16"), (128, "bf16"), (64, "f32"), (100, "f32")])
    top = rng.choice([40, 600, 2500, 6000])
    lens = [rng.choice([0, 1, top, rng.randint(0, top), rng.randint(0, 70)]) for _ in range(rng.choice([1, 3, 20, 150]))]
    c = Cache(lens, Hkv, D, dt, rng.choice([1, 5, 16, 64]), seed, width=rng.choice([None, 6000]))
    Q = torch.randn(len(lens), Hq, D, generator=c.gen, device="cuda").to(DT[dt])
    O = c.call(ac, Q)
    assert O.isfinite().all() and (O[c.len == 0] == 0).all()
    c.check(O, Q)


@pytest.mark.parametrize("Hq,D", [(1, 64), (4, 128), (16, 64)])
def test_each_row_of_many_short_requests_and_a_long_one(ac, Hq, D):  # noqa: F811
    """All requests alike but one: each result is compared."""
    c = Cache([40] * 640 + [9000] + [64] * 60, 1, D, "bf16", 16, Hq)
    Q = torch.randn(701, Hq, D, generator=c.gen, device="cuda").bfloat16()
    c.check(c.call(ac, Q), Q)


def test_nothing_to_attend_to(ac):  # noqa: F811
    for dt in ("bf16", "f32"):
        _, _, O = _case(ac, [0, 0, 0], 4, 2, 64, dt, 16)
        assert (O == 0).all()


@pytest.mark.parametrize("dt,more", [("bf16", 64), ("f32", 4)])
def test_pages_that_lie_apart(ac, dt, more):  # noqa: F811
    _case(ac, EDGES, 4, 2, 128, dt, 16, more=more, width=40)


def test_requests_that_share_pages_and_empty_batches(ac):  # noqa: F811
    c = Cache([100, 100, 37, 100], 2, 64, "bf16", 16, 3)
    c.table[1], c.rows[1] = c.table[0], c.rows[0]
    c.table[3] = c.table[0]
    c.table[3, :2], c.rows[3] = c.table[2, :2], [torch.cat([a[:, :32], b[:, 32:]], 1) for a, b in zip(c.rows[2], c.rows[0])]
    Q = torch.randn(4, 4, 64, generator=c.gen, device="cuda").bfloat16()
    c.check(c.call(ac, Q), Q)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    ws, none = torch.empty(ac.attention_paged_workspace_bytes(1, 4, 2, 64), dtype=torch.uint8, device="cuda"), Q[:0]
    kv = torch.empty(0, 2, 3, 64, dtype=torch.bfloat16, device="cuda")
    ac.attention_paged(none, c.k, c.v, i32(0, 3), i32(0), none.clone(), ws)
    ac.attncache_page_append(kv, kv, i32(0, 3), c.k, c.v)
    ac.attncache_page_plan(i32(0), i32(0), i32(2), i32(5), i32(0, 3), i32(0), i32(0), i32(2), i32(0, 1), page_size=16)
    ac.attention_cross(none.view(0, 4, 1, 64), kv, kv, none.clone().view(0, 4, 1, 64))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_keys_whose_page_is_out_of_range_are_hidden(ac, dt):  # noqa: F811
    page = 12
    c = Cache([100, 50, 12], 2, 64, dt, page, 5)
    for b, j, p in ((0, 3, c.k.shape[0]), (0, 8, -1), (1, 0, 2**31 - 1), (2, 0, -2**31)):
        c.table[b, j] = p
    for b, gone in enumerate(([3, 8], [0], [0])):
        at = torch.arange(c.rows[b][0].shape[1], device="cuda") // page
        keep = ~torch.isin(at, torch.tensor(gone, device="cuda"))
        c.rows[b] = [r[:, keep] for r in c.rows[b]]
    Q = torch.randn(3, 4, 64, generator=c.gen, device="cuda").to(DT[dt])
    c.check(c.call(ac, Q), Q)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_lengths_are_clamped_to_the_table(ac, dt):  # noqa: F811
    c, Q, O = _case(ac, [64, 20, 0], 4, 2, 64, dt, 16, width=4)
    c.len = torch.tensor([5000, 20, -9], dtype=torch.int32, device="cuda")
    assert torch.equal(c.call(ac, Q), O)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_scale_and_large_scores(ac, dt):  # noqa: F811
    c = Cache([90, 700, 33], 2, 128, dt, 16, 8)
    Q = (30 * torch.randn(3, 6, 128, generator=c.gen, device="cuda")).to(DT[dt])
    c.check(c.call(ac, Q, scale=0.3), Q, scale=0.3)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_infinite_and_lowest_scores(ac, dt):  # noqa: F811
    """Keys of -inf and of the type's lowest value weigh nothing next to others; a NaN among the keys makes the row NaN."""
    c = Cache([200, 40, 5], 1, 64, dt, 16, 9)
    Q = torch.randn(3, 2, 64, generator=c.gen, device="cuda").abs().to(DT[dt])
    low = torch.finfo(DT[dt]).min
    for b, j, x in ((0, 3, -float("inf")), (0, 150, low), (1, 0, -float("inf")), (2, 1, float("nan"))):
        c.k[c.table[b, j // 16].item(), :, j % 16] = x
        c.rows[b][0][:, j] = x
    O = c.call(ac, Q)
    assert O[2].isnan().all()
    for b, gone in ((0, [3, 150]), (1, [0])):
        keep = [j for j in range(c.rows[b][0].shape[1]) if j not in gone]
        c.rows[b] = [r[:, keep] for r in c.rows[b]]
    c.check(O, Q, [0, 1])


def test_pages_behind_two_gibi_elements(ac):  # noqa: F811
    n, Hkv, page, D, m = 40_000, 4, 128, 128, 1000
    k, v = (torch.empty(n, Hkv, page, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    mine = [39_999, 0, 33_333, 12, 20_000, 39_000, 7, 38_000]
    g = torch.Generator(device="cuda").manual_seed(4)
    rows = [torch.randn(Hkv, m, D, generator=g, device="cuda").bfloat16() for _ in range(2)]
    for j, p in enumerate(mine):
        c = min(page, m - j * page)
        k[p, :, :c], v[p, :, :c] = (r[:, j * page:j * page + c] for r in rows)
    Q = torch.randn(1, 8, D, generator=g, device="cuda").bfloat16()
    O, ws = torch.empty_like(Q), torch.empty(ac.attention_paged_workspace_bytes(1, 8, Hkv, D), dtype=torch.uint8, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    ac.attention_paged(Q, k, v, i32([mine]), i32([m]), O, ws)
    for h in range(Hkv):
        gen.check(O[0, 2 * h:2 * h + 2], *gen.attend(Q[0, 2 * h:2 * h + 2], rows[0][h], rows[1][h]))


def test_the_same_result_every_time_on_any_stream(ac):  # noqa: F811
    c, Q, O = _case(ac, [40, 3000, 700, 0, 64], 8, 2, 128, "bf16", 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            assert torch.equal(c.call(ac, Q), O)
        assert torch.equal(c.call(ac, Q, stream=torch.cuda.current_stream()), O)


def test_two_graphs_with_one_workspace(ac):  # noqa: F811
    calls, sizes = [], (([900, 3, 2000], 8, 2, 128), ([17] * 40 + [4000], 4, 4, 64))
    ws = torch.full((max(ac.attention_paged_workspace_bytes(len(x), *s) for x, *s in sizes) // 4,), float("nan"), device="cuda")
    for lens, Hq, Hkv, D in sizes:
        c = Cache(lens, Hkv, D, "bf16", 16, D)
        Q = torch.randn(len(lens), Hq, D, generator=c.gen, device="cuda").bfloat16()
        O = torch.zeros_like(Q)
        go = lambda c=c, Q=Q, O=O: ac.attention_paged(Q, c.k, c.v, c.table, c.len, O, ws)  # noqa: E731
        go()
        want = O.clone()
        c.check(want, Q, [0, len(lens) - 1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            go()
        calls.append((graph, go, O, want))
    for i in range(8):
        for graph, go, O, want in calls:
            O.fill_(7.0)
            go() if i % 3 == 2 else graph.replay()
            assert torch.equal(O, want)


@pytest.mark.parametrize("dt,page,D", [("bf16", 16, 64), ("bf16", 12, 128), ("f32", 5, 100)])
def test_prompts_and_generated_tokens_together(ac, dt, page, D):  # noqa: F811
    """A prefill by exact attention, its K and V into pages, then tokens one by one: plan, append, attention, as a captured step
    that goes on by itself.  Every result is that of exact attention over the whole sequence at its place."""
    B, Hq, Hkv, S, steps = 3, 4, 2, 32, 40
    lens = [32, 20, 1]
    g = torch.Generator(device="cuda").manual_seed(D)
    n_all = S + steps
    q, k, v = (torch.randn(B, h, n_all, D, generator=g, device="cuda").to(DT[dt]) for h in (Hq, Hkv, Hkv))
    n, width = 3 * -(-n_all // page) + 1, -(-n_all // page)
    i32 = lambda *s, x=0: torch.full(s, x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, ring, state = i32(B, width, x=-1), torch.randperm(n).int().cuda(), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    seq, added, slot, new = i32(B), i32(B), i32(B, S), torch.tensor(lens, dtype=torch.int32, device="cuda")
    kp, vp = (torch.full((n, Hkv, page, D), float("nan"), dtype=DT[dt], device="cuda") for _ in range(2))
    Q0, K0, V0 = (t[:, :, :S].contiguous() for t in (q, k, v))
    O0 = torch.empty_like(Q0)
    ac.attention_exact(Q0, K0, V0, O0, key_len=new)
    ac.attncache_page_plan(seq, new, state, ring, table, seq, added, state, slot, page_size=page)
    ac.attncache_page_append(K0, V0, slot, kp, vp)
    assert added.tolist() == lens and seq.tolist() == lens
    one = i32(B, x=1)
    slot1 = i32(B, 1)
    qs, ks, vs = (torch.empty(B, h, 1, D, dtype=DT[dt], device="cuda") for h in (Hq, Hkv, Hkv))
    O, ws = torch.empty(B, Hq, D, dtype=DT[dt], device="cuda"), torch.empty(
        ac.attention_paged_workspace_bytes(B, Hq, Hkv, D), dtype=torch.uint8, device="cuda")

    def step():
        ac.attncache_page_plan(seq, one, state, ring, table, seq, added, state, slot1, page_size=page)
        ac.attncache_page_append(ks, vs, slot1, kp, vp)
        ac.attention_paged(qs.view(B, Hq, D), kp, vp, table, seq, O, ws)
    at = list(lens)

    def feed():
        for b, p in enumerate(at):
            for to, src in ((qs, q), (ks, k), (vs, v)):
                to[b, :, 0] = src[b, :, p]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(steps):
        feed()
        step() if i % 7 == 3 else graph.replay()
        for b in range(B):
            at[b] += 1
            for h in range(Hq):
                kk, vv = k[b, h // 2, :at[b]], v[b, h // 2, :at[b]]
                gen.check(O[b, h:h + 1], *gen.attend(q[b, h, at[b] - 1][None], kk, vv))
        assert seq.tolist() == at
