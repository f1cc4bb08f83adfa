"""Attention of a batch whose requests share prefixes, against plain attention in 64 bits.  What no request's token lies in is NaN:
unused pages, places behind a request's last token, the workspace, and other rows' pages of a prefix that is read through the first."""
import random

import pytest
import torch

from tests.test_gpu_paged_attention import DT, TYPES, Cache
from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu


def width(B, Hkv, D, dt, page):
    """Entries of a row from which on it has room for more than 128 tokens, and K and V of all rows' are more than 64 MiB: prefixes are then read once."""
    return max(2 ** 26 // (B * Hkv * D * (4 if dt == "bf16" else 8)), 128) // page + 1


def build(groups, alone, Hkv, D, dt, page, seed=0, more=0, blank=True, wide=True):
    """groups: (prefix, [tokens behind it, or None: a request of half the prefix]); alone: lengths of requests at the end.  wide: rows of the
    table are at least as long as that a prefix is read once; entries behind the tokens' are no pages."""
    lens = [p // 2 if n is None else p + n for p, rows in groups for n in rows] + list(alone)
    c = Cache(lens, Hkv, D, dt, page, seed + sum(lens), more=more)
    first, share = [0], []
    for p, rows in groups:
        f = first[-1]
        have = [b for b, n in zip(range(f, f + len(rows)), rows) if n is not None]
        for b in have[1:]:
            lead = have[0]
            for x in (0, 1):
                c.rows[b][x] = torch.cat([c.rows[lead][x][:, :p], c.rows[b][x][:, p:]], 1)
            full = p // page
            old = c.table[b, :full].clone()
            c.table[b, :full] = c.table[lead, :full]
            if blank and len(old):
                c.k[old.long()] = c.v[old.long()] = float("nan")
            if p % page:        # its own page from here on; the prefix's tokens in it are read through the first request
                q = int(c.table[b, full])
                for to, rows_ in ((c.k, c.rows[b][0]), (c.v, c.rows[b][1])):
                    to[q, :, :p % page] = float("nan") if blank else rows_[:, full * page:p]
        first.append(f + len(rows))
        share.append(p)
    if wide:
        B, n = c.table.shape
        far = torch.full((B, max(width(B, Hkv, D, dt, page) - n, 0)), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
        c.table = torch.cat([c.table, far], 1).contiguous()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return c, i32(first), i32(share)


def call(ac, c, Q, first, share, **kw):  # noqa: F811
    B, Hq, D = Q.shape
    room = torch.full((B + 1, Hq, D), 7.0, dtype=Q.dtype, device="cuda")
    need = ac.attention_paged_shared_workspace_bytes(B, Hq, c.k.shape[1], D, share.numel())
    ws = torch.full((need // 4 + 1,), float("nan"), device="cuda")
    ac.attention_paged_shared(Q, c.k, c.v, c.table, c.len, first, share, room[:B], ws[:-1], **kw)
    assert (room[B] == 7.0).all() and ws[-1].isnan()
    return room[:B]


def case(ac, groups, alone, Hq, Hkv, D, dt, page, some=None, **kw):  # noqa: F811
    c, first, share = build(groups, alone, Hkv, D, dt, page, **kw)
    B = len(c.rows)
    Q = torch.randn(B, Hq, D, generator=c.gen, device="cuda").to(DT[dt])
    O = call(ac, c, Q, first, share)
    assert O.isfinite().all()
    c.check(O, Q, some if some is not None or B <= 70 else sorted(random.Random(B).sample(range(B), 40)))
    return c, Q, O, first, share


EDGES = [(33, [1, 0, 5]), (64, [64, 1]), (1, [0, 0, 31, 33]), (31, [2]), (16, [0, 17, 1, 1, 1]), (65, [100, None, 7]), (128, [0, None, None]),
         (40, [9, 8, 7, 6, 5, 4, 3, 2, 1])]
# groups, requests alone, heads, head dimension, type, page: units of 16 rows, workgroups of 128, one group and many, prefixes cut and whole
CASES = [([(3000, [1] * 64)], [], 32, 8, 128, "bf16", 16), ([(16000, [5, 300] * 32)], [], 8, 2, 64, "bf16", 16),
         ([(500, [20] * 33)] * 3, [40, 0, 9], 4, 4, 128, "bf16", 16), ([(70, [3] * 20)] * 30, [1, 2], 8, 2, 64, "bf16", 7),
         ([(1000, [0, 1, 2]), (2000, [50] * 129), (64, [1] * 40)], [333], 2, 1, 64, "bf16", 48), ([(20000, [10] * 3)], [30000], 8, 1, 128, "bf16", 128),
         ([(640, [7] * 8)] * 40, [], 16, 2, 128, "bf16", 10), ([(9, [1] * 150)], [], 3, 3, 64, "bf16", 1), ([(700, [1] * 5)] * 2, [3], 40, 1, 64, "bf16", 16),
         ([(1500, [3, 900])] * 6, [20] * 9, 6, 2, 80, "f32", 10), ([(2000, [1] * 40)], [5], 4, 2, 128, "f32", 16), ([(300, [2] * 17)] * 5, [], 3, 1, 199, "f32", 7),
         ([(1030, [9] * 3)] * 3, [], 33, 1, 256, "f32", 32), ([(100, [1] * 4)] * 50, [7] * 30, 2, 2, 33, "f32", 16), ([(5000, [1, 2])], [], 4, 4, 64, "f32", 16),
         ([(2000, [30] * 600)], [], 8, 8, 64, "bf16", 16), ([(512, [64] * 4)] * 300, [], 4, 1, 128, "bf16", 16),
         ([(100, [1, 2, 3])], [], 4, 1, 64, "bf16", 16), ([(3000, [1, 200])], [77], 10, 2, 128, "bf16", 16)]


# more than 256 requests: the list is made before; few rows of a group, and many
MANY = [([(50, [3] * 8)] * 40, [9] * 20, Hq, 1, D, dt, 16) for D, dt in TYPES for Hq in (1, 4)]
MANY += [([(300, [5] * 20)] * 15, [700], 4, 2, D, "bf16", 16) for D in (64, 128)] + [([(40, [1])] * 300 + [(90, [2, 3] * 20)], [], 1, 1, 64, "bf16", 16)]
MANY += [([(40, [1])] * 1100, [], 1, 1, D, dt, 16) for D, dt in ((64, "bf16"), (64, "f32"))]
MANY += [([(40, [1, 2])] * 150, [], 1, 1, 64, "bf16", 16), ([(3000, [2] * 3)] * 3, [5], 32, 1, 128, "bf16", 16)]
# more than 6,144 rows, of few parts and of many
MANY += [([(50, [3] * 8)] * 40, [9, 0] * 10, 20, 1, D, dt, 16) for D, dt in TYPES] + [([(3000, [2] * 199 + [0])], [0, 5], 32, 1, D, dt, 16) for D, dt in TYPES[:3]]
# caches of more than 4 GiB
FAR, FAR_MANY, FAR_HEADS = [(400, [20] * 9), (90, [1, 2])], [(400, [20] * 130), (90, [1, 2] * 70)], [(4, 1, 64), (8, 2, 128)]


@pytest.mark.parametrize("c", MANY, ids=lambda c: f"{len(c[0])}x{c[0][0][0]}x{len(c[0][0][1])}-{len(c[1])}-" + "-".join(map(str, c[2:])))
def test_more_requests_than_a_workgroup_lists(ac, c):  # noqa: F811
    case(ac, *c)


@pytest.mark.parametrize("Hq,Hkv,D", FAR_HEADS)
@pytest.mark.parametrize("groups,stride", [(FAR, 1 << 24), (FAR_MANY, 1 << 20)], ids=["few", "many"])
def test_a_cache_of_more_than_four_gib(ac, groups, stride, Hq, Hkv, D):  # noqa: F811
    """Pages far apart: places beyond 2^32 bytes."""
    c, first, share = build(groups, [3], Hkv, D, "bf16", 16)
    n, at = c.k.shape[0], {}
    for name in "kv":
        old = getattr(c, name)
        at[name] = torch.empty((n - 1) * stride + old[0].numel(), dtype=torch.bfloat16, device="cuda")
        new = at[name].as_strided(old.shape, (stride, *old.stride()[1:]))
        new.copy_(old)
        setattr(c, name, new)
    assert 2 ** 32 < n * stride * 2 < 2 ** 34
    Q = torch.randn(len(c.rows), Hq, D, generator=c.gen, device="cuda").bfloat16()
    c.check(call(ac, c, Q, first, share), Q, sorted(random.Random(1).sample(range(len(c.rows)), 8)))


@pytest.mark.parametrize("page", [1, 7, 16, 48, 128])
@pytest.mark.parametrize("D,dt", TYPES)
def test_edges(ac, page, D, dt):  # noqa: F811
    case(ac, EDGES, [0, 1, 50], 6, 2, D, dt, page)


@pytest.mark.parametrize("c", CASES, ids=lambda c: f"{len(c[0])}x{c[0][0][0]}x{len(c[0][0][1])}-{len(c[1])}-" + "-".join(map(str, c[2:])))
def test_groups(ac, c):  # noqa: F811
    case(ac, *c)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (5, 1), (12, 12), (32, 8), (17, 1), (33, 1), (40, 2)])
def test_head_layouts(ac, Hq, Hkv, dt):  # noqa: F811
    case(ac, [(90, [1, 2, 3] * 4), (300, [40, 1])], [70, 1], Hq, Hkv, 64, dt, 16)


@pytest.mark.parametrize("seed", range(16))
def test_drawn(ac, seed):  # noqa: F811
    rng = random.Random(seed)
    Hkv = rng.choice([1, 2, 3, 8])
    Hq = Hkv * rng.choice([1, 2, 4, 5, 19])
    D, dt = rng.choice([(64, "bf16"), (128, "bf16"), (64, "f32"), (100, "f32")])
    groups = [(rng.randint(1, rng.choice([40, 600, 3000])), [rng.choice([0, 1, rng.randint(0, 300), None]) for _ in range(rng.choice([1, 2, 5, 30]))])
              for _ in range(rng.choice([1, 3, 12]))]
    case(ac, groups, [rng.randint(0, 500) for _ in range(rng.choice([0, 1, 7]))], Hq, Hkv, D, dt, rng.choice([1, 5, 16, 64]), seed=seed)


@pytest.mark.parametrize("dt,more", [("bf16", 64), ("f32", 4)])
def test_pages_that_lie_apart(ac, dt, more):  # noqa: F811
    case(ac, EDGES, [5], 4, 2, 128, dt, 16, more=more)


@pytest.mark.parametrize("D,dt", TYPES)
def test_it_is_attention_over_pages(ac, D, dt):  # noqa: F811
    """Whatever is said to be shared: groups out of order and range, of one or none, prefixes longer than the requests or negative."""
    lens = [100, 90, 200, 90, 5, 0, 300, 100]
    c, first, share = build([(80, [20, 10, 120, 10])], [5, 0, 300, 100], 2, D, dt, 16, blank=False)
    assert c.len.tolist() == lens
    Q = torch.randn(8, 4, D, generator=c.gen, device="cuda").to(DT[dt])
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for first, share in (([0, 4], [80]), ([0, 4], [50]), ([0, 4], [81 - 1]), ([0, 4, 4, 5, 8], [64, 9, 70, 0]), ([0, 8], [2 ** 31 - 1]), ([0, 8], [-7]),
                         ([-5, 4, 2, 4], [80, 80, 3]), ([0, 2, 1, 4], [80, 90, 80]), ([2, 4, 99], [80, 300]), ([8, 8], [80]), ([99, -1], [80]), ([0], []),
                         ([1, 3], [80]), ([0, 4] + [4] * 2000, [80] + [5] * 2000)):
        c.check(call(ac, c, Q, i32(first), i32(share) if share else torch.zeros(0, dtype=torch.int32, device="cuda")), Q)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_keys_whose_page_is_out_of_range_are_hidden(ac, dt):  # noqa: F811
    c, first, share = build([(200, [30] * 40), (70, [9, 60])], [50], 2, 64, dt, 16)
    gone = {b: set() for b in range(43)}
    for b, j, p in ((0, 3, c.k.shape[0]), (0, 13, -1), (40, 1, 2 ** 31 - 1), (41, 6, -9), (42, 0, -2 ** 31)):
        c.table[b, j] = p
        gone[b].add(j)
    for b in range(40):
        gone[b].add(3)       # the prefix is read through request 0
    gone[41].add(1)
    for b, g in gone.items():
        at = torch.arange(c.rows[b][0].shape[1], device="cuda") // 16
        keep = ~torch.isin(at, torch.tensor(sorted(g) or [-1], device="cuda"))
        c.rows[b] = [r[:, keep] for r in c.rows[b]]
    Q = torch.randn(43, 4, 64, generator=c.gen, device="cuda").to(DT[dt])
    c.check(call(ac, c, Q, first, share), Q)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_large_scores_and_a_scale(ac, dt):  # noqa: F811
    c, first, share = build([(700, [30] * 20)], [90], 2, 64, dt, 16)
    Q = (40 * torch.randn(21, 4, 64, generator=c.gen, device="cuda")).to(DT[dt])
    c.check(call(ac, c, Q, first, share, scale=0.2), Q, scale=0.2)


@pytest.mark.parametrize("rows", [3, 40])
def test_every_key_counts_once(ac, rows):  # noqa: F811
    """Q is zero: a result is the mean of V, whose marked column of each block of keys tells which were seen."""
    P, own, D = 5000, 70, 64
    c, first, share = build([(P, [own] * rows)] * 2, [P], 2, D, "bf16", 16)
    B = len(c.rows)
    one = torch.nn.functional.one_hot((torch.arange(P + own, device="cuda") // 32) % D, D).bfloat16()
    for b in range(B):
        n = c.rows[b][1].shape[1]
        for j in range(-(-n // 16)):
            q, m = int(c.table[b, j]), min(16, n - 16 * j)
            c.v[q, :, :m] = one[16 * j:16 * j + m]
    O = call(ac, c, torch.zeros(B, 8, D, dtype=torch.bfloat16, device="cuda"), first, share)
    for b in (0, 1, rows - 1, rows, B - 2, B - 1):
        want = one[:c.rows[b][1].shape[1]].double().mean(0)
        assert ((O[b].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want).all()


def test_many_requests_and_groups(ac):  # noqa: F811
    case(ac, [(40, [3, 1])] * 1500, [9] * 100, 2, 1, 64, "bf16", 16)
    case(ac, [(40, [3])] * 1100 + [(100, [1] * 70)], [9] * 3, 2, 1, 64, "bf16", 16)


def test_a_captured_call_two_streams_and_the_same_result_every_time(ac):  # noqa: F811
    for dt in ("bf16", "f32"):
        c, first, share = build([(900, [30] * 20), (2000, [5, 7])], [90], 2, 64, dt, 16)
        Q = torch.randn(23, 4, 64, generator=c.gen, device="cuda").to(DT[dt])
        want = call(ac, c, Q, first, share).clone()
        need = ac.attention_paged_shared_workspace_bytes(23, 4, 2, 64, 2)
        ws = [torch.zeros(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
        O = [torch.zeros_like(Q) for _ in range(2)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ac.attention_paged_shared(Q, c.k, c.v, c.table, c.len, first, share, O[0], ws[0])
        for _ in range(4):
            O[0].zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(O[0], want)
        s = [torch.cuda.Stream() for _ in range(2)]
        for o in O:
            o.zero_()
        torch.cuda.synchronize()
        for x in range(2):
            ac.attention_paged_shared(Q, c.k, c.v, c.table, c.len, first, share, O[x], ws[x], stream=s[x])
        torch.cuda.synchronize()
        assert torch.equal(O[0], want) and torch.equal(O[1], want)


@pytest.mark.parametrize("c", [(EDGES, [0, 1, 50], 6, 2, D, dt, page) for D, dt in TYPES for page in (7, 16)]
                         + [([(70, [3] * 20)] * 3, [1, 2], 40, 2, 64, "bf16", 7), ([(2000, [1] * 4)], [5], 4, 1, 128, "bf16", 16), ([(300, [2] * 17)], [], 3, 1, 199, "f32", 7)],
                         ids=lambda c: f"{len(c[0])}x{c[0][0][0]}x{len(c[0][0][1])}-{len(c[1])}-" + "-".join(map(str, c[2:])))
def test_little_to_read(ac, c):  # noqa: F811
    """K and V of all rows' tokens are no more than 64 MiB: every request by itself, as with no groups at all."""
    c, Q, O, first, share = case(ac, *c, wide=False, blank=False)
    B, Hkv, D = Q.shape[0], c.k.shape[1], Q.shape[2]
    assert 2 * B * c.table.shape[1] * c.k[0].numel() * Q.element_size() <= 2 ** 26
    assert torch.equal(O, c.call(ac, Q)) and torch.equal(O, call(ac, c, Q, first[:1], share[:0]))


SHORT = ([(20, [3, 0, 7] * 4)] * 100, [1, 0, 30], 4, 1)


@pytest.mark.parametrize("D,dt", TYPES)
def test_many_requests_with_little_to_read(ac, D, dt):  # noqa: F811
    case(ac, *SHORT, D, dt, 16, wide=False, blank=False)
    case(ac, [(50, [0, 2] * 4)], [9] * 22, 48, 48, D, dt, 10, [0, 3, 7, 8, 29], wide=False, blank=False)


def test_an_empty_batch(ac):  # noqa: F811
    c, first, share = build([(20, [1, 2])], [], 2, 64, "bf16", 16)
    none = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    ac.attention_paged_shared(none, c.k, c.v, c.table[:0], c.len[:0], first, share, none.clone(), torch.empty(16, dtype=torch.uint8, device="cuda"))
