"""Attention of one new token within a window over pages, against plain attention in 64 bits.  What no token that is seen lies in is
NaN, and pages in the gap are not even named."""
import pytest
import torch

from tests import generation as gen
from tests.test_gpu_paged_attention import DT, EDGES, HEADS, TYPES, Cache
from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu


def visible(n, window, sinks):
    return [j for j in range(n) if j >= n - window or j < sinks]


def case(ac, lens, Hq, Hkv, D, dt, page, window, sinks, some=None, **kw):  # noqa: F811
    c = Cache(lens, Hkv, D, dt, page, sum(lens) + D, **kw)
    wild = [-1, -2 ** 31, 2 ** 31 - 1, c.k.shape[0]]
    for b, n in enumerate(lens):
        at = visible(n, window, sinks)
        alive = {j // page for j in at}
        for j in range(-(-n // page)):
            q = int(c.table[b, j])
            gone = [t for t in range(j * page, min(n, (j + 1) * page)) if not (t >= n - window or t < sinks)]
            if gone:
                c.k[q, :, gone[0] % page:gone[-1] % page + 1] = c.v[q, :, gone[0] % page:gone[-1] % page + 1] = float("nan")
            if j not in alive:
                c.table[b, j] = wild[j % 4]
        c.rows[b] = [r[:, at] for r in c.rows[b]]
    B = len(lens)
    Q = torch.randn(B, Hq, D, generator=c.gen, device="cuda").to(DT[dt])
    room = torch.full((B + 1, Hq, D), 7.0, dtype=Q.dtype, device="cuda")
    ws = torch.full((ac.attention_paged_workspace_bytes(B, Hq, Hkv, D) // 4,), float("nan"), device="cuda")
    ac.attention_paged_window(Q, c.k, c.v, c.table, c.len, room[:B], ws, window=window, sinks=sinks)
    assert (room[B] == 7.0).all() and room[:B].isfinite().all()
    c.check(room[:B], Q, some if some is not None or B <= 40 else sorted({0, 1, 2, B // 2, B - 2, B - 1}))
    return c, Q, room[:B]


WINDOWS = [(1, 0), (1, 1), (5, 3), (31, 1), (32, 32), (64, 4), (100, 20), (4096, 4), (2 ** 31 - 1, 2 ** 31 - 1), (16, 2 ** 31 - 1)]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("page", [1, 7, 16, 128])
def test_windows_and_pages(ac, page, window, sinks):  # noqa: F811
    for D, dt in ((64, "bf16"), (128, "f32")):
        case(ac, EDGES, 6, 2, D, dt, page, window, sinks)


@pytest.mark.parametrize("D,dt", TYPES)
def test_types(ac, D, dt):  # noqa: F811
    case(ac, EDGES, 6, 2, D, dt, 16, 50, 9)
    case(ac, [2500, 3, 1300, 0, 1100], 6, 2, D, dt, 16, 1000, 9)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_head_layouts(ac, Hq, Hkv, dt):  # noqa: F811
    case(ac, [70, 1, 600, 33], Hq, Hkv, 64, dt, 16, 40, 5)


# lengths, heads, head dimension, type, page, window, sinks: units in one launch, and runs and joins with one, four and eight waves a row
RUNS = [([70, 0, 4000, 31, 0, 0, 1, 5500], 40, 2, 64, "bf16", 16, 3000, 40), ([9000, 1] * 40, 2, 2, 64, "bf16", 128, 4000, 16),
        ([2100] * 9 + [0] * 70 + [33] * 60 + [9000], 24, 8, 128, "bf16", 48, 5000, 1), ([5000] * 64, 8, 8, 128, "bf16", 16, 2500, 4),
        ([30] * 200 + [2700] * 3, 4, 4, 64, "f32", 16, 1500, 17), ([1030] + [3] * 350, 4, 2, 256, "f32", 16, 900, 4),
        ([1200] * 30 + [5] * 90, 2, 1, 199, "f32", 7, 900, 0), ([20000], 33, 1, 128, "bf16", 32, 7000, 100), ([1500, 0, 40, 3100], 6, 2, 80, "f32", 10, 1100, 3),
        ([4000] * 300, 4, 4, 64, "bf16", 16, 100, 4), ([7000] * 100, 12, 4, 128, "f32", 16, 300, 4), ([2100, 70], 6, 2, 33, "f32", 5, 1100, 60),
        ([3000] * 20, 2, 2, 64, "f32", 16, 1200, 4), ([3000] * 30, 4, 4, 128, "f32", 16, 1200, 4), ([3000] * 300, 2, 2, 80, "f32", 16, 1200, 4),
        ([1500] * 300, 2, 2, 40, "f32", 16, 1200, 4), ([1500] * 150, 2, 2, 40, "f32", 16, 1200, 4), ([1500, 9] * 20, 2, 2, 40, "f32", 16, 1200, 4),
        ([1500] * 150, 2, 2, 199, "f32", 16, 1200, 4), ([1500, 2] * 9, 2, 2, 199, "f32", 16, 1200, 4), ([3000] * 3, 64, 2, 128, "f32", 16, 1200, 4),
        ([4000] * 20, 4, 4, 64, "bf16", 16, 3000, 4), ([4000] * 9, 8, 8, 128, "bf16", 16, 3000, 4), ([4000] * 90, 16, 2, 128, "bf16", 16, 3000, 4)]
RUNS += [([40] * 600 + [5000], 2, 1, 64, "bf16", 16, 3000, 4)] + [([40] * 600 + [3000], 2, 1, D, "f32", 16, 1500, 4) for D in (64, 33, 80, 199)]
RUNS += [([100] * 150, 2, 2, D, dt, 16, 50, 4) for D, dt in ((128, "bf16"), (64, "f32"), (40, "f32"), (80, "f32"))]


@pytest.mark.parametrize("c", RUNS, ids=lambda c: f"{len(c[0])}x{max(c[0])}-" + "-".join(map(str, c[1:])))
def test_runs_over_many_units(ac, c):  # noqa: F811
    case(ac, *c)


def test_a_window_over_everything_is_attention_over_pages(ac):  # noqa: F811
    c, Q, O = case(ac, [100, 2000, 1, 0], 4, 2, 64, "bf16", 16, 5000, 0)
    E = c.call(ac, Q)
    assert torch.equal(O, E)


def test_a_captured_step_goes_on_by_itself(ac):  # noqa: F811
    """Plan, append, attention in a window, pages behind it given back: replayed in place."""
    B, H, D, p, n, width, window, sinks = 3, 2, 64, 4, 40, 30, 17, 5
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, seq, ring, state = torch.full((B, width), -1, dtype=torch.int32, device="cuda"), i32([0] * B), i32(list(range(n))), i32([0, n])
    k, v = (torch.full((n, H, p, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    new, added, slot, same = i32([1] * B), i32([0] * B), i32([[0]] * B), i32(list(range(B)))
    K, V, Q, O = (torch.randn(B, H, 1, D, device="cuda").bfloat16() for _ in range(4))
    ws = torch.empty(max(ac.attncache_page_fork_workspace_bytes(B, width, n), ac.attention_paged_workspace_bytes(B, H, H, D)),
                     dtype=torch.uint8, device="cuda")

    def step():
        ac.attncache_page_plan(seq, new, state, ring, table, seq, added, state, slot, page_size=p)
        ac.attncache_page_append(K, V, slot, k, v)
        ac.attention_paged_window(Q[:, :, 0].contiguous(), k, v, table, seq, O.view(B, H, D), ws, window=window, sinks=sinks)
        ac.attncache_page_fork(same, seq, state, ring, table, table, seq, state, k, v, ws, window=window, sinks=sinks)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    past = [(K.clone(), V.clone())]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(100):
        for t in (K, V, Q):
            t.copy_(torch.randn(B, H, 1, D, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        past.append((K.clone(), V.clone()))
        assert seq.tolist() == [len(past)] * B
        at = visible(len(past), window, sinks)
        for b in range(B):
            for h in range(H):
                kk, vv = (torch.stack([past[j][x][b, h, 0] for j in at]) for x in (0, 1))
                gen.check(O[b, h], *gen.attend(Q[b, h], kk, vv))
        held = sum(len({j // p for j in range(len(past)) if j >= (len(past) - window) // p * p or j < -(-sinks // p) * p}) for _ in range(B))
        assert n - state[1].item() == held


LENS, SOME = [300, 0, 1, 19, 20, 21, 24, 25, 26, 33] * 7, [0, 1, 2, 3, 5, 7, 11, 36, 60, 69]      # (of 70: more than 1,024 units of 16 heads)


@pytest.mark.parametrize("D,dt", TYPES)
def test_many_requests_with_short_windows(ac, D, dt):  # noqa: F811
    case(ac, LENS, 32, 16, D, dt, 16, 20, 5, SOME)
    case(ac, LENS, 20, 1, D, dt, 7, 30, 0, SOME)
    case(ac, LENS[:35] * 16, 4, 2, D, dt, 16, 1, 1, SOME)
    case(ac, LENS, 8, 4, D, dt, 16, 200, 5, SOME)      # (fewer and larger units)


@pytest.mark.parametrize("D", [1, 2, 3, 4, 5, 15, 17, 33, 36, 65, 100, 101, 127, 129, 199, 200, 255])
def test_infinities_in_single_columns(ac, D):  # noqa: F811
    """Binary32 rows of any length: a key of which one column is -inf weighs nothing, a value of which one is infinite fills that column and no other."""
    lens, cols = [60, 3000], sorted({0, max(D - 18, 0), *range(max(D - 5, 0), D)})
    c = Cache(lens, 2, D, "f32", 16, D)
    Q = torch.randn(2, 6, D, generator=c.gen, device="cuda").abs() + 0.1
    for b, n in enumerate(lens):
        for j, col in enumerate(cols):
            if 17 * j < n:
                c.k[c.table[b, j], :, j, col] = -float("inf")       # key 17 j
        c.v[c.table[b, 1], :, 2, D - 1] = float("inf")
    keep = [[j for j in range(n) if j % 17 or j >= 17 * len(cols)] for n in lens]
    ws = torch.empty(ac.attention_paged_workspace_bytes(2, 6, 2, D), dtype=torch.uint8, device="cuda")
    O = [torch.empty_like(Q) for _ in range(2)]
    ac.attention_paged(Q, c.k, c.v, c.table, c.len, O[0], ws)
    ac.attention_paged_window(Q, c.k, c.v, c.table, c.len, O[1], ws, window=4000)
    for b in range(2):
        c.rows[b] = [r[:, keep[b]] for r in c.rows[b]]
    for o in O:
        assert (o[:, :, D - 1] == float("inf")).all()
        for b in range(2):
            for h in range(2):
                want, terms, bound = gen.attend(Q[b, 3 * h:3 * h + 3], c.rows[b][0][h], c.rows[b][1][h])
                if D > 1:
                    gen.check(o[b, 3 * h:3 * h + 3, :D - 1], want[:, :D - 1], terms[:, :D - 1], bound)
