"""The operators of generation at sizes near their limits, where index arithmetic of 32 bits comes to its end.  (The arithmetic alone:
test_generation_index.py, without a GPU.)"""
import pytest
import torch

from tests import generation as gen
from tests.test_gpu_paged_attention import Cache
from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,first", [(1_200_000_000, 1_100_000_000), (1_200_000_000, 1_199_999_998), (1_500_000_000, 1_499_999_999)])
def test_a_ring_of_more_than_two_to_the_thirty_pages(ac, n, first, in_place):  # noqa: F811
    """Pages of one token: the ring's entries, its first one and what is given back behind its last one have numbers beyond 2^30."""
    ring, count = torch.empty(n, dtype=torch.int32, device="cuda"), 10
    around = torch.arange(-4, 16, device="cuda") + first
    pages = torch.arange(20, device="cuda").int() * 60_000_000 % n + 5
    ring[around % n] = pages
    seq, new, state, slot = _i32([0, 5, 3]), _i32([2, 1, -1]), _i32([first, count]), torch.full((3, 2), 99, dtype=torch.int32, device="cuda")
    table = _i32([[-1] * 8, [1, 2, 3, 4, 6] + [-1] * 3, [7, 8, n - 1] + [-1] * 5])
    out = (seq, new, state) if in_place else tuple(torch.full_like(t, 77) for t in (seq, new, state))
    ac.attncache_page_plan(seq, new, state, ring, table, *out, slot, page_size=1)
    p = pages.tolist()
    assert out[0].tolist() == [2, 6, 0] and out[1].tolist() == [2, 1, 0]
    assert out[2].tolist() == [(first + 3) % n, count]
    assert slot.tolist() == [[p[4], p[5]], [p[6], -1], [-1, -1]]
    assert table.tolist() == [[p[4], p[5]] + [-1] * 6, [1, 2, 3, 4, 6, p[6], -1, -1], [7, 8, n - 1] + [-1] * 5]
    assert ring[around % n].tolist() == p[:14] + [7, 8, n - 1] + p[17:]


def test_runs_of_more_than_two_to_the_thirty_blocks(ac):  # noqa: F811
    """64 x 2^20 rows over 4,096 keys in binary32: 1,082,130,432 blocks of 16 x 16 with what the units count beside them, 1,056,769 a run.
    Compared: rows of the first and last units, of the units in which runs begin and of some others."""
    B, Sq, Sk, D = 64, 1 << 20, 4096, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    Q, K, V = (torch.randn(B, 1, s, D, generator=g, device="cuda") for s in (Sq, Sk, Sk))
    O = torch.full_like(Q, float("nan"))
    ws = torch.full((ac.attention_cross_workspace_bytes(B, 1, 1, Sq, Sk, D, Q.dtype) // 4,), float("nan"), device="cuda")
    ac.attention_cross(Q, K, V, O, ws)
    assert O.isfinite().all()
    per, cost = 1_056_769, Sk // 16 + 2
    units = {0, 1, B * Sq // 16 - 1} | {w * per // cost + x for w in range(0, 1024, 31) for x in (-1, 0, 1)} | {12345 * i for i in range(300)}
    by_item = {}
    for u in units:
        if 0 <= u < B * Sq // 16:
            by_item.setdefault(u * 16 // Sq, []).append(u * 16 % Sq)
    for b, rows in by_item.items():
        at = (torch.tensor(rows, device="cuda")[:, None] + torch.arange(16, device="cuda")).flatten()
        gen.check(O[b, 0, at], *gen.attend(Q[b, 0, at], K[b, 0], V[b, 0]))


def test_more_than_two_to_the_thirty_blocks_of_many_requests(ac):  # noqa: F811
    """2^19 requests on 8 heads, 8,144 tokens each in shared pages: 4,194,304 units of 255 blocks of 32 keys and two further ones."""
    B, H, D, page, width, n = 1 << 19, 8, 64, 16, 509, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    kp, vp = (torch.randn(n, H, page, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    Q = torch.randn(B, H, D, generator=g, device="cuda").bfloat16()
    table = torch.randint(0, n, (B, width), generator=g, device="cuda", dtype=torch.int32)
    lens = torch.full((B,), page * width, dtype=torch.int32, device="cuda")
    O = torch.full_like(Q, float("nan"))
    ws = torch.full((ac.attention_paged_workspace_bytes(B, H, H, D) // 4,), float("nan"), device="cuda")
    ac.attention_paged(Q, kp, vp, table, lens, O, ws)
    assert O.isfinite().all()
    per, cost = -(-B * H * 257 // 2048), 257
    runs = {w * per // cost // H for w in range(0, 2048, 97)}
    for b in sorted({0, 1, B - 2, B - 1} | runs | {x + 1 for x in runs}):
        k, v = (t[table[b].long()].transpose(0, 1).flatten(1, 2) for t in (kp, vp))
        for h in range(H):
            gen.check(O[b, h:h + 1], *gen.attend(Q[b, h:h + 1], k[h], v[h]))


@pytest.mark.parametrize("Hq,Hkv,D,dt", [(16, 2, 64, "bf16"), (12, 12, 64, "f32")])
def test_every_row_of_many_requests(ac, Hq, Hkv, D, dt):  # noqa: F811
    """More output rows than the join has waves: each wave has some that follow one another, over the ends of requests and over empty ones."""
    rnd = torch.Generator().manual_seed(D + Hq)
    lens = torch.randint(0, 130, (3000,), generator=rnd) * (torch.rand(3000, generator=rnd) < 0.7)
    lens[[0, 17, 18, 1500, 2999]] = torch.tensor([2500, 0, 1900, 3100, 1])
    c = Cache(lens.tolist(), Hkv, D, dt, 16, 5, width=200)
    Q = torch.randn(3000, Hq, D, generator=c.gen, device="cuda").to(c.k.dtype)
    O = c.call(ac, Q)
    assert O.isfinite().all() and (O[c.len == 0] == 0).all()
    c.check(O, Q, lens.nonzero().flatten().tolist())


def test_long_stretches_of_empty_requests(ac):  # noqa: F811
    """A run goes from a request to the next one that has tokens, past half a million that have none."""
    B = (1 << 20) + 3
    some = sorted({0, 1, 2, 64, 65, 200, 5000, 5063, 5064, 5065, 500_000, B - 130, B - 66, B - 65, B - 2, B - 1} | set(range(300_000, 300_400, 7)))
    few = Cache([1 + 331 * i % 1997 for i in range(len(some))], 1, 64, "bf16", 16, 6, width=130)
    c = Cache([0], 1, 64, "bf16", 16, 7)
    c.k, c.v = few.k, few.v
    c.table, c.len = torch.full((B, 130), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    c.table[some], c.len[some] = few.table, few.len
    Q = torch.randn(B, 3, 64, generator=c.gen, device="cuda").bfloat16()
    O = c.call(ac, Q)
    few.check(O[some], Q[some])
    assert (O[c.len == 0] == 0).all()


def test_items_left_out_between_others(ac):  # noqa: F811
    """Cross attention by runs with more rows than the join has waves, most items left out by row_sel and some empty."""
    B, H, Sq, Sk, D = 3000, 2, 8, 2100, 64
    g = torch.Generator(device="cuda").manual_seed(8)
    Q, K, V = (torch.randn(B, H, s, D, generator=g, device="cuda", dtype=torch.bfloat16) for s in (Sq, Sk, Sk))
    lens = torch.randint(0, 400, (B,), generator=torch.Generator().manual_seed(9)).int().cuda()
    lens[::9], lens[5] = 0, Sk
    sel = torch.full((B,), 3, dtype=torch.int32, device="cuda")
    sel[5:1000:3] = sel[2000:2100] = sel[-1] = -1
    O = torch.full_like(Q, 7.0)
    ws = torch.full((ac.attention_cross_workspace_bytes(B, H, H, Sq, Sk, D, Q.dtype) // 4,), float("nan"), device="cuda")
    ac.attention_cross(Q, K, V, O, ws, row_sel=sel, key_len=lens)
    assert (O[sel >= 0] == 7.0).all()
    for b in (sel < 0).nonzero().flatten().tolist():
        n = int(lens[b])
        for h in range(H):
            gen.check(O[b, h], *gen.attend(Q[b, h], K[b, h, :n], V[b, h, :n]))


@pytest.mark.parametrize("B,S,fresh", [(40_000, 1500, True), (20_000, 1025, False), (200_000, 200, True)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plans_of_more_requests_than_workgroups(ac, B, S, fresh, in_place):  # noqa: F811
    """Several rows a workgroup although each has more slots than one writes elsewhere; more is wanted than is free."""
    from perf import operators
    st = operators.prepare(dict(kind="plan", B=B, S=S, page=16, max_pages=200, lo=1, hi=S if fresh else 1500, fresh=fresh,
                                ended=0 if fresh else B // 5, short=True, spare=30), 11)
    want = operators._plain_plan(st)
    if in_place:
        st.update(seq_len_out=st["seq_len"], added=st["new_len"], free_state_out=st["free_state"])
    st["slot"].fill_(99)
    ac.attncache_page_plan(*(st[n] for n in ("seq_len", "new_len", "free_state", "free_pages", "page_table", "seq_len_out", "added",
                                             "free_state_out", "slot")), page_size=16)
    assert 0 < int((want["added"] > 0).sum()) < B
    for name, x in want.items():
        assert torch.equal(st[name], x), name
