"""The page plan and K and V rows into their pages, against the same kept by hand."""
import random

import pytest
import torch

from tests.generation import Pages
from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _run(ac, st, new, S, page, in_place, slot=None):
    B = st["table"].shape[0]
    slot = torch.full((B, S), 99, dtype=torch.int32, device="cuda") if slot is None else slot
    if in_place:
        out = dict(seq=st["seq"], added=new, state=st["state"])
    else:
        out = {n: torch.full_like(t, 77) for n, t in (("seq", st["seq"]), ("added", new), ("state", st["state"]))}
    ac.attncache_page_plan(st["seq"], new, st["state"], st["ring"], st["table"], out["seq"], out["added"], out["state"], slot,
                           page_size=page)
    st["seq"], st["state"] = out["seq"], out["state"]
    return out["added"], slot


# requests, most new tokens, page size, row of the table, pages, steps
PLANS = [(1, 1, 16, 4, 5, 80), (1, 1, 1, 3, 3, 6), (5, 3, 10, 9, 40, 30), (64, 1, 16, 8, 300, 40), (64, 2, 16, 40, 90, 60),
         (300, 17, 7, 20, 2500, 12), (1500, 2, 16, 5, 4000, 6), (1500, 40, 16, 9, 9000, 6), (3, 3001, 64, 120, 200, 6),
         (2, 5000, 1, 9000, 11000, 4), (257, 9, 48, 3, 500, 8), (4097, 1, 16, 3, 9000, 4)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", PLANS, ids=str)
def test_plans_of_many_steps(ac, case, in_place):  # noqa: F811
    B, S, page, width, n, steps = case
    rng = random.Random(B + S + page)
    order = list(range(n))
    rng.shuffle(order)
    hand = Pages(n, page, width, B, order)
    st = dict(seq=_i32(hand.len), state=_i32([0, n]), ring=_i32(order), table=_i32(hand.table))
    refused = 0
    for _ in range(steps):
        new = [rng.choice([-1, 0, 1, 1, S, S, S + 3, rng.randint(0, S)]) for _ in range(B)]
        added, slots = hand.step(new, S)
        got_added, got_slots = _run(ac, st, _i32(new), S, page, in_place)
        refused += sum(a < min(x, S) for a, x in zip(added, new))
        assert got_added.tolist() == added
        assert got_slots.tolist() == slots
        assert st["seq"].tolist() == hand.len and st["state"].tolist() == [hand.first, hand.count]
        assert st["table"].tolist() == hand.table and st["ring"].tolist() == hand.ring
    live = sum(-(-t // page) for t in hand.len)
    assert live + hand.count == n     # no page is lost or held twice
    held = [q for b, t in enumerate(hand.len) for q in hand.table[b][:-(-t // page)]]
    assert len(set(held)) == len(held)


def test_a_captured_plan_goes_on_by_itself(ac):  # noqa: F811
    B, page, width, n = 9, 4, 6, 40
    order = list(range(n))
    random.Random(3).shuffle(order)
    hand = Pages(n, page, width, B, order)
    st = dict(seq=_i32(hand.len), state=_i32([0, n]), ring=_i32(order), table=_i32(hand.table))
    new, out = _i32([1] * B), torch.zeros(B, dtype=torch.int32, device="cuda")
    slot = torch.zeros(B, 1, dtype=torch.int32, device="cuda")

    def step():
        ac.attncache_page_plan(st["seq"], new, st["state"], st["ring"], st["table"], st["seq"], out, st["state"], slot,
                               page_size=page)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(30):
        todo = [1] * B if i % 4 else [-1 if b == i // 4 else 1 for b in range(B)]
        new.copy_(_i32(todo))
        if i % 5 == 2:
            step()
        else:
            graph.replay()
        added, slots = hand.step(todo, 1)
        assert out.tolist() == added and slot.tolist() == slots and st["seq"].tolist() == hand.len
        assert st["state"].tolist() == [hand.first, hand.count] and st["table"].tolist() == hand.table


def test_lengths_and_states_out_of_range_are_clamped(ac):  # noqa: F811
    # (a length beyond its row counts as a full row, a negative one as none; the ring's first is taken modulo its size)
    page, width, n, S = 8, 3, 10, 4
    order = list(range(n))
    seq, state, table = _i32([1000, -5, 3]), _i32([-3, 99]), _i32([[0, 1, 2], [-1] * 3, [3, -1, -1]])
    st = dict(seq=seq, state=state, ring=_i32(order), table=table)
    added, slot = _run(ac, st, _i32([2, 3, 0]), S, page, False)
    assert added.tolist() == [0, 3, 0] and st["seq"].tolist() == [24, 3, 3]
    assert slot.tolist() == [[-1] * 4, [56, 57, 58, -1], [-1] * 4]
    assert st["state"].tolist() == [8, 9] and st["table"][1].tolist() == [7, -1, -1]


def test_page_numbers_out_of_range_give_no_slot(ac):  # noqa: F811
    n, page = 6, 4
    st = dict(seq=_i32([2, 4, 4]), state=_i32([0, 3]), ring=_i32([100, -1, 5, 0, 0, 0]), table=_i32([[9, 9], [1, 9], [2, 9]]))
    added, slot = _run(ac, st, _i32([1, 2, 1]), 2, page, False)
    assert added.tolist() == [1, 2, 1] and slot.tolist() == [[-1, -1], [-1, -1], [-1, -1]]
    assert st["table"].tolist() == [[9, 9], [1, 100], [2, -1]]


# B, H, S, D, dtype, pages, page size, further elements of a page
APPENDS = [(1, 1, 1, 64, "bf16", 1, 1, 0), (128, 8, 1, 128, "bf16", 300, 16, 0), (7, 3, 33, 64, "bf16", 40, 16, 64),
           (4, 2, 129, 128, "bf16", 9, 100, 8), (64, 16, 31, 64, "bf16", 200, 10, 0), (3, 2, 17, 1, "f32", 60, 1, 3),
           (5, 3, 50, 33, "f32", 30, 16, 0), (5, 3, 50, 100, "f32", 30, 16, 4), (2, 4, 40, 199, "f32", 20, 7, 1),
           (9, 1, 21, 256, "f32", 5, 64, 0), (2, 5, 300, 80, "f32", 100, 8, 0)]


@pytest.mark.parametrize("case", APPENDS, ids=str)
def test_rows_go_to_their_slots(ac, case):  # noqa: F811
    B, H, S, D, dt, n, page, more = case
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(B * S + D)
    K, V = (torch.randn(B, H, S, D, generator=g, device="cuda").to(dtype) for _ in range(2))
    room = torch.randn(2, n, H * page * D + more, generator=g, device="cuda").to(dtype)
    pages = [room[i].as_strided((n, H, page, D), (H * page * D + more, page * D, D, 1),
                                i * n * (H * page * D + more)) for i in range(2)]
    start = room.clone()
    order = torch.randperm(n * page, generator=torch.Generator().manual_seed(S))[:B * S]
    slot = torch.full((B * S,), -1, dtype=torch.int32)
    slot[:len(order)] = order.int()
    slot = slot[torch.randperm(B * S, generator=torch.Generator().manual_seed(7))]
    some = torch.rand(B * S, generator=torch.Generator().manual_seed(9))
    slot[some < 0.1] = torch.tensor([-1, n * page, 2**31 - 1, -2**31])[torch.arange(int((some < 0.1).sum())) % 4].int()
    ac.attncache_page_append(K, V, slot.view(B, S).cuda(), *pages)
    want = start.clone()
    for i, rows in enumerate((K, V)):
        to = want[i].as_strided((n, H, page, D), (H * page * D + more, page * D, D, 1), i * n * (H * page * D + more))
        for x, s in enumerate(slot.tolist()):
            if 0 <= s < n * page:
                to[s // page, :, s % page] = rows[x // S, :, x % S]
    assert torch.equal(room, want)


def test_layers_and_both_tensors_in_one_array(ac):  # noqa: F811
    """[n_pages][K, V][layers x heads][page][D]: a layer's part of it is a view whose pages lie far apart."""
    n, L, H, page, D, B, S = 12, 3, 2, 16, 64, 4, 20
    g = torch.Generator(device="cuda").manual_seed(1)
    cache = torch.zeros(n, 2, L * H, page, D, device="cuda", dtype=torch.bfloat16)
    K, V = (torch.randn(B, L, H, S, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    slot = torch.randperm(n * page, generator=torch.Generator().manual_seed(2))[:B * S].int().view(B, S).cuda()
    for layer in range(L):
        part = cache[:, :, layer * H:(layer + 1) * H]
        ac.attncache_page_append(K[:, layer].contiguous(), V[:, layer].contiguous(), slot, part[:, 0], part[:, 1])
    at = slot.long()
    for rows, which in ((K, 0), (V, 1)):
        got = cache[at // page, which, :, at % page]                       # [B,S,L*H,D]
        assert torch.equal(got, rows.flatten(1, 2).transpose(1, 2))
    whole = torch.zeros_like(cache)
    ac.attncache_page_append(K.flatten(1, 2), V.flatten(1, 2), slot, whole[:, 0], whole[:, 1])
    assert torch.equal(whole, cache)


def test_rows_behind_two_gibi_elements(ac):  # noqa: F811
    n, H, page, D = 40_000, 4, 128, 128                                   # 2.6e9 elements, 5.2 GB a tensor
    pages = [torch.empty(n, H, page, D, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    slot = _i32([[n * page - 1, 0, 33_000 * page + 5, -1]])
    K, V = (torch.randn(1, H, 4, D, device="cuda").bfloat16() for _ in range(2))
    ac.attncache_page_append(K, V, slot, *pages)
    for rows, to in zip((K, V), pages):
        assert torch.equal(to[n - 1, :, page - 1], rows[0, :, 0]) and torch.equal(to[0, :, 0], rows[0, :, 1])
        assert torch.equal(to[33_000, :, 5], rows[0, :, 2])
