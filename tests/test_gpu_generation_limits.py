"""The operators of generation at sizes near their limits, where index arithmetic of 32 bits comes to its end.  (The arithmetic alone:
test_generation_index.py, without a GPU.)"""
import pytest
import torch

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
