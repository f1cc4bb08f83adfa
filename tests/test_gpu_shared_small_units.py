"""Attention of requests that share prefixes where there is little to read and units are many: the same whatever is said to be shared, and no further from the
definition than attention over pages."""
import pytest
import torch

from tests import generation as gen
from tests.test_gpu_paged_attention import DT, TYPES
from tests.test_gpu_parity_small import ac  # noqa: F401
from tests.test_gpu_shared_attention import build, call

pytestmark = pytest.mark.gpu


# 1,203 requests of one K/V head, up to 30 tokens; 822 of 20 heads, which are two units, up to 55 (in binary32 too few of those for a wave each)
@pytest.mark.parametrize("groups,alone,Hq,Hkv", [([(20, [3, 0, 7] * 4)] * 100, [1, 0, 30], 4, 1), ([(50, [0, 5] * 4)] * 100, [9, 0] * 11, 20, 1)], ids=["4x1", "20x1"])
@pytest.mark.parametrize("D,dt", TYPES)
def test_many_small_units_and_attention_over_pages(ac, D, dt, groups, alone, Hq, Hkv):  # noqa: F811
    c, first, share = build(groups, alone, Hkv, D, dt, 16, wide=False, blank=False)
    B = len(c.rows)
    assert B * Hkv * -(-Hq // 16) >= 1024
    Q = torch.randn(B, Hq, D, generator=c.gen, device="cuda").to(DT[dt])
    O = call(ac, c, Q, first, share)
    assert torch.equal(O, call(ac, c, Q, first[:1], share[:0]))      # no groups: the same launch
    E = c.call(ac, Q)                                                # (may add up in another order)
    for b in range(0, B, 23):
        for h in range(Hkv):
            want = gen.attend(Q[b], c.rows[b][0][h], c.rows[b][1][h])
            gen.check(O[b], *want)
            gen.check(E[b], *want)
    empty = c.len == 0
    assert empty.any() and (O[empty] == 0).all() and (E[empty] == 0).all()
