"""Attention over pages by runs and units of many requests: each row of each request against plain attention in 64 bits."""
import pytest
import torch

from tests import test_gpu_paged_attention as paged
from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu

CASES = (paged.RUNS + [(lens, *t, 16) for lens in paged.RAGGED for t in paged.RAGGED_TYPES if len(lens) > 40] +
         [(paged.EDGES * 5, 6, 2, D, dt, 16) for D, dt in paged.TYPES])


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{max(c[0])}-" + "-".join(map(str, c[1:])))
def test_every_row(ac, case):  # noqa: F811
    lens, Hq, Hkv, D, dt, page = case
    c = paged.Cache(lens, Hkv, D, dt, page, sum(lens) + 3 * D)
    Q = torch.randn(len(lens), Hq, D, generator=c.gen, device="cuda").to(c.k.dtype)
    O = c.call(ac, Q)
    assert (O[c.len == 0] == 0).all()
    c.check(O, Q, c.len.nonzero().flatten().tolist())
