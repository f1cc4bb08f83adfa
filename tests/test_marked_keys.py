"""Whether marked keys do what they are for, in 64 bits and without a GPU: a result from which a block of keys is missing, or that has one
twice, is told from the right one, whichever block it is, in each head by itself."""
import pytest
import torch

from tests import marked_keys as mk


@pytest.mark.parametrize("dtype,block", [(torch.bfloat16, 32), (torch.float32, 16)])
@pytest.mark.parametrize("n,H,D", [(131_073, 2, 64), (131_072, 2, 128), (70_001, 3, 64), (30_000, 2, 128), (20_001, 2, 64), (9_000, 2, 128), (4_129, 1, 64)])
@pytest.mark.parametrize("times", [0, 2])
def test_each_block_is_noticed(n, H, D, dtype, block, times):
    V = mk.marks(n, H, D).double()
    start = torch.arange(0, n, block)
    first = torch.nn.functional.pad(V.cumsum(1), (0, 0, 1, 0))
    per_block = first[:, (start + block).clamp(max=n)] - first[:, start]                # [H,blocks,D]
    size = ((start + block).clamp(max=n) - start).double()[None, :, None]
    got = ((V.sum(1, keepdim=True) + (times - 1) * per_block) / (n + (times - 1) * size)).to(dtype).double()
    want = V.sum(1, keepdim=True) / n
    noticed = ((got - want).abs() > mk.tolerance(dtype) * want).any(2)
    # (a last block of a few keys is too little for a bf16 result of hundreds of them)
    assert noticed[:, size.flatten() >= (32 if dtype == torch.bfloat16 else 1)].all()
    mk.check(want.to(dtype), V)
