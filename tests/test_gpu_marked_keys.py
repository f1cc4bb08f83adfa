"""Attention over long contexts with marked keys: no block of keys is lost or counted twice, at the ends of runs, pages and chunks or
anywhere else.  Whether a single block would be noticed: test_marked_keys.py."""
import pytest
import torch

from tests import marked_keys as mk
from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("lens,width", [([131_072, 30_000, 70_001, 9_000, 33], None), ([131_073], None), ([70_001, 0, 1, 70_000] * 3, None),
                                        ([9_000] * 20 + [2_113] * 30 + [0, 40] * 20, 2_000), ([4_129] * 64, None)],
                         ids=lambda x: f"{len(x)}x{max(x)}" if isinstance(x, list) else str(x))
@pytest.mark.parametrize("Hq,Hkv,D,dt,page", [(8, 2, 128, "bf16", 16), (6, 2, 64, "bf16", 7), (2, 2, 64, "bf16", 128), (20, 1, 128, "bf16", 64),
                                              (6, 2, 128, "f32", 16), (2, 1, 80, "f32", 10), (17, 1, 64, "f32", 64)])
def test_paged(ac, lens, width, Hq, Hkv, D, dt, page):  # noqa: F811
    held = [-(-n // page) for n in lens]
    n_pages = sum(held) + 2
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(len(lens)))
    table = torch.full((len(lens), max(max(held), (width or 0) * 16 // page)), -1)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.full((n_pages, Hkv, page, D), float("nan"), device="cuda", dtype=DT[dt]) for _ in range(2))
    V = {n: mk.marks(n, Hkv, D).cuda() for n in set(lens)}
    at = 0
    for b, (n, q) in enumerate(zip(lens, held)):
        table[b, :q] = order[at:at + q]
        at += q
        j = torch.arange(n, device="cuda")
        to = table[b].cuda()[j // page], slice(None), j % page
        k[to] = torch.randn(n, Hkv, D, generator=g, device="cuda").to(DT[dt])
        v[to] = V[n].transpose(0, 1).to(DT[dt])
    Q, O = (torch.zeros(len(lens), Hq, D, device="cuda", dtype=DT[dt]) for _ in range(2))
    ws = torch.full((ac.attention_paged_workspace_bytes(len(lens), Hq, Hkv, D) // 4,), float("nan"), device="cuda")
    ac.attention_paged(Q, k, v, table.int().cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), O, ws)
    for b, n in enumerate(lens):
        if n:
            mk.check(O[b].view(Hkv, Hq // Hkv, D), V[n])
        else:
            assert (O[b] == 0).all()


# few rows (runs of blocks, units) and many (chunks in LDS, with reference points that stay and that follow)
@pytest.mark.parametrize("B,Hq,Hkv,Sq,lens", [(3, 6, 2, 1, [70_001, 0, 131_072]), (2, 4, 4, 30, [20_001, 9_000]), (6, 12, 12, 1, [2_049, 33, 1_500, 4_129, 31, 0]),
                                              (3, 8, 4, 700, [20_001, 4_129, 0]), (2, 16, 16, 513, [9_000, 635]), (40, 4, 2, 33, [700, 639, 64, 96] * 10)])
@pytest.mark.parametrize("D,dt", [(64, "bf16"), (128, "bf16"), (64, "f32"), (128, "f32"), (36, "f32"), (101, "f32"), (256, "f32")])
def test_cross(ac, B, Hq, Hkv, Sq, lens, D, dt):  # noqa: F811
    Sk = max(lens)
    g = torch.Generator(device="cuda").manual_seed(2)
    K = torch.randn(B, Hkv, Sk, D, generator=g, device="cuda").to(DT[dt])
    V = torch.full_like(K, float("nan"))
    marks = {n: mk.marks(n, Hkv, D).cuda() for n in set(lens)}
    for b, n in enumerate(lens):
        V[b, :, :n], K[b, :, n:] = marks[n].to(DT[dt]), float("nan")
    Q, O = (torch.zeros(B, Hq, Sq, D, device="cuda", dtype=DT[dt]) for _ in range(2))
    ws = torch.full((max(4, ac.attention_cross_workspace_bytes(B, Hq, Hkv, Sq, Sk, D, DT[dt]) // 4),), float("nan"), device="cuda")
    ac.attention_cross(Q, K, V, O, ws, key_len=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    for b, n in enumerate(lens):
        if n:
            mk.check(O[b].view(Hkv, Hq // Hkv * Sq, D), marks[n])
        else:
            assert (O[b] == 0).all()
