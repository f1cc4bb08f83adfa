"""Rotated heads of which only Q's or only K's are normalised, against 64 bits: a wave that goes from Q heads to K heads keeps no weights of the former."""
import pytest
import torch

from tests.test_gpu_parity_small import ac  # noqa: F401
from tests.test_gpu_rotate import DT, expect, near

pytestmark = pytest.mark.gpu

# tokens, heads, K/V heads, head dimension, type, rotated columns: many tokens (all heads in one workgroup, of which a wave takes every fourth, three or so at
# a time) and few; pairs that lie whole pieces apart and not, rows of whole pieces and not, columns that do not turn
SIZES = [(9000, 5, 3, 128, "bf16", 128), (9000, 6, 2, 128, "bf16", 94), (18000, 9, 3, 64, "bf16", 62), (18000, 3, 5, 64, "bf16", 20),
         (9000, 5, 3, 64, "f32", 64), (5000, 5, 3, 128, "f32", 30), (3000, 10, 2, 256, "f32", 256), (2500, 6, 3, 33, "f32", 32), (2500, 5, 2, 101, "f32", 100),
         (2500, 3, 3, 199, "f32", 90), (7, 1, 1, 128, "bf16", 94), (7, 32, 8, 64, "bf16", 64), (7, 5, 3, 100, "f32", 50), (1, 40, 2, 128, "f32", 126)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_one_of_both_is_normalised(ac, size, which, interleaved):  # noqa: F811
    B, Hq, Hkv, D, dt, rot = size
    g = torch.Generator(device="cuda").manual_seed(B + D)
    X = (3 * torch.randn(B, 1, (Hq + 2 * Hkv) * D, generator=g, device="cuda")).to(DT[dt])      # (a norm that is left out shows)
    pos = torch.arange(B, device="cuda").int().view(B, 1)
    freq = ac.attncache_rotary_frequencies(rot).cuda()
    w = 1 + 0.3 * torch.randn(D, generator=g, device="cuda")
    qw, kw = (w, None) if which == "q" else (None, w)
    Q, K, V = (torch.full((B, h, 1, D), 7.0, dtype=DT[dt], device="cuda") for h in (Hq, Hkv, Hkv))
    ac.attncache_rotate(X, pos, freq, Q, K, V, q_weight=qw, k_weight=kw, eps=1e-5, interleaved=interleaved)
    want, tol = expect(X, pos, freq, Hq, Hkv, D, qw, kw, 1e-5, 1.0, interleaved)
    for t, lo, hi in ((Q, 0, Hq), (K, Hq, Hq + Hkv), (V, Hq + Hkv, Hq + 2 * Hkv)):
        near(t, want[:, lo:hi], tol[:, lo:hi], torch.ones(1, 1, 1, 1, dtype=torch.bool, device="cuda"))
