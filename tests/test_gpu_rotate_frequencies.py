"""Rotated heads with frequencies of any sign and size, at near and far positions, against 64 bits."""
import math

import pytest
import torch

from tests.test_gpu_parity_small import ac  # noqa: F401
from tests.test_gpu_rotate import expect, near

pytestmark = pytest.mark.gpu

# none, hardly any, a rotation taken back, whole and half turns a position and beside them, beyond a turn
ODD = [0.0, -0.0, 1e-300, -1e-300, 1e-16, -1e-16, -2.5e-16, -3.4e-16, -4e-16, 1e-9, -1e-9, -1e-4, 0.3, -0.3, -1.0, math.pi, -math.pi, 2 * math.pi, -2 * math.pi,
       math.nextafter(2 * math.pi, 7), -math.nextafter(2 * math.pi, 7), math.nextafter(2 * math.pi, 6), -math.nextafter(2 * math.pi, 6), 4 * math.pi, -6 * math.pi,
       math.pi / 2, -math.pi / 2, -7.0, 1e3, -1e3, 2.0 ** 20 + 0.1, -2.0 ** 20 - 0.1]


@pytest.mark.parametrize("first", [0, 10 ** 6, 2 ** 31 - 12])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_frequencies_of_any_sign_and_size(ac, dt, interleaved, first):  # noqa: F811
    S, D, g = 11, 64, torch.Generator(device="cuda").manual_seed(first % 97)
    X = torch.randn(1, S, 4 * D, generator=g, device="cuda").to(dt)
    pos = (first + torch.arange(S, device="cuda")).int().view(1, S)
    Q, K, V = (torch.empty(1, h, S, D, dtype=dt, device="cuda") for h in (2, 1, 1))
    for f in ODD:      # by itself: the tolerance grows with the largest angle
        freq = torch.full((D // 2,), f, dtype=torch.float64, device="cuda")
        ac.attncache_rotate(X, pos, freq, Q, K, V, interleaved=interleaved)
        want, tol = expect(X, pos, freq, 2, 1, D, None, None, 1e-6, 1.0, interleaved)
        for t, lo, hi in ((Q, 0, 2), (K, 2, 3), (V, 3, 4)):
            near(t, want[:, lo:hi], tol[:, lo:hi], torch.ones(1, 1, 1, 1, dtype=torch.bool, device="cuda"))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_a_negative_frequency_is_the_rotation_taken_back(ac, dt):  # noqa: F811
    """Sines change their sign and nothing else: the second half of a pair with -f is what the first half is with f when the two change places."""
    S, D, g = 9, 128, torch.Generator(device="cuda").manual_seed(3)
    X = torch.randn(1, S, 3 * D, generator=g, device="cuda").to(dt)
    swap = X.view(1, S, 3, 2, D // 2).flip(3).reshape(1, S, 3 * D).contiguous()
    freq = ac.attncache_rotary_frequencies(D).cuda()
    for first in (0, 5, 10 ** 7, 2 ** 31 - 10):
        pos = (first + torch.arange(S, device="cuda")).int().view(1, S)
        out = []
        for x, f in ((X, freq), (swap, -freq)):
            out.append([torch.empty(1, 1, S, D, dtype=dt, device="cuda") for _ in range(3)])
            ac.attncache_rotate(x, pos, f, *out[-1])
        for a, b in zip(*out):
            a, b = a.view(S, 2, D // 2).double(), b.view(S, 2, D // 2).flip(1).double()
            x = X.double().abs()
            # a product and a sum in binary32 each way, whose order the two calls may not share, and the rounding of the result
            assert ((a - b).abs() <= 4 * 2.0 ** -24 * 2 * x.max() + (2.0 ** -7 * a.abs() if dt == torch.bfloat16 else 0)).all()
