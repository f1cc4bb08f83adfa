"""Attention within a window at scores far beyond a million: the largest ones weigh one, whatever is lost of the differences between them."""
import pytest
import torch

from tests.test_gpu_parity_small import ac  # noqa: F401
from tests.test_gpu_window_attention import DT, call, seen_by

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponent", [20, 27, 29, 30, 31, 33, 36, 40, 60])
@pytest.mark.parametrize("D,dt", [(64, "bf16"), (128, "bf16"), (64, "f32"), (100, "f32")])
def test_equal_scores_of_any_size(ac, D, dt, exponent):  # noqa: F811
    """One column says what a score is, a whole number of sixteen bits times a power of two, the same for all keys of a row but for a few that score nothing:
    a result is the mean of the others' V."""
    S, window, sinks, H = 150, 40, 3, 6
    odd = torch.tensor([129.0, 131, 165, 173, 201, 255], device="cuda")      # eight bits each
    Q, K = torch.zeros(1, H, S, D, device="cuda"), torch.zeros(1, H, S, D, device="cuda")
    Q[0, :, :, 5] = odd[torch.arange(S, device="cuda") % 6] * 2.0 ** (exponent - 14)
    K[0, :, :, 5] = odd[:H, None]
    nothing = torch.arange(S, device="cuda") % 7 == 3
    K[0, :, nothing] = 0
    V = torch.randint(-20, 20, (1, H, S, D), device="cuda").float()
    Q, K, V = (x.to(DT[dt]) for x in (Q, K, V))
    O = call(ac, Q, K, V, None, window, sinks, scale=1.0)
    p = (seen_by(S, S, window, sinks) & ~nothing).double()
    want = torch.matmul(p, V[0].double()) / p.sum(-1, keepdim=True)
    # all weights are the same, but not one: n products, n sums of them and n of the weights round once each, by 2^-24 of at most the sum of all terms' sizes;
    # then a reciprocal, a product and the result's rounding
    terms = torch.matmul(p, V[0].double().abs()) / p.sum(-1, keepdim=True)
    tol = (2.0 ** -8 if dt == "bf16" else 0) * want.abs() + (3 * (window + sinks) + 4) * 2.0 ** -24 * terms
    assert ((O[0].double() - want).abs() <= tol).all()
