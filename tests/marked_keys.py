"""Keys that can be missed: data for long sequences where each block of keys moves the result by far more than a kernel may be off.

Against rows of normal values a lost block is lost among tens of thousands of others: a result goes to zero with their number, and
what a kernel may be off by does not.  Here Q is zero, so that all weights are one, and V is one in a single column of each group of 32
keys and zero elsewhere, so that a result is the share of the keys that are marked in its column: n / D of n, of which a group is one in
n / (32 D).  The weights, their sum (below 2^24) and the marked ones' are whole numbers, which no arithmetic rounds; what is left is a
division, a product and the result's own rounding."""
import torch

GROUP = 32


def marks(n, H, D):
    """V [H,n,D] of ones and zeros; heads mark other columns."""
    column = (torch.arange(n) // GROUP + 5 * torch.arange(H)[:, None]) % D
    return torch.zeros(H, n, D).scatter_(2, column[:, :, None], 1.0)


def tolerance(dtype):
    """Relative: half a step of bf16, or a division (2.5 steps of binary32 at the most) and a product, half a step each."""
    return (2.0 ** -8 if dtype == torch.bfloat16 else 0.0) + 6 * 2.0 ** -24


def check(o, V):
    """o [...,H,rows,D] for V [H,n,D]."""
    want = (V.double().sum(1) / V.shape[1]).unsqueeze(-2).to(o.device)
    bad = ~((o.double() - want).abs() <= tolerance(o.dtype) * want)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:3].tolist())
