"""References in 64 bits for the operators of generation after the prefill, and how far a kernel may be from them.

bf16: a weight is rounded once (by 2^-8 of itself), in numerator and denominator alike, so a result moves by at most
2^-8 sum_j p_j |v_j - o| <= 2^-8 (terms + |o|), and its own rounding is 2^-8 |o|; binary32 sums add what is below.
binary32: a score of D products is off by at most D + 8 roundings of its terms, a weight by twice that, by its exponential and
the scaling of its argument (64 bits of range at the most: 2^-24 each, twice), and a sum over n keys by n + 16 roundings."""
import torch


def attend(q, k, v, scale=None):
    """q [R,D] to k and v [n,D]: result, sum of the terms' magnitudes, and the binary32 bound relative to the latter."""
    q, k, v = q.double(), k.double(), v.double()
    n, D = k.shape
    scale = D ** -0.5 if scale is None else scale
    if n == 0:
        z = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
        return z, z, z[:, :1]
    p = torch.softmax(q @ k.t().contiguous() * scale, -1)
    size = (q.abs() @ k.abs().t().contiguous()).amax(-1, keepdim=True) * scale
    return p @ v, p @ v.abs(), (2 * (D + 8) * size + 2 * (n + 16) + 256) * 2.0 ** -24


def check(o, want, terms, bound):
    got = o.double()
    if o.dtype == torch.bfloat16:
        tol = 2.0 ** -8 * 1.01 * (2 * want.abs() + terms) + terms * torch.clamp(bound, max=1e-2) + 1e-30
    else:
        tol = terms * bound + want.abs() * 2.0 ** -23 + 1e-30
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()), float(tol.min()))


class Pages:
    """The plan of a step, kept by hand."""

    def __init__(self, n_pages, page, max_pages, B, order):
        self.n, self.p, self.width = n_pages, page, max_pages
        self.ring, self.first, self.count = list(order), 0, n_pages
        self.table = [[-7] * max_pages for _ in range(B)]
        self.len = [0] * B

    def step(self, new, S):
        held = lambda t: -(-t // self.p)  # noqa: E731
        queue, taken, freed, added, slots = 0, 0, [], [], []
        for b, n in enumerate(new):
            row, s, took = self.table[b], self.len[b], 0
            if n < 0:
                freed += row[:held(s)]
                self.len[b] = 0
            else:
                n = min(n, S)
                need = held(s + n) - held(s)
                if s + n <= self.width * self.p:
                    queue += need
                    if need == 0 or queue <= self.count:
                        took = n
                        for i in range(need):
                            row[held(s) + i] = self.ring[(self.first + taken + i) % self.n]
                        taken += need
                self.len[b] = s + took
            added.append(took)
            slots.append([row[(s + t) // self.p] * self.p + (s + t) % self.p if t < took else -1 for t in range(S)])
        for i, q in enumerate(freed):
            self.ring[(self.first + self.count + i) % self.n] = q
        self.first, self.count = (self.first + taken) % self.n, self.count - taken + len(freed)
        return added, slots
