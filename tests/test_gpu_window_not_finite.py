"""Attention of prompts within a window where rows of Q, or values, are not finite: who sees them gets what they are, nobody else notices, and the call stays
within a few times its own duration."""
import pytest
import torch

from tests import generation as gen
from tests.test_gpu_parity_small import ac  # noqa: F401
from tests.test_gpu_window_attention import DT, TYPES, attend, call, data, seen_by

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
# B, Hq, Hkv, S, window, sinks: one head on a K and V and several, workgroups of one item's last rows, binary32 in workgroups of 32 rows and of 64
SIZES = [(1, 4, 2, 300, 40, 3), (2, 3, 3, 97, 20, 0), (33, 12, 4, 100, 30, 5), (2, 8, 1, 200, 1000, 0)]


def spoil(V, seed):
    """Some values of some keys, all of one key, a column of many keys."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    S, D = V.shape[2:]
    V = V.clone()
    kinds = torch.tensor([NAN, INF, -INF], device="cuda")
    at = torch.rand(V.shape, generator=g, device="cuda") < 0.3
    at &= (torch.rand(V.shape[:3], generator=g, device="cuda") < 0.04)[..., None]
    V[at] = kinds[torch.randint(3, (int(at.sum()),), generator=g, device="cuda")].to(V.dtype)
    V[0, 0, S // 2] = NAN
    V[-1, -1, S // 3:S // 3 + 40, D // 2] = INF
    V[-1, -1, S // 2:S // 2 + 9, D // 2] = -INF
    return V


@pytest.mark.parametrize("steep", [1, 40])
@pytest.mark.parametrize("D,dt", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_values_go_to_the_rows_that_see_them(ac, size, D, dt, steep):  # noqa: F811
    """steep: scores grow by hundreds, so that earlier weights become nothing in binary32; they are not nothing."""
    B, Hq, Hkv, S, window, sinks = size
    lens = None if B == 1 else [(S, S // 2, 3, 0)[b % 4] for b in range(B)]
    Q, K, V, lens = data(B, Hq, Hkv, S, D, dt, lens)
    Q = Q * steep
    bad = spoil(V, S + D)
    seen = torch.stack([seen_by(S, S if lens is None else int(n), window, sinks) for n in (lens if lens is not None else [S] * B)])
    g = Hq // Hkv
    met = lambda x: (seen[:, None].double() @ x.double()).repeat_interleave(g, 1) > 0  # noqa: E731
    up, down = (met((bad == v) | bad.isnan()) for v in (INF, -INF))
    clean = call(ac, Q, K, torch.where(bad.isfinite(), bad, torch.zeros_like(bad)), lens, window, sinks)
    assert clean.isfinite().all()
    O = call(ac, Q, K, bad, lens, window, sinks)
    want = clean + torch.where(up, INF, 0.0).to(O.dtype) + torch.where(down, -INF, 0.0).to(O.dtype)
    assert torch.equal(O.isnan(), want.isnan()) and torch.equal(torch.nan_to_num(O), torch.nan_to_num(want))
    assert (up & down).any() and not (up | down).all() and (D < 33 or (up & ~down).any())


@pytest.mark.parametrize("D,dt", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_rows_that_are_not_finite_stay_by_themselves(ac, size, D, dt):  # noqa: F811
    """Padding of Q holds anything, as memory does that nobody wrote; K and V of the last keys too, where no length hides them."""
    B, Hq, Hkv, S, window, sinks = size
    real = [(S - 9, S // 2, 3, 0)[b % 4] for b in range(B)]
    Q, K, V, lens = data(B, Hq, Hkv, S, D, dt, None if B == 1 else real)
    for value in (NAN, INF, -INF):
        odd = Q.clone()
        for b, n in enumerate(real):
            odd[b, :, n:] = value
            odd[b, :, n + 1::3] = 5.0
        if value != value and B == 1:
            K[:, :, real[0]:] = V[:, :, real[0]:] = NAN
        O = call(ac, odd, K, V, lens, window, sinks)
        for b, n in enumerate(real):
            for h in {0, Hq - 1} if n and b in (0, 1, B - 1) else ():      # (rows of one wave move their reference points together: equal but for roundings)
                seen = seen_by(S, n, window, sinks)[:n]
                gen.check(O[b, h, :n], *attend(Q[b, h, :n], K[b, h * Hkv // Hq], V[b, h * Hkv // Hq], seen))
            if value != value and n > window:
                assert O[b, :, n:S:3].isnan().all() if lens is None else O[b, :, n:min(n + window - 1, S):3].isnan().all()


@pytest.mark.parametrize("D,dt", [(64, "bf16"), (128, "bf16"), (64, "f32"), (128, "f32"), (100, "f32")])
def test_what_is_not_finite_takes_a_few_times_as_long(ac, D, dt):  # noqa: F811
    S, window = 1500, 700
    Q, K, V, _ = data(2, 8, 4, S, D, dt, None)
    O = torch.empty_like(Q)

    def took(Q, K, V):
        best = INF
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            for _ in range(4):
                ac.attention_window(Q, K, V, O, window=window, sinks=4)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    usual = took(Q, K, V)
    rows, values, sink = Q.clone(), V.clone(), V.clone()
    rows[:, :, 1000:] = NAN
    sink[:, :, 2] = NAN
    values[:, :, ::50, 3] = INF
    for q, v in ((rows, V), (Q, sink), (Q, values), (rows, values)):
        assert took(q, K, v) < 12 * usual      # (four walks in the place of one, three of which set values apart at up to three times its duration, and what a timer is off by)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_scores_of_minus_infinity_weigh_nothing_beside_infinite_values(ac, dt):  # noqa: F811
    S, D = 130, 64
    Q, K, V, _ = data(1, 2, 1, S, D, dt, None)
    Q.abs_()
    K[0, 0, 40:44], V[0, 0, 41], V[0, 0, 100, 5] = -INF, INF, -INF
    O = call(ac, Q, K, V, None, 60, 2)
    seen = seen_by(S, S, 60, 2)
    t = torch.arange(S, device="cuda")
    assert (O[0, :, 100:, 5] == -INF).all()
    seen[:, 40:44] = False
    V[0, 0, 41], V[0, 0, 100, 5] = 0, 0
    for h in range(2):
        w = attend(Q[0, h], torch.nan_to_num(K[0, 0], neginf=0.0), V[0, 0], seen)
        keep = (t < 100) | (t >= 160)
        gen.check(O[0, h][keep], *(x[keep] for x in w))
