"""Attention of prompts within a window and with first tokens that stay visible, against plain attention in 64 bits.  Padding is NaN, and
so is what is not to be written."""
import random

import pytest
import torch

from tests import generation as gen
from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def seen_by(S, n, window, sinks):
    t, j = torch.arange(S, device="cuda")[:, None], torch.arange(S, device="cuda")
    return (j <= t) & ((j > t - window) | (j < sinks)) & (j < n)


def attend(q, k, v, seen, scale=None):
    """As generation.attend, for rows that see different keys: q [R,D], k and v [n,D], seen [R,n].  What is hidden from all rows may be
    anything; hidden values are replaced before the products."""
    q, k, v = q.double(), k.double(), v.double()
    some = seen.any(0)
    k, v = (torch.where(some[:, None], x, torch.zeros_like(x)) for x in (k, v))
    n, D = int(seen.sum(-1).max()), k.shape[1]
    scale = D ** -0.5 if scale is None else scale
    s = (q @ k.t().contiguous() * scale).masked_fill(~seen, -float("inf"))
    p = torch.nan_to_num(torch.softmax(s, -1))
    size = (q.abs() @ k.abs().t().contiguous()).amax(-1, keepdim=True) * scale
    return p @ v, p @ v.abs(), (2 * (D + 8) * size + 2 * (n + 16) + 256) * 2.0 ** -24


def data(B, Hq, Hkv, S, D, dt, lens):
    g = torch.Generator(device="cuda").manual_seed(B + S + D)
    Q, K, V = (torch.randn(B, h, S, D, generator=g, device="cuda").to(DT[dt]) for h in (Hq, Hkv, Hkv))
    if lens is not None:
        for b, n in enumerate(lens):
            K[b, :, max(n, 0):] = V[b, :, max(n, 0):] = float("nan")
        lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    return Q, K, V, lens


def call(ac, Q, K, V, lens, window, sinks, sel=None, **kw):  # noqa: F811
    room = torch.full((Q.shape[0] + 1, *Q.shape[1:]), 7.0, dtype=Q.dtype, device="cuda")
    ac.attention_window(Q, K, V, room[:-1], window=window, sinks=sinks, key_len=lens, row_sel=sel, **kw)
    assert (room[-1] == 7.0).all()
    return room[:-1]


def check(O, Q, K, V, lens, window, sinks, heads, scale=None):
    S = Q.shape[2]
    g = Q.shape[1] // K.shape[1]
    for b, h in heads:
        n = S if lens is None else min(max(int(lens[b]), 0), S)
        gen.check(O[b, h], *attend(Q[b, h], K[b, h // g], V[b, h // g], seen_by(S, n, window, sinks), scale))


def some_heads(B, Hq, most=12):
    every = [(b, h) for b in range(B) for h in range(Hq)]
    return every if len(every) <= most else random.Random(B * Hq).sample(every, most - 2) + [(0, 0), (B - 1, Hq - 1)]


# B, Hq, Hkv, S: one token, block borders and beside them, heads alone and many on a K and V
SIZES = [(1, 1, 1, 1), (2, 4, 2, 2), (3, 3, 1, 15), (2, 6, 2, 17), (1, 5, 1, 31), (2, 4, 4, 32), (2, 8, 1, 33), (9, 3, 3, 64), (2, 7, 1, 65), (4, 12, 12, 96),
         (2, 8, 2, 127), (1, 40, 2, 130), (17, 4, 2, 200), (1, 2, 2, 513), (1, 8, 2, 1100)]
TYPES = [(64, "bf16"), (128, "bf16"), (64, "f32"), (128, "f32"), (3, "f32"), (33, "f32"), (36, "f32"), (80, "f32"), (101, "f32"), (199, "f32"), (200, "f32"), (256, "f32")]
MANY = [(33, 12, 4, 100), (20, 24, 2, 50)]      # (binary32: more than 256 workgroups of 64 rows)
WINDOWS = [(1, 0), (1, 1), (7, 3), (32, 0), (33, 70), (64, 4), (100, 16), (300, 64), (10 ** 9, 0), (5, 10 ** 9), (2 ** 31 - 1, 2 ** 31 - 1)]


@pytest.mark.parametrize("D,dt", TYPES)
@pytest.mark.parametrize("size", MANY, ids=str)
def test_many_items(ac, size, D, dt):  # noqa: F811
    B, Hq, Hkv, S = size
    lens = [(S, 1, 0, (S + 1) // 2, S - 1, min(S, 40))[b % 6] for b in range(B)]
    Q, K, V, lens = data(*size, D, dt, lens)
    O = call(ac, Q, K, V, lens, 20, 5)
    assert O.isfinite().all()
    check(O, Q, K, V, lens, 20, 5, some_heads(B, Hq, 12))


@pytest.mark.parametrize("D,dt", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sizes(ac, size, D, dt):  # noqa: F811
    B, Hq, Hkv, S = size
    for i, (window, sinks) in enumerate([(7, 3), (64, 4), (100, 65)] if S < 300 else [(130, 4)]):
        lens = [(S, 1, 0, (S + 1) // 2, S - 1, min(S, 40))[b % 6] for b in range(B)] if i != 1 else None
        Q, K, V, lens = data(*size, D, dt, lens)
        O = call(ac, Q, K, V, lens, window, sinks)
        assert O.isfinite().all()
        check(O, Q, K, V, lens, window, sinks, some_heads(B, Hq, 6))


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("size", [(2, 4, 2, 200), (1, 6, 1, 301), (3, 2, 2, 97)], ids=str)
@pytest.mark.parametrize("D,dt", [(64, "bf16"), (128, "bf16"), (128, "f32"), (50, "f32")])
def test_windows(ac, size, window, sinks, D, dt):  # noqa: F811
    B, Hq, _, S = size
    for lens in (None, [(S // 3, S, 2)[b % 3] for b in range(B)]):
        Q, K, V, n = data(*size, D, dt, lens)
        check(call(ac, Q, K, V, n, window, sinks), Q, K, V, n, window, sinks, some_heads(B, Hq))


@pytest.mark.parametrize("seed", range(20))
def test_drawn(ac, seed):  # noqa: F811
    rng = random.Random(seed)
    Hkv = rng.choice([1, 2, 3, 8])
    Hq, B, S = Hkv * rng.choice([1, 2, 3, 4, 5, 8]), rng.choice([1, 2, 5]), rng.randint(1, 700)
    D, dt = rng.choice([(64, "bf16"), (128, "bf16"), (64, "f32"), (100, "f32"), (128, "f32")])
    window, sinks = rng.choice([1, rng.randint(1, 50), rng.randint(1, S + 5)]), rng.choice([0, 1, 4, rng.randint(0, S), 33])
    lens = [rng.choice([S, rng.randint(0, S)]) for _ in range(B)] if rng.random() < 0.6 else None
    Q, K, V, lens = data(B, Hq, Hkv, S, D, dt, lens)
    O = call(ac, Q, K, V, lens, window, sinks)
    assert O.isfinite().all()
    check(O, Q, K, V, lens, window, sinks, some_heads(B, Hq))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_items_that_are_left_out_and_none_at_all(ac, dt):  # noqa: F811
    B, S = 9, 75
    Q, K, V, _ = data(B, 4, 2, S, 64, dt, None)
    sel = torch.tensor([-1 if b % 4 else b for b in range(B)], dtype=torch.int32, device="cuda")
    O = call(ac, Q, K, V, None, 20, 4, sel)
    assert (O[sel >= 0] == 7.0).all()
    check(O, Q, K, V, None, 20, 4, [(b, 3) for b in range(B) if b % 4])
    sel.fill_(0)
    assert (call(ac, Q, K, V, None, 20, 4, sel) == 7.0).all()
    ac.attention_window(Q[:0], K[:0], V[:0], Q[:0].clone(), window=3)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_lengths_out_of_range_scale_and_large_scores(ac, dt):  # noqa: F811
    B, S = 3, 150
    Q, K, V, _ = data(B, 4, 2, S, 128, dt, None)
    Q *= 30
    lens = torch.tensor([9999, -4, S], dtype=torch.int32, device="cuda")
    check(call(ac, Q, K, V, lens, 60, 3, scale=0.3), Q, K, V, lens, 60, 3, some_heads(B, 4), scale=0.3)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("D,dt", [(64, "bf16"), (128, "bf16"), (64, "f32"), (33, "f32")])
def test_a_hidden_key_touches_no_row(ac, D, dt, value):  # noqa: F811
    """K and V of some keys are not finite: rows that see none of them are as if they were zeros, the others not a number (or infinite)."""
    S, window, sinks, odd = 300, 40, 3, (70, 131, 299)
    Q, K, V, _ = data(1, 4, 2, S, D, dt, None)
    Kz, Vz = K.clone(), V.clone()
    for j in odd:
        K[:, :, j] = V[:, :, j] = value
        Kz[:, :, j] = Vz[:, :, j] = 0
    O = call(ac, Q, K, V, None, window, sinks)
    t = torch.arange(S, device="cuda")
    meets = torch.zeros(S, dtype=torch.bool, device="cuda")
    for j in odd:
        meets |= (t >= j) & (t < j + window)
    seen = seen_by(S, S, window, sinks)
    for h in range(4):
        want, terms, bound = attend(Q[0, h], Kz[0, h // 2], Vz[0, h // 2], seen)
        gen.check(O[0, h][~meets], want[~meets], terms[~meets], bound[~meets])
    if value != value:
        assert O[0][:, meets].isnan().all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_an_infinite_value_that_is_seen(ac, dt):  # noqa: F811
    S, window = 100, 20
    Q, K, V, _ = data(1, 2, 1, S, 64, dt, None)
    V[0, 0, 50, 7] = float("inf")
    O = call(ac, Q, K, V, None, window, 0)
    t = torch.arange(S, device="cuda")
    meets = (t >= 50) & (t < 50 + window)
    assert (O[0][:, meets, 7] == float("inf")).all()
    rest = O[0].clone()
    rest[:, meets, 7] = 0
    assert rest.isfinite().all()
    V[0, 0, 50, 7] = 0
    for h in range(2):
        w = attend(Q[0, h], K[0, 0], V[0, 0], seen_by(S, S, window, 0))
        keep = torch.ones(S, 64, dtype=torch.bool, device="cuda")
        keep[meets, 7] = False
        gen.check(torch.where(keep, O[0, h].double(), w[0]).to(torch.float64 if dt == "f32" else O.dtype) if dt == "f32" else
                  torch.where(keep, O[0, h], w[0].to(O.dtype)), *w)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_scores_of_minus_infinity_and_the_lowest_value(ac, dt):  # noqa: F811
    S = 130
    Q, K, V, _ = data(1, 2, 1, S, 64, dt, None)
    Q.abs_()
    K[0, :, 5], K[0, :, 64:96] = torch.finfo(DT[dt]).min, -float("inf")
    O = call(ac, Q, K, V, None, 200, 0)
    seen = seen_by(S, S, 200, 0)
    seen[:, 5] = False
    seen[:, 64:96] = False
    K[0, :, 5] = K[0, :, 64:96] = 0
    rows = torch.arange(S, device="cuda") != -1
    for h in range(2):
        w = attend(Q[0, h], K[0, 0], V[0, 0], seen)
        gen.check(O[0, h][rows], *(x[rows] for x in w))


@pytest.mark.parametrize("D,dt", [(64, "bf16"), (128, "bf16"), (128, "f32")])
def test_a_window_over_everything_is_causal_attention(ac, D, dt):  # noqa: F811
    Q, K, V, _ = data(4, 8, 2, 256, D, dt, None)
    O, E = call(ac, Q, K, V, None, 256, 0), torch.empty_like(Q)
    ac.attention_exact(Q, K, V, E, causal=True)
    seen = seen_by(256, 256, 256, 0)
    for b, h in some_heads(4, 8, 4):      # both are within the same distance of the definition
        for o in (O, E):
            gen.check(o[b, h], *attend(Q[b, h], K[b, h // 4], V[b, h // 4], seen))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_every_key_in_the_window_counts_once(ac, dt):  # noqa: F811
    """Q is zero: a result is the mean of the seen V, whose marked column of each group of keys tells which were seen."""
    S, window, sinks, D = 1500, 400, 40, 64
    Q = torch.zeros(1, 2, S, D, dtype=DT[dt], device="cuda")
    K = torch.randn(1, 2, S, D, device="cuda").to(DT[dt])
    V = torch.nn.functional.one_hot((torch.arange(S, device="cuda") // 8) % D, D).to(DT[dt]).expand(1, 2, S, D).contiguous()
    O = call(ac, Q, K, V, None, window, sinks)
    seen = seen_by(S, S, window, sinks).double()
    want = seen @ V[0, 0].double() / seen.sum(-1, keepdim=True)
    tol = ((2.0 ** -8 if dt == "bf16" else 0) + 6 * 2.0 ** -24) * want     # whole numbers, a division, a product, a rounding
    assert ((O[0].double() - want).abs() <= tol).all()


def test_a_captured_call_another_stream_and_the_same_result_every_time(ac):  # noqa: F811
    for dt in ("bf16", "f32"):
        Q, K, V, _ = data(3, 4, 2, 333, 64, dt, None)
        want = call(ac, Q, K, V, None, 100, 4).clone()
        O = torch.zeros_like(Q)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ac.attention_window(Q, K, V, O, window=100, sinks=4)
        for _ in range(4):
            O.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(O, want)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        O.zero_()
        s.wait_stream(torch.cuda.current_stream())
        ac.attention_window(Q, K, V, O, window=100, sinks=4, stream=s)
        s.synchronize()
        assert torch.equal(O, want)
