"""Attention to another sequence's states, against plain attention in 64 bits.  Padding behind the real states is NaN, as are the
workspace and, where nothing is to be written, the result."""
import pytest
import torch

from tests import generation as gen
from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _data(B, Hq, Hkv, Sq, Sk, D, dt, lens):
    g = torch.Generator(device="cuda").manual_seed(B + Sq + Sk + D)
    Q, K, V = (torch.randn(B, h, s, D, generator=g, device="cuda").to(DT[dt])
               for h, s in ((Hq, Sq), (Hkv, Sk), (Hkv, Sk)))
    if lens is not None:
        for b, n in enumerate(lens):
            K[b, :, max(n, 0):] = V[b, :, max(n, 0):] = float("nan")
        lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    return Q, K, V, lens


def _call(ac, Q, K, V, lens, sel=None, **kw):  # noqa: F811
    B, Hq, Sq, D = Q.shape
    room = torch.full((B + 1, Hq, Sq, D), 7.0, dtype=Q.dtype, device="cuda")
    need = ac.attention_cross_workspace_bytes(B, Hq, K.shape[1], Sq, K.shape[2], D, Q.dtype)
    ws = torch.full((need // 4,), float("nan"), device="cuda") if need else None
    ac.attention_cross(Q, K, V, room[:B], ws, key_len=lens, row_sel=sel, **kw)
    assert (room[B] == 7.0).all()
    return room[:B]


def _check(O, Q, K, V, lens, items, scale=None):
    B, Hq, Sq, D = Q.shape
    Hkv, Sk = K.shape[1:3]
    g = Hq // Hkv
    for b in items:
        n = Sk if lens is None else min(max(int(lens[b]), 0), Sk)
        for h in range(Hkv):
            q = Q[b, h * g:(h + 1) * g].reshape(-1, D)
            gen.check(O[b, h * g:(h + 1) * g].reshape(-1, D), *gen.attend(q, K[b, h, :n], V[b, h, :n], scale))


# B, Hq, Hkv, Sq, Sk: one row and many, one key and many, few and many heads on a K and V
SIZES = [(1, 1, 1, 1, 1), (3, 4, 2, 1, 50), (2, 6, 2, 5, 1), (5, 3, 3, 33, 65), (2, 8, 1, 9, 200), (1, 40, 1, 1, 700),
         (1, 2, 2, 100, 3001), (4, 12, 12, 1, 1000), (40, 4, 4, 64, 64), (33, 8, 4, 65, 127), (9, 16, 16, 129, 31), (70, 6, 2, 23, 130),
         (2, 64, 32, 260, 333), (130, 1, 1, 200, 97), (1, 1, 1, 1, 70001),
         (70, 8, 8, 33, 40), (130, 6, 3, 40, 70), (3, 40, 2, 1, 2500), (260, 4, 4, 33, 20), (20, 12, 12, 1, 100), (9, 16, 8, 111, 705),
         (400, 6, 3, 1, 1100)]
TYPES = [(64, "bf16"), (128, "bf16"), (64, "f32"), (128, "f32"), (3, "f32"), (33, "f32"), (36, "f32"), (80, "f32"), (101, "f32"), (199, "f32"), (256, "f32")]


@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("D,dt", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sizes(ac, size, D, dt, padded):  # noqa: F811
    B, Hq, Hkv, Sq, Sk = size
    lens = [(Sk, 1, 0, (Sk + 1) // 2, Sk - 1, min(Sk, 64), min(Sk, 32))[b % 7] for b in range(B)] if padded else None
    Q, K, V, lens = _data(*size, D, dt, lens)
    O = _call(ac, Q, K, V, lens)
    assert O.isfinite().all()
    _check(O, Q, K, V, lens, range(B) if B < 8 else sorted({0, 1, 2, 3, 5, B // 2, B - 2, B - 1}))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(6, 4, 2, 3, 90), (40, 8, 4, 70, 75)], ids=str)
def test_items_that_are_left_out(ac, size, dt):  # noqa: F811
    B, Sk = size[0], size[4]
    lens = [(Sk, 0, 7)[b % 3] for b in range(B)]
    Q, K, V, lens = _data(*size, 64, dt, lens)
    sel = torch.tensor([-1 if b % 4 else b for b in range(B)], dtype=torch.int32, device="cuda")
    O = _call(ac, Q, K, V, lens, sel)
    assert (O[sel >= 0] == 7.0).all()
    _check(O, Q, K, V, lens, [b for b in range(B) if b % 4])
    sel.fill_(0)
    assert (_call(ac, Q, K, V, lens, sel) == 7.0).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(3, 4, 2, 3, 90), (40, 8, 4, 70, 75)], ids=str)
def test_lengths_out_of_range_scale_and_large_scores(ac, size, dt):  # noqa: F811
    Q, K, V, _ = _data(*size, 128, dt, None)
    Q *= 30
    lens = torch.tensor([(9999, -4, size[4])[b % 3] for b in range(size[0])], dtype=torch.int32, device="cuda")
    O = _call(ac, Q, K, V, lens, scale=0.3)
    _check(O, Q, K, V, lens, range(0, size[0], 5), scale=0.3)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 2, 1, 2, 200), (64, 4, 4, 64, 130)], ids=str)
def test_infinite_and_lowest_keys(ac, size, dt):  # noqa: F811
    Q, K, V, _ = _data(*size, 64, dt, None)
    Q.abs_()
    K[0, :, 5], K[0, :, 129] = -float("inf"), torch.finfo(DT[dt]).min
    K[1, :, 70] = float("nan")
    O = _call(ac, Q, K, V, None)
    assert O[1].isnan().all()
    keep = [j for j in range(size[4]) if j not in (5, 129)]
    _check(O, Q, K[:, :, keep].contiguous(), V[:, :, keep].contiguous(), None, [0])


@pytest.mark.parametrize("D,dt", [(64, "bf16"), (128, "bf16")])
def test_both_ways_agree_with_exact_attention(ac, D, dt):  # noqa: F811
    """The same Q, K and V, of one length, through attention_exact without a mask."""
    Q, K, V, _ = _data(8, 32, 8, 128, 128, D, dt, None)
    O, E = _call(ac, Q, K, V, None), torch.empty_like(Q)
    ac.attention_exact(Q, K, V, E, causal=False)
    assert (O.float() - E.float()).abs().max() <= 2.0 ** -8 * 4 * 1.5     # (two results of |o| < 1.5, each off by at most 2^-8 (2 |o| + terms))


def test_a_captured_call_and_the_same_result_every_time(ac):  # noqa: F811
    for size in ((3, 4, 2, 1, 900), (40, 8, 4, 70, 75)):
        Q, K, V, _ = _data(*size, 64, "bf16", None)
        want = _call(ac, Q, K, V, None).clone()
        O = torch.zeros_like(Q)
        ws = torch.zeros(max(16, ac.attention_cross_workspace_bytes(*size, 64, Q.dtype)), dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ac.attention_cross(Q, K, V, O, ws)
        for i in range(6):
            O.fill_(7.0)
            ac.attention_cross(Q, K, V, O, ws) if i == 3 else graph.replay()
            assert torch.equal(O, want)


def test_a_prompt_and_generated_tokens_to_one_encoder(ac):  # noqa: F811
    """A decoder's rows all at once and one by one give the same, whichever kernel serves them."""
    B, Hq, Hkv, Sq, Sk, D = 6, 8, 4, 70, 150, 64
    Q, K, V, lens = _data(B, Hq, Hkv, Sq, Sk, D, "bf16", [150, 1, 64, 0, 99, 33])
    _check(_call(ac, Q, K, V, lens), Q, K, V, lens, range(B))
    for t in (0, 33, 69):
        row = Q[:, :, t:t + 1].contiguous()
        _check(_call(ac, row, K, V, lens), row, K, V, lens, range(B))


def test_many_rows_behind_two_gibi_elements(ac):  # noqa: F811
    B, H, Sk, D = 34, 32, 16_000, 128                                       # 2.2e9 elements, 4.5 GB a tensor
    g = torch.Generator(device="cuda").manual_seed(1)
    K, V = (torch.zeros(B, H, Sk, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    for b in (0, B - 1):
        for t in (K, V):
            t[b] = torch.randn(H, Sk, D, generator=g, device="cuda").bfloat16()
    for Sq in (1, 64):
        Q = torch.randn(B, H, Sq, D, generator=g, device="cuda").bfloat16()
        O = _call(ac, Q, K, V, None)
        for b in (0, B - 1):
            for h in (0, H - 1):
                gen.check(O[b, h], *gen.attend(Q[b, h], K[b, h], V[b, h]))


@pytest.mark.parametrize("keys", [(700, 33, 1.0), (700, 33, 40.0), (700, 650, 300.0), (1500, 1400, 1e4)])
def test_scores_that_outgrow_the_first_keys(ac, keys):  # noqa: F811
    """Keys whose scores exceed those of the first ones by little, by a lot and beyond the range of the weights; and rows whose first
    keys are all -inf."""
    Sk, at, by = keys
    Q, K, V, _ = _data(20, 8, 4, 70, Sk, 128, "bf16", None)
    K[:, :, at] = (Q[:, ::2, 5] * by / 11.3).clamp(-1e6, 1e6)
    V[3] *= 1e30
    K[4, :, :40] = -float("inf")
    Q[4] = Q[4].abs()
    O = _call(ac, Q, K, V, None)
    _check(O, Q, K, V, None, [0, 3, 7, 19])
    _check(O, Q[:, :], K[:, :, 40:].contiguous(), V[:, :, 40:].contiguous(), None, [4])


@pytest.mark.parametrize("far", [0.0, 40.0])
def test_low_scores_behind_keys_that_nobody_sees(ac, far):  # noqa: F811
    """Rows whose first keys are all -inf, and whose other scores are so low that 2^score is zero."""
    Q, K, V, _ = _data(20, 8, 4, 70, 700, 128, "bf16", None)
    Q.abs_()
    K -= far
    K[::2, :, :40] = -float("inf")
    O = _call(ac, Q, K, V, None)
    _check(O, Q, K, V, None, [1, 19])
    _check(O, Q, K[:, :, 40:].contiguous(), V[:, :, 40:].contiguous(), None, [0, 18])
