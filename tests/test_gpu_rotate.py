"""Heads from a projection's rows, normalised and rotated, against 64 bits.  Padding holds NaN, places that nothing goes to are looked at."""
import math

import pytest
import torch

from tests.test_gpu_parity_small import ac  # noqa: F401

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def expect(X, pos, freq, Hq, Hkv, D, qw, kw, eps, amp, interleaved):
    """[B,H,S,D] in 64 bits and how far a result may be from it: the norm's sum of D squares (half of its roundings after the root) and
    a few roundings beside it, and a rotation whose sine and cosine are off by 2^-22, whose angle, up to half a turn in binary32, is off
    by pi 2^-24 and by 2^-51 of itself as the product is formed; both halves of a pair count."""
    B, S, _ = X.shape
    x = X.double().view(B, S, Hq + 2 * Hkv, D).transpose(1, 2)
    rot = 0 if freq is None else 2 * freq.numel()
    far = 0.0
    out, size = x.clone(), x.abs()
    for lo, hi, w in ((0, Hq, qw), (Hq, Hq + Hkv, kw)):
        y = x[:, lo:hi]
        if w is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
        z, s = y.clone(), y.abs()
        if rot:
            t = pos.double()[:, None, :, None] * freq
            far = t.abs().max().item() * 2.0 ** -51
            c, n = torch.cos(t) * amp, torch.sin(t) * amp
            a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
            z[..., a], z[..., b] = y[..., a] * c - y[..., b] * n, y[..., b] * c + y[..., a] * n
            s[..., a] = s[..., b] = (y[..., a].abs() + y[..., b].abs()) * abs(amp)
        out[:, lo:hi], size[:, lo:hi] = z, s
    tol = size * ((D / 2 + 8 + 4 + 4 + 4) * 2.0 ** -24 + far) + 1e-37
    tol[:, Hq + Hkv:] = 0
    if X.dtype == torch.bfloat16:
        tol[:, :Hq + Hkv] += 2.0 ** -8 * out[:, :Hq + Hkv].abs()
    return out, tol


def near(got, want, tol, real):
    m = real.expand_as(got)
    bad = m & ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), (got.double() - want)[bad][:4].tolist(), bad.nonzero()[:3].tolist())


def case(ac, B, S, Hq, Hkv, D, dt, rot, *, interleaved=False, norm=True, dense=True, page=0, base=10000.0, seed=0, far=0, pads=True,  # noqa: F811
         extra=0, amp=1.0, apart=0):
    g = torch.Generator(device="cuda").manual_seed(seed + B + S)
    width = (Hq + 2 * Hkv) * D
    room = torch.randn(B, S, width + extra, generator=g, device="cuda").to(DT[dt])
    X = room[:, :, extra // 2:extra // 2 + width] if extra else room
    lens = [(S if b % 3 == 0 else b * 7 % (S + 1)) if pads else S for b in range(B)]
    pos = torch.tensor([[far + 3 * t + b if t < lens[b] else -1 - t for t in range(S)] for b in range(B)], dtype=torch.int32, device="cuda")
    real = (pos >= 0)[:, None, :, None]
    X[pos < 0] = float("nan")
    freq = ac.attncache_rotary_frequencies(rot, base=base).cuda() if rot else None
    qw, kw = (1 + 0.3 * torch.randn(D, generator=g, device="cuda") for _ in range(2)) if norm else (None, None)
    Q = torch.full((B, Hq, S, D), 7.0, dtype=DT[dt], device="cuda")
    K, V = (torch.full((B, Hkv, S, D), 7.0, dtype=DT[dt], device="cuda") if dense else None for _ in range(2))
    kw_pages = {}
    if page:
        n = (B * S) // page + 4
        size = Hkv * page * D + apart
        k, v = (torch.full((n, size), 5.0, dtype=DT[dt], device="cuda").as_strided((n, Hkv, page, D), (size, page * D, D, 1)) for _ in range(2))
        slot = torch.randperm(n * page, generator=g, device="cuda")[:B * S].view(B, S).int()
        slot[0, S // 2] = -1 if B % 2 else n * page      # not written, whatever the row
        kw_pages = dict(slot=slot, k_pages=k, v_pages=v)
    ac.attncache_rotate(X, pos, freq, Q, K, V, q_weight=qw, k_weight=kw, eps=1e-5, amplitude=amp, interleaved=interleaved, **kw_pages)
    want, tol = expect(torch.nan_to_num(X), pos.clamp(min=0), freq, Hq, Hkv, D, qw, kw, 1e-5, amp, interleaved)
    parts = {"Q": (0, Hq), "K": (Hq, Hq + Hkv), "V": (Hq + Hkv, Hq + 2 * Hkv)}
    for name, t in (("Q", Q), ("K", K), ("V", V)):
        if t is not None:
            near(t, want[:, slice(*parts[name])], tol[:, slice(*parts[name])], real)
            assert (t[~real.expand_as(t)] == 7).all()
    if page:
        ok = (pos >= 0) & (slot >= 0) & (slot < n * page)
        at = slot[ok].long()
        for name, pages in (("K", k), ("V", v)):
            w, tl = (x[:, slice(*parts[name])].transpose(1, 2)[ok] for x in (want, tol))      # [rows,Hkv,D]
            near(pages[at // page, :, at % page], w, tl, torch.ones(1, 1, 1, dtype=torch.bool, device="cuda"))
            pages[at // page, :, at % page] = 5
            assert (pages.as_strided((n, size), (size, 1)) == 5).all()


SIZES = [(1, 1, 1, 1, 64, "bf16", 64), (128, 1, 32, 8, 128, "bf16", 128), (3, 7, 5, 1, 128, "bf16", 64), (4, 33, 12, 12, 64, "bf16", 32),
         (2, 300, 8, 2, 128, "bf16", 128), (5, 9, 3, 3, 64, "bf16", 20), (5, 9, 3, 3, 128, "bf16", 2), (2, 5, 4, 2, 64, "bf16", 0),
         (3, 7, 5, 1, 80, "f32", 40), (2, 94, 24, 8, 128, "f32", 128), (2, 5, 2, 2, 33, "f32", 32), (2, 5, 2, 1, 199, "f32", 198),
         (2, 5, 2, 1, 256, "f32", 256), (1, 3, 1, 1, 1, "f32", 0), (4, 3, 2, 1, 2, "f32", 2), (2, 6, 3, 1, 100, "f32", 50), (2, 6, 3, 1, 64, "f32", 8),
         (2, 6, 3, 1, 200, "f32", 64), (1, 2, 40, 1, 64, "bf16", 64), (3, 2, 1, 1, 128, "f32", 6),
         (2, 6, 3, 1, 36, "f32", 10), (2, 6, 3, 1, 200, "f32", 30), (2, 40, 6, 2, 128, "bf16", 94), (2, 40, 6, 2, 64, "bf16", 62), (2, 9, 3, 1, 64, "f32", 62), (2, 6, 3, 1, 101, "f32", 100)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(map(str, s)))
def test_sizes(ac, size, norm, interleaved):  # noqa: F811
    case(ac, *size, norm=norm, interleaved=interleaved, page=16, seed=1)


@pytest.mark.parametrize("page,apart", [(1, 0), (7, 0), (16, 64), (128, 8)])
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_pages_alone_and_beside_dense_heads(ac, dt, dense, page, apart):  # noqa: F811
    case(ac, 5, 21, 6, 2, 64, dt, 64, dense=dense, page=page, apart=apart)
    case(ac, 9, 1, 6, 2, 64, dt, 64, dense=dense, page=page, apart=apart)


@pytest.mark.parametrize("dt,extra", [("bf16", 16), ("f32", 8)])
def test_rows_of_a_wider_product(ac, dt, extra):  # noqa: F811
    case(ac, 4, 13, 4, 2, 128, dt, 128, extra=extra)
    case(ac, 1, 13, 4, 2, 64, dt, 64, extra=extra)
    case(ac, 6, 1, 4, 2, 64, dt, 64, extra=extra)


def test_rows_of_items_in_another_order(ac):  # noqa: F811
    """[S,B,...]: the items' stride is smaller than the rows'."""
    B, S, H, D = 3, 5, 2, 64
    X = torch.randn(S, B, (H + 2) * D, device="cuda").bfloat16().transpose(0, 1)
    pos = torch.arange(S, device="cuda").int().expand(B, S).contiguous()
    freq = ac.attncache_rotary_frequencies(D).cuda()
    out = [[torch.empty(B, h, S, D, dtype=torch.bfloat16, device="cuda") for h in (H, 1, 1)] for _ in range(2)]
    ac.attncache_rotate(X, pos, freq, *out[0])
    ac.attncache_rotate(X.contiguous(), pos, freq, *out[1])
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("far", [10 ** 5, 10 ** 7, 2 ** 31 - 200])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_far_positions(ac, dt, far):  # noqa: F811
    case(ac, 2, 9, 2, 1, 64, dt, 64, far=far, pads=False)
    case(ac, 2, 9, 2, 1, 64, dt, 64, far=far, pads=False, base=500000.0, amp=1.25, norm=False)


def test_many_tokens(ac):  # noqa: F811
    case(ac, 40, 1000, 4, 2, 64, "bf16", 64, page=16)
    case(ac, 5000, 1, 2, 1, 128, "bf16", 128, page=16, pads=False)


def test_more_rows_than_31_bits_count(ac):  # noqa: F811
    B, Hq = 1 << 20, 2049
    X = torch.randn(B, 1, Hq + 2, device="cuda")
    Q, K, V = torch.zeros(B, Hq, 1, 1, device="cuda"), torch.zeros(B, 1, 1, 1, device="cuda"), torch.zeros(B, 1, 1, 1, device="cuda")
    ac.attncache_rotate(X, torch.zeros(B, 1, dtype=torch.int32, device="cuda"), None, Q, K, V)
    for b in (0, (1 << 19) - 50, B - 600):      # one number a head, nothing to normalise or rotate
        assert torch.equal(Q[b:b + 600].view(-1, Hq), X[b:b + 600, 0, :Hq])
    assert torch.equal(K.view(B), X[:, 0, Hq]) and torch.equal(V.view(B), X[:, 0, Hq + 1])


def test_an_infinity_stays_in_its_head_and_nothing_to_do_is_done(ac):  # noqa: F811
    B, S, D = 2, 3, 64
    X = torch.randn(B, S, 4 * D, device="cuda")
    clean, freq = X.clone(), ac.attncache_rotary_frequencies(D).cuda()
    X[1, 1, D + 3], X[0, 2, 3 * D] = float("inf"), float("nan")
    pos = torch.arange(S, device="cuda").int().expand(B, S).contiguous()
    w = torch.ones(D, device="cuda")
    out = [[torch.empty(B, h, S, D, device="cuda") for h in (2, 1, 1)] for _ in range(2)]
    for x, o in ((X, out[0]), (clean, out[1])):
        ac.attncache_rotate(x, pos, freq, *o, q_weight=w, k_weight=w)
    same = [a == b for a, b in zip(*out)]
    assert not same[0][1, 1, 1].any() and not same[2][0, 0, 2, 0]
    same[0][1, 1, 1], same[2][0, 0, 2, 0] = True, True
    assert all(s.all() for s in same)
    none = torch.empty(0, S, 4 * D, device="cuda")
    ac.attncache_rotate(none, pos[:0], freq, *(torch.empty(0, h, S, D, device="cuda") for h in (2, 1, 1)))


def test_a_captured_call_follows_its_inputs(ac):  # noqa: F811
    B, S, D = 3, 4, 64
    X = torch.randn(B, S, 4 * D, device="cuda").bfloat16()
    pos = torch.arange(S, device="cuda").int().expand(B, S).contiguous()
    freq = ac.attncache_rotary_frequencies(D).cuda()
    out, want = ([torch.zeros(B, h, S, D, dtype=torch.bfloat16, device="cuda") for h in (2, 1, 1)] for _ in range(2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ac.attncache_rotate(X, pos, freq, *out)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ac.attncache_rotate(X, pos, freq, *out)
    for i in range(4):
        X.copy_(torch.randn(B, S, 4 * D, device="cuda"))
        pos += i
        graph.replay()
        ac.attncache_rotate(X, pos, freq, *want)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_frequencies_are_those_of_the_formula(ac):  # noqa: F811
    for rot in (2, 64, 128):
        f = ac.attncache_rotary_frequencies(rot, base=10000.0)
        assert f.tolist() == pytest.approx([10000.0 ** (-2 * i / rot) for i in range(rot // 2)], rel=1e-14)
        assert math.isclose(f[0], 1.0)
