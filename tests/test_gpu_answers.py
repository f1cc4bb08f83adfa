"""Several answers to one prompt, from the projection's product to the attention of each new token, as a program runs them: heads rotated, a prompt's
attention, rows into pages, the row forked, then steps of all answers of which some end; every token is compared with plain attention in 64 bits."""
import pytest
import torch

from tests import generation as gen
from tests.test_gpu_parity_small import ac  # noqa: F401
from tests.test_gpu_shared_attention import width as wide
from tests.test_gpu_rotate import expect
from tests.test_gpu_window_attention import attend, seen_by

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 4)])
@pytest.mark.parametrize("dt,D,page", [("bf16", 64, 16), ("bf16", 128, 7), ("f32", 80, 10)])
def test_answers_to_one_prompt(ac, dt, D, page, window, sinks):  # noqa: F811
    B, S, Hq, Hkv, steps = 6, 45, 4, 2, 12
    width, n = -(-(S + steps) // page) + 1, 80
    g = torch.Generator(device="cuda").manual_seed(D)
    draw = lambda *s: torch.randn(*s, generator=g, device="cuda").to(DT[dt])  # noqa: E731
    empty = lambda *s: torch.empty(s, dtype=DT[dt], device="cuda")  # noqa: E731
    freq, qw, kw = ac.attncache_rotary_frequencies(D).cuda(), *(1 + 0.2 * torch.randn(D, generator=g, device="cuda") for _ in range(2))
    k, v = (torch.full((n, Hkv, page, D), float("nan"), dtype=DT[dt], device="cuda") for _ in range(2))
    table, seq, ring, state = i32([[-1] * width] * B), i32([0] * B), i32(list(range(n))), i32([0, n])
    added, same = i32([0] * B), i32(list(range(B)))
    ws_fork = torch.empty(ac.attncache_page_fork_workspace_bytes(B, width, n), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(ac.attention_paged_shared_workspace_bytes(B, Hq, Hkv, D, 1), ac.attention_paged_workspace_bytes(B, Hq, Hkv, D)), dtype=torch.uint8, device="cuda")

    # the prompt, of which row 0 holds the tokens
    slot = torch.zeros(B, S, dtype=torch.int32, device="cuda")
    ac.attncache_page_plan(seq, i32([S] + [0] * (B - 1)), state, ring, table, seq, added, state, slot, page_size=page)
    X, pos = draw(1, S, (Hq + 2 * Hkv) * D), torch.arange(S, device="cuda").int().view(1, S)
    Q, K, V = empty(1, Hq, S, D), empty(1, Hkv, S, D), empty(1, Hkv, S, D)
    ac.attncache_rotate(X, pos, freq, Q, K, V, q_weight=qw, k_weight=kw, slot=slot[:1].contiguous(), k_pages=k, v_pages=v)
    want, tol = expect(X, pos, freq, Hq, Hkv, D, qw, kw, 1e-6, 1.0, False)
    for t, lo, hi in ((Q, 0, Hq), (K, Hq, Hq + Hkv), (V, Hq + Hkv, Hq + 2 * Hkv)):
        assert ((t.double() - want[:, lo:hi]).abs() <= tol[:, lo:hi]).all()
    O = empty(1, Hq, S, D)
    ac.attention_window(Q, K, V, O, window=window or S, sinks=sinks)
    for h in range(Hq):
        gen.check(O[0, h], *attend(Q[0, h], K[0, h // 2], V[0, h // 2], seen_by(S, S, window or S, sinks)))
    past = [[(K[0, :, t], V[0, :, t]) for t in range(S)]] + [[] for _ in range(B - 1)]

    # all rows answer it; then some of them end, and others go on in their place
    for step in range(steps):
        source = [0] * B if step == 0 else [0, 1, 1, 3, -1, 5] if step == 5 else [3, 3, 0, 1, 2, -1] if step == 8 else list(range(B))
        ac.attncache_page_fork(i32(source), seq, state, ring, table, table, seq, state, k, v, ws_fork, window=window, sinks=sinks)
        past = [list(past[s]) if s >= 0 else [] for s in source]
        assert seq.tolist() == [len(p) for p in past]
        alive = [len(p) > 0 for p in past]
        pos = seq.view(B, 1).clone()
        pos[~torch.tensor(alive, device="cuda")] = -1
        slot = torch.zeros(B, 1, dtype=torch.int32, device="cuda")
        ac.attncache_page_plan(seq, i32([int(a) for a in alive]), state, ring, table, seq, added, state, slot, page_size=page)
        assert added.tolist() == [int(a) for a in alive]
        X, q = draw(B, 1, (Hq + 2 * Hkv) * D), torch.zeros(B, Hq, 1, D, dtype=DT[dt], device="cuda")
        ac.attncache_rotate(X, pos, freq, q, q_weight=qw, k_weight=kw, slot=slot, k_pages=k, v_pages=v)
        O = empty(B, Hq, D)
        if window:
            ac.attention_paged_window(q.view(B, Hq, D), k, v, table, seq, O, ws, window=window, sinks=sinks)
        else:
            long = torch.full((B, wide(B, Hkv, D, dt, page)), -1, dtype=torch.int32, device="cuda")      # of which a prefix is read once
            ac.attention_paged_shared(q.view(B, Hq, D), k, v, torch.cat([table, long], 1) if step % 2 else table, seq, i32([0, B]), i32([S]), O, ws)
        t, s = table.tolist(), seq.tolist()
        for b in range(B):
            if not alive[b]:
                assert s[b] == 0 and (O[b] == 0).all()
                continue
            j = s[b] - 1
            past[b].append((k[t[b][j // page], :, j % page].clone(), v[t[b][j // page], :, j % page].clone()))
            assert len(past[b]) == s[b]
            at = [x for x in range(s[b]) if not window or x >= s[b] - window or x < sinks]
            kk, vv = (torch.stack([past[b][x][i] for x in at], 1) for i in (0, 1))
            for h in range(Hkv):
                gen.check(O[b, 2 * h:2 * h + 2], *gen.attend(q[b, 2 * h:2 * h + 2, 0], kk[h], vv[h]))
    # every page is one row's or several rows', or free
    t, first, count = table.tolist(), *state.tolist()
    held = {q for b in range(B) for q in t[b][:-(-seq[b].item() // page)] if q >= 0}
    free = [ring[(first + i) % n].item() for i in range(count)]
    assert len(set(free)) == count and not held & set(free) and len(held) + count == n
