"""Several answers to long prompts, as cases that can be timed and compared: a projection's rows split into rotated heads,
rows of a paged cache forked and given back, attention of a batch whose requests share long prefixes, and attention
within a sliding window with a few first tokens that stay visible, over prompts and over pages.

``listed()`` holds the cases that stand for the whole range, ``draw()`` makes more of it, ``prepare()`` makes what a
program has in hand before the call, ``run()`` is one pass: in plain torch, or through the public entry points where
``own`` is true.  ``exact()`` is the same result from the definition, in 64 bits.

A cache of n pages holds ``k_pages`` and ``v_pages`` [n][H][page][D]; row ``j`` of request ``b`` lies in page
``page_table[b][j // page]`` at offset ``j % page``.  Free pages wait in a ring, ``free_pages`` [n] with
``free_state`` = (first, number).
"""
import math
import random

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # One generated token of each request of an 8B-shaped layer: heads normalised and rotated, K and V to their pages.
        dict(name="rotate-step", kind="rotate", B=128, S=1, Hq=32, Hkv=8, D=128, rot=128, dt="bf16", lo=100, hi=8000,
             interleaved=False, norm=True, dense=False, page=16, scaling="none"),
        # Ragged prompts of a 1B-shaped layer: for the attention of the prefill and for the cache.
        dict(name="rotate-prompts", kind="rotate", B=32, S=1024, Hq=32, Hkv=8, D=64, rot=64, dt="bf16", lo=200, hi=1024,
             interleaved=False, norm=False, dense=True, page=16, scaling="ramp"),
        # Binary32, a head of odd size of which half is rotated, in pairs of neighbours, at far positions.
        dict(name="rotate-fp32", kind="rotate", B=16, S=94, Hq=24, Hkv=8, D=80, rot=40, dt="f32", lo=40, hi=94,
             interleaved=True, norm=True, dense=True, page=0, scaling="linear"),
        # Beams change places: eight requests of four beams, one layer's cache.
        dict(name="fork-beams", kind="fork", groups=8, width=4, H=8, D=128, dt="bf16", page=16, lo=300, hi=2000, fresh=False,
             ended=2, window=0, sinks=0, short=False, spare=100),
        # Sixteen answers begin at each of eight prompts, all layers of a 1B-shaped model folded into the heads.
        dict(name="fork-answers", kind="fork", groups=8, width=16, H=128, D=64, dt="bf16", page=64, lo=500, hi=2000,
             fresh=True, ended=0, window=0, sinks=0, short=False, spare=40),
        # 64 answers to one long document.
        dict(name="shared-answers", kind="shared", groups=1, width=64, alone=0, Hq=32, Hkv=8, D=128, dt="bf16", page=16,
             plo=16000, phi=16000, lo=1, hi=500, short=0),
        # Requests that share one of sixteen instructions, and a few that share nothing.
        dict(name="shared-groups", kind="shared", groups=16, width=8, alone=6, Hq=32, Hkv=8, D=64, dt="bf16", page=16,
             plo=500, phi=4000, lo=20, hi=1000, short=2),
        # Binary32, three query heads on one K and V, few answers to prompts of odd length.
        dict(name="shared-fp32", kind="shared", groups=4, width=4, alone=1, Hq=24, Hkv=8, D=128, dt="f32", page=10,
             plo=300, phi=1500, lo=1, hi=100, short=0),
        # Long prompts through a layer with a window.
        dict(name="window-prompts", kind="window", B=4, Hq=32, Hkv=8, S=4096, D=128, dt="bf16", window=1024, sinks=4,
             lo=4096, hi=4096, skipped=0),
        # Binary32, ragged, a short window.
        dict(name="window-fp32", kind="window", B=16, Hq=24, Hkv=8, S=333, D=128, dt="f32", window=100, sinks=4, lo=50,
             hi=333, skipped=0),
        # A generated token of each request of a layer with a window; pages between the first tokens and the window are gone.
        dict(name="window-step", kind="window_step", B=128, Hq=32, Hkv=8, D=128, dt="bf16", page=16, window=4096, sinks=4,
             lo=1000, hi=200000),
        # A few requests with a short window: latency counts.
        dict(name="window-few", kind="window_step", B=4, Hq=32, Hkv=8, D=64, dt="bf16", page=16, window=500, sinks=16, lo=100,
             hi=9000),
    ]


# ------------------------------------------------------------------------------- drawn cases
_MAX_BYTES = 2.0e9       # one pass
_MAX_STATE = 5.0e9       # what a state holds
_MAX_GATHER = 4.0e9      # what a plain form gathers, elements
_MAX_SCORES = 2.2e9      # rows times keys of a window over prompts, all heads
_MAX_FLOPS_F32 = 8.0e9


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _state(case):
    """(elements of a state, elements that a plain form gathers, scores of one) at the most."""
    kind = case["kind"]
    if kind == "rotate":
        n = case["B"] * case["S"] * (case["Hq"] + 2 * case["Hkv"]) * case["D"]
        return 3 * n, n, 0
    if kind == "fork":
        pages = _fork_pages(case)
        n = 2 * case["H"] * case["page"] * case["D"]
        return pages * n, case["groups"] * case["width"] * n, 0
    row = 2 * case["Hkv"] * case["D"]
    if kind == "shared":
        rows = case["groups"] * case["width"] + case["alone"]
        each = case["phi"] + case["hi"] + case["page"]
        return row * (case["groups"] * (case["phi"] + case["page"]) + rows * (case["hi"] + 2 * case["page"])), row * rows * each, 0
    if kind == "window":
        S = case["S"]
        return row * case["B"] * S, row * case["B"] * S, case["B"] * case["Hq"] * S * S
    n = row * case["B"] * (case["window"] + case["sinks"] + 2 * case["page"])
    return n, n, 0


def _fit(case):
    """Halve the batch, then the lengths, until a pass and its state fit the limits above."""
    while True:
        w = work(case)
        state, gather, scores = _state(case)
        if (w["bytes"] <= _MAX_BYTES and state * _SIZE[case["dt"]] <= _MAX_STATE and gather <= _MAX_GATHER and
                scores <= _MAX_SCORES and (case["dt"] != "f32" or w["flops"] <= _MAX_FLOPS_F32)):
            return case
        for name in ("B", "groups", "width", "S", "phi", "window", "hi", "spare", "H"):
            if case.get(name, 1) > 1:
                case[name] //= 2
                break
        for low, high in (("lo", "hi"), ("plo", "phi")):
            if high in case:
                if case["kind"] in ("rotate", "window") and (case["S"] > 1 or case["kind"] == "window"):
                    case["hi"] = min(case["hi"], case["S"])
                case[low] = min(case[low], case[high])
        if case["kind"] == "fork":
            case["ended"] = min(case["ended"], case["groups"] * case["width"] // 2)
        if "skipped" in case:
            case["skipped"] = min(case["skipped"], case["B"] // 2)


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "fork", "fork", "shared", "shared", "shared", "window", "window", "window_step",
                       "window_step"])
    page = rng.choice([1, 8, 10, 16, 16, 16, 32, 48, 64, 128])
    f32 = rng.random() < 0.25
    dt = "f32" if f32 else "bf16"
    D = rng.choice([32, 64, 80, 100, 128, 199, 256]) if f32 else rng.choice([64, 128])
    hkv = rng.choice([1, 2, 4, 8, 12])
    g = rng.choice([1, 1, 2, 3, 4, 8])
    heads = dict(Hq=hkv * g, Hkv=hkv, D=D, dt=dt)
    if kind == "rotate":
        S = rng.choice([1, 1, _log_int(rng, 1, 2048)])
        hi = S if S > 1 else _log_int(rng, 1, 200000)
        rot = rng.choice([D - D % 2, D - D % 2, D // 4 * 2, max(2, rng.randrange(D // 2 + 1) * 2)])
        dense = rng.random() < 0.6
        return _fit(dict(kind=kind, B=_log_int(rng, 1, 256), S=S, **heads, rot=rot, lo=_log_int(rng, 1, hi), hi=hi,
                         interleaved=rng.random() < 0.4, norm=rng.random() < 0.5, dense=dense,
                         page=page if not dense or rng.random() < 0.6 else 0,
                         scaling=rng.choice(["none", "none", "linear", "base", "ramp"])))
    if kind == "fork":
        hi = _log_int(rng, 4, 8000)
        window = rng.choice([0, 0, 0, _log_int(rng, 1, hi)])
        groups, width = _log_int(rng, 1, 64), rng.choice([1, 2, 4, 5, 8, 16])
        return _fit(dict(kind=kind, groups=groups, width=width, H=hkv * rng.choice([1, 1, 4, 16]), D=D, dt=dt, page=page,
                         lo=_log_int(rng, 1, hi), hi=hi, fresh=rng.random() < 0.4, ended=rng.randrange(groups * width // 2 + 1),
                         window=window, sinks=rng.choice([0, 1, 4, 20]) if window else 0, short=rng.random() < 0.2,
                         spare=rng.choice([1, 30, 200])))
    if kind == "shared":
        phi, hi = _log_int(rng, 1, 30000), _log_int(rng, 1, 3000)
        return _fit(dict(kind=kind, groups=_log_int(rng, 1, 32), width=_log_int(rng, 1, 64), alone=rng.choice([0, 0, 1, 9]),
                         **heads, page=page, plo=_log_int(rng, 1, phi), phi=phi, lo=_log_int(rng, 1, hi), hi=hi,
                         short=rng.choice([0, 0, 1, 3])))
    sinks = rng.choice([0, 1, 4, 4, 16, 100])
    if kind == "window":
        S = _log_int(rng, 1, 8192 if not f32 else 1500)
        c = dict(kind=kind, B=_log_int(rng, 1, 32), **heads, S=S, window=_log_int(rng, 1, max(1, 2 * S // 3) + 10),
                 sinks=sinks, lo=_log_int(rng, 1, S), hi=S, skipped=0)
        c["skipped"] = rng.choice([0, 0, c["B"] // 2])
        return _fit(c)
    hi = _log_int(rng, 1, 300000)
    return _fit(dict(kind=kind, B=_log_int(rng, 1, 256), **heads, page=page, window=_log_int(rng, 1, 8000), sinks=sinks,
                     lo=_log_int(rng, 1, hi), hi=hi))


# ------------------------------------------------------------------------------- sizes
def _spread(n, lo, hi):
    """n lengths spread over [lo, hi] by their logarithm; the seed only says which request has which."""
    return [max(lo, min(hi, int(round(math.exp(math.log(lo) + (i + 0.5) / n * (math.log(hi) - math.log(lo)))))))
            for i in range(n)]


def _fork_pages(case):
    held = [-(-n // case["page"]) for n in _spread(case["groups"], case["lo"], case["hi"])]
    return sum(h + 3 * case["width"] for h in held) + case["spare"] + 1


def _visible(case, n):
    return min(n, case["window"] + min(case["sinks"], max(0, n - case["window"])))


def work(case):
    kind, size = case["kind"], _SIZE[case["dt"]]
    if kind == "rotate":
        B, S, D, Hq, Hkv = (case[x] for x in ("B", "S", "D", "Hq", "Hkv"))
        rows = sum(_spread(B, case["lo"], case["hi"])) if S > 1 else B
        times = case["dense"] + (case["page"] > 0)
        bytes_ = size * rows * D * ((Hq + 2 * Hkv) + Hq + 2 * Hkv * times) + 4.0 * B * S * (1 + (case["page"] > 0)) + 4.0 * case["rot"]
        return {"bytes": float(bytes_ + (8.0 * D if case["norm"] else 0)), "flops": float(rows * (Hq + Hkv) * (3 * case["rot"] + 4 * D * case["norm"]))}
    if kind == "fork":
        p, W, bytes_ = case["page"], case["width"], 0.0
        sources = 1 if case["fresh"] else W * (1 - (1 - 1 / W) ** W)     # beams that go on, where each is drawn
        for n in _spread(case["groups"], case["lo"], case["hi"]):
            held = -(-n // p)
            # rows that are not the first of their source take the tokens of the last page with them
            bytes_ += (W - sources) * (4.0 * (n % p) * case["H"] * case["D"] * size) + W * held * 8.0
        return {"bytes": bytes_ + 16.0 * case["groups"] * case["width"], "flops": 0.0}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    row = 2.0 * Hkv * D * size
    if kind == "shared":
        rows = case["groups"] * case["width"] + case["alone"]
        own_ = sum(_spread(rows, case["lo"], case["hi"]))
        prefix = _spread(case["groups"], case["plo"], case["phi"])
        alone = case["alone"] * prefix[-1]
        keys = own_ + alone + sum(p * case["width"] for p in prefix)
        tables = 4.0 * keys / case["page"]
        return {"bytes": row * (sum(prefix) + own_ + alone) + 2.0 * rows * Hq * D * size + tables, "flops": 4.0 * keys * Hq * D}
    if kind == "window":
        lens = _spread(case["B"], case["lo"], case["hi"])[case["skipped"]:]
        S, W, s = case["S"], case["window"], case["sinks"]
        pairs = 0
        for n in lens:
            # rows below n: as far as the window, then with the first tokens beside it
            for t in range(S):
                hi, lo = min(t + 1, n), max(0, t + 1 - W)
                pairs += max(0, hi - lo) + min(s, lo, n)
        return {"bytes": size * D * (2.0 * len(lens) * S * Hq + 2.0 * sum(lens) * Hkv), "flops": 4.0 * pairs * Hq * D}
    keys = sum(_visible(case, n) for n in _spread(case["B"], case["lo"], case["hi"]))
    return {"bytes": row * keys + 2.0 * case["B"] * Hq * D * size + 4.0 * keys / case["page"], "flops": 4.0 * keys * Hq * D}


# ------------------------------------------------------------------------------- inputs
def _frequencies(case):
    """Radians a position of each pair, and the factor of the rotated columns."""
    rot, kind, factor, original = case["rot"], case["scaling"], 8.0, 4096
    base = 10000.0 * (factor ** (rot / (rot - 2)) if kind == "base" and rot > 2 else 1.0)
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if kind == "linear":
            f /= factor
        elif kind == "ramp":
            share = min(1.0, max(0.0, (original * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)))
            f = share * f + (1 - share) * f / factor
        out.append(f)
    return out, (1.0 if kind in ("none", "linear") else 0.1 * math.log(factor) + 1.0)


def _host(case, seed):
    """Lengths and pages as Python lists: the same for prepare() and exact()."""
    rng = random.Random(seed * 7919 + 17)
    kind = case["kind"]
    h = {}
    if kind == "fork":
        W, p = case["width"], case["page"]
        B, n = case["groups"] * W, _fork_pages(case)
        lens = _spread(case["groups"], case["lo"], case["hi"])
        rng.shuffle(lens)
        pages = list(range(n))
        rng.shuffle(pages)
        max_pages = -(-case["hi"] // p) + 2
        table, seq, from_ = [[-1] * max_pages for _ in range(B)], [0] * B, [0] * B
        for q, m in enumerate(lens):
            held = -(-m // p)
            if case["fresh"]:
                table[q * W][:held] = [pages.pop() for _ in range(held)]
                seq[q * W] = m
                from_[q * W:(q + 1) * W] = [q * W] * W
                continue
            for b in range(q * W, (q + 1) * W):     # full pages up to some place are the first beam's, the others a beam's own
                cut = 0 if b == q * W else rng.randrange(max(0, held - 3), held)
                table[b][:held] = table[q * W][:cut] + [pages.pop() for _ in range(held - cut)]
                seq[b], from_[b] = m, q * W + rng.randrange(W)
        for b in rng.sample(range(B), case["ended"]):
            from_[b] = -1
        h.update(table=table, seq=seq, from_=from_, first=rng.randrange(n), max_pages=max_pages, n=n)
        wanted = min(len(pages), max(1, B // 3)) if case["short"] else len(pages)
        free = pages[:wanted]
        h["free"] = [-1] * n
        for i, q in enumerate(free):
            h["free"][(h["first"] + i) % n] = q
        h["count"] = len(free)
        return h
    if kind == "shared":
        G, W, p = case["groups"], case["width"], case["page"]
        rows = G * W + case["alone"]
        own_, prefix = _spread(rows, case["lo"], case["hi"]), _spread(G, case["plo"], case["phi"])
        rng.shuffle(own_)
        alone = prefix[-1]
        rng.shuffle(prefix)
        of = [b // W if b < G * W else -1 for b in range(rows)]
        seq = [own_[b] + (prefix[of[b]] if of[b] >= 0 else alone) for b in range(rows)]
        for b in rng.sample(range(G * W), min(case["short"], G * W)):
            seq[b] = max(0, prefix[of[b]] // 2)
        full = [m // p for m in prefix]
        n = sum(full) + sum(-(-s // p) - (full[q] if q >= 0 and s // p >= full[q] else 0) for s, q in zip(seq, of)) + rows + 3
        pages = list(range(n))
        rng.shuffle(pages)
        shared = [[pages.pop() for _ in range(f)] for f in full]
        width = max(-(-s // p) for s in seq)
        table = []
        for s, q in zip(seq, of):
            held = max(1, -(-s // p))
            mine = shared[q][:held] if q >= 0 else []
            mine = mine + [pages.pop() for _ in range(held - len(mine))]
            table.append(mine + [-1] * (max(width, 1) - held))
        h.update(table=table, seq=seq, of=of, prefix=prefix, full=full, n=n, first=[q * W for q in range(G + 1)])
        return h
    lens = _spread(case["B"], case["lo"], case["hi"])
    rng.shuffle(lens)
    h["lens"] = lens
    if kind == "rotate":
        S, p = case["S"], case["page"]
        far = 100000 if case["scaling"] != "none" else 0
        h["pos"] = [[far + t if t < n else -1 for t in range(S)] if S > 1 else [n] for n in lens]
        if p:
            need = [-(-n // p) + 1 for n in lens] if S > 1 else [1] * len(lens)
            h["n"] = sum(need) + 2
            pages = list(range(h["n"]))
            rng.shuffle(pages)
            h["slot"] = []
            for n, q in zip(lens, need):
                start = rng.randrange(p)
                mine = [pages.pop() for _ in range(q)]
                count = n if S > 1 else 1
                h["slot"].append([mine[(start + t) // p] * p + (start + t) % p for t in range(count)] + [-1] * (S - count))
    elif kind == "window":
        h["skip"] = rng.sample(range(case["B"]), case["skipped"])
        order = sorted(lens)      # the shortest are those that are left out, as work() has it
        rest = order[case["skipped"]:]
        rng.shuffle(rest)
        it, left = iter(rest), iter(order)
        h["lens"] = [next(left) if b in h["skip"] else next(it) for b in range(case["B"])]
    else:
        p, W, s = case["page"], case["window"], case["sinks"]
        alive = [[j for j in range(-(-n // p)) if j * p < s or (j + 1) * p > n - W] for n in lens]
        h["n"] = sum(len(a) for a in alive) + 3
        pages = list(range(h["n"]))
        rng.shuffle(pages)
        h["max_pages"] = -(-case["hi"] // p)
        h["alive"] = [[(j, pages.pop()) for j in a] for a in alive]
    return h


def _randn(gen, dt, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).to(_DT[dt])


def _inputs(case, seed):
    h, kind, dt, D = _host(case, seed), case["kind"], case["dt"], case["D"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    st = dict(kind=kind, case=case)
    if kind == "rotate":
        B, S, Hq, Hkv, p = (case[x] for x in ("B", "S", "Hq", "Hkv", "page"))
        freq, amp = _frequencies(case)
        st.update(X=_randn(gen, dt, B, S, (Hq + 2 * Hkv) * D), pos=i32(h["pos"]), amp=amp,
                  freq=torch.tensor(freq, dtype=torch.float64, device="cuda"),
                  Q=torch.zeros(B, Hq, S, D, dtype=_DT[dt], device="cuda"), K=None, V=None, slot=None, k_pages=None, v_pages=None,
                  q_weight=None, k_weight=None)
        if case["norm"]:
            st["q_weight"], st["k_weight"] = (1.0 + 0.2 * _randn(gen, "f32", D) for _ in range(2))
        if case["dense"]:
            st["K"], st["V"] = (torch.zeros(B, Hkv, S, D, dtype=_DT[dt], device="cuda") for _ in range(2))
        if p:
            st["k_plain"], st["v_plain"] = (torch.zeros(h["n"] + 1, Hkv, p, D, dtype=_DT[dt], device="cuda") for _ in range(2))
            st.update(slot=i32(h["slot"]), k_pages=st["k_plain"][:-1], v_pages=st["v_plain"][:-1])
        return st
    if kind == "fork":
        shape, B = (h["n"] + 1, case["H"], case["page"], D), len(h["seq"])
        st.update(from_row=i32(h["from_"]), seq_len=i32(h["seq"]), free_state=i32([h["first"], h["count"]]), free_pages=i32(h["free"]),
                  page_table=i32(h["table"]), table_out=torch.full((B, h["max_pages"]), -1, dtype=torch.int32, device="cuda"),
                  seq_len_out=torch.zeros(B, dtype=torch.int32, device="cuda"), sinks=case["sinks"], window=case["window"],
                  free_state_out=torch.zeros(2, dtype=torch.int32, device="cuda"),
                  k_plain=_randn(gen, dt, *shape), v_plain=_randn(gen, dt, *shape))
        st.update(k_pages=st["k_plain"][:-1], v_pages=st["v_plain"][:-1])
        return st
    Hq, Hkv = case["Hq"], case["Hkv"]
    if kind == "shared":
        p, rows = case["page"], len(h["seq"])
        st.update(Q=_randn(gen, dt, rows, Hq, D), k_pages=_randn(gen, dt, h["n"], Hkv, p, D), v_pages=_randn(gen, dt, h["n"], Hkv, p, D),
                  page_table=i32(h["table"]), lens=i32(h["seq"]), share_first=i32(h["first"]), share_len=i32(h["prefix"]))
        # the page in which a prefix ends is copied for each request
        for q, (full, m) in enumerate(zip(h["full"], h["prefix"])):
            mine = [b for b in range(rows) if h["of"][b] == q and h["seq"][b] >= m]
            if m % p and len(mine) > 1:
                at = torch.tensor([h["table"][b][full] for b in mine], device="cuda")
                for pages in (st["k_pages"], st["v_pages"]):
                    pages[at, :, :m % p] = pages[at[:1], :, :m % p].clone()
        return st
    B = case["B"]
    st.update(lens=i32(h["lens"]), window=case["window"], sinks=case["sinks"])
    if kind == "window":
        S = case["S"]
        sel = [0 if b in h["skip"] else -1 for b in range(B)]
        st.update(Q=_randn(gen, dt, B, Hq, S, D), K=_randn(gen, dt, B, Hkv, S, D), V=_randn(gen, dt, B, Hkv, S, D), row_sel=i32(sel),
                  O=torch.zeros(B, Hq, S, D, dtype=_DT[dt], device="cuda"))
        return st
    p = case["page"]
    table = torch.full((B, h["max_pages"]), -1, dtype=torch.int32)
    for b, a in enumerate(h["alive"]):
        table[b, torch.tensor([j for j, _ in a])] = torch.tensor([q for _, q in a], dtype=torch.int32)
    st.update(Q=_randn(gen, dt, B, Hq, D), k_pages=_randn(gen, dt, h["n"], Hkv, p, D), v_pages=_randn(gen, dt, h["n"], Hkv, p, D),
              page_table=table.cuda())
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    kind = case["kind"]
    if own and kind in ("fork", "shared", "window_step"):
        from paper_2510_25979_amd import binding as ac
        if kind == "fork":
            need = ac.attncache_page_fork_workspace_bytes(*st["page_table"].shape, st["free_pages"].numel())
        else:
            B, Hq, D = st["Q"].shape
            st["O"] = torch.empty_like(st["Q"])
            need = (ac.attention_paged_workspace_bytes(B, Hq, case["Hkv"], D) if kind == "window_step" else
                    ac.attention_paged_shared_workspace_bytes(B, Hq, case["Hkv"], D, case["groups"]))
        st["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------------------- one pass
def run(st):
    if own:
        return _run_own(st)
    return {"rotate": _plain_rotate, "fork": _plain_fork, "shared": _plain_shared, "window": _plain_window,
            "window_step": _plain_window_step}[st["kind"]](st)


def _run_own(st):
    from paper_2510_25979_amd import binding as ac
    kind, case = st["kind"], st["case"]
    if kind == "rotate":
        ac.attncache_rotate(st["X"], st["pos"], st["freq"], st["Q"], st["K"], st["V"], q_weight=st["q_weight"],
                            k_weight=st["k_weight"], eps=1e-6, amplitude=st["amp"], interleaved=case["interleaved"],
                            slot=st["slot"], k_pages=st["k_pages"], v_pages=st["v_pages"])
        return {n: st[n] for n in ("Q", "K", "V", "k_pages", "v_pages") if st[n] is not None}
    if kind == "fork":
        ac.attncache_page_fork(st["from_row"], st["seq_len"], st["free_state"], st["free_pages"], st["page_table"],
                               st["table_out"], st["seq_len_out"], st["free_state_out"], st["k_pages"], st["v_pages"], st["ws"],
                               sinks=st["sinks"], window=st["window"])
        return {n: st[n] for n in ("table_out", "seq_len_out", "free_state_out", "free_pages", "k_pages", "v_pages")}
    if kind == "shared":
        ac.attention_paged_shared(st["Q"], st["k_pages"], st["v_pages"], st["page_table"], st["lens"], st["share_first"],
                                  st["share_len"], st["O"], st["ws"])
    elif kind == "window":
        ac.attention_window(st["Q"], st["K"], st["V"], st["O"], window=st["window"], sinks=st["sinks"], row_sel=st["row_sel"],
                            key_len=st["lens"])
    else:
        ac.attention_paged_window(st["Q"], st["k_pages"], st["v_pages"], st["page_table"], st["lens"], st["O"], st["ws"],
                                  window=st["window"], sinks=st["sinks"])
    return {"O": st["O"]}


def _plain_rotate(st):
    case, X, pos = st["case"], st["X"], st["pos"]
    Hq, Hkv, D, rot = (case[x] for x in ("Hq", "Hkv", "D", "rot"))
    B, S, _ = X.shape
    x = X.float().view(B, S, Hq + 2 * Hkv, D)
    angle = pos.double()[:, :, None, None] * st["freq"]          # [B,S,1,rot/2]; 64 bits: positions are far
    cos, sin = (torch.cos(angle) * st["amp"]).float(), (torch.sin(angle) * st["amp"]).float()
    out = {}
    for name, lo, hi, weight in (("Q", 0, Hq, "q_weight"), ("K", Hq, Hq + Hkv, "k_weight"), ("V", Hq + Hkv, Hq + 2 * Hkv, None)):
        y = x[:, :, lo:hi]
        if weight:
            if st[weight] is not None:
                y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * st[weight]
            first = slice(0, rot, 2) if case["interleaved"] else slice(0, rot // 2)
            second = slice(1, rot, 2) if case["interleaved"] else slice(rot // 2, rot)
            z = y.clone()
            z[..., first] = y[..., first] * cos - y[..., second] * sin
            z[..., second] = y[..., second] * cos + y[..., first] * sin
            y = z
        y = y.transpose(1, 2).to(X.dtype)
        if st[name] is not None:
            out[name] = torch.where((pos >= 0)[:, None, :, None], y, st[name])
        pages = {"K": "k_plain", "V": "v_plain"}.get(name)
        if pages and st["slot"] is not None:
            n, _, p, _ = st["k_pages"].shape
            slot = torch.where(pos < 0, torch.full_like(pos, -1), st["slot"]).long().flatten()
            slot = torch.where(slot < 0, torch.full_like(slot, n * p), slot)       # the page behind the last is nobody's
            st[pages][slot // p, :, slot % p] = y.transpose(1, 2).reshape(-1, Hkv, D)
    if st["slot"] is not None:
        out.update(k_pages=st["k_pages"], v_pages=st["v_pages"])
    return out


def _plain_fork(st):
    from_, seq, old = st["from_row"].long(), st["seq_len"].long(), st["page_table"].long()
    B, width = old.shape
    n, _, p, _ = st["k_pages"].shape
    dev = seq.device
    first, count = st["free_state"].long().unbind()
    row, j = torch.arange(B, device=dev), torch.arange(width, device=dev)
    there = from_ >= 0
    src = from_.clamp(min=0)
    ln = torch.where(there, seq[src], torch.zeros_like(seq))
    held, part = (ln + p - 1) // p, ln % p
    # who keeps the page in which a row ends: the row itself, or the first that takes it
    rank = torch.where(there, torch.where(from_ == row, torch.full_like(row, -1), row), torch.full_like(row, B))
    best = torch.full((B,), B, device=dev).scatter_reduce(0, src, rank, "amin")
    copies = there & (part > 0) & (rank != best[src])
    upto = torch.cumsum(copies.long(), 0)
    served = there & (~copies | (upto <= count))
    copies = copies & served
    fresh = st["free_pages"].long()[(first + upto - 1) % n]
    mine = served[:, None] & (j < held[:, None])
    last = held - 1
    taken = old[src]
    new = torch.where(copies[:, None] & (j == last[:, None]), fresh[:, None], taken)
    if st["window"] > 0:
        gone = ((j + 1) * p <= (ln - st["window"])[:, None]) & (j * p >= st["sinks"])
        new = torch.where(gone, torch.full_like(new, -1), new)
    table = torch.where(mine, new, st["table_out"].long())
    # pages that somebody had and nobody has
    had, has = (torch.zeros(n + 1, dtype=torch.bool, device=dev) for _ in range(2))
    before = torch.where((j < ((seq + p - 1) // p)[:, None]) & (old >= 0), old, torch.full_like(old, n))
    after = torch.where(mine & (new >= 0), new, torch.full_like(new, n))
    had[before.flatten()] = True
    has[after.flatten()] = True
    free = (had & ~has)[:n]
    place = torch.cumsum(free.long(), 0) - 1
    ring = torch.cat([st["free_pages"], st["free_pages"][:1]])
    to = torch.where(free, (first + count + place) % n, torch.full_like(place, n))
    ring[to] = torch.arange(n, device=dev, dtype=torch.int32)
    took = copies.sum()
    # tokens of the last page
    here = torch.where(copies, torch.gather(taken, 1, last.clamp(min=0)[:, None])[:, 0], torch.full_like(last, n))
    there_ = torch.where(copies, fresh, torch.full_like(fresh, n))
    keep = (torch.arange(p, device=dev) < part[:, None])[:, None, :, None]
    for pages in (st["k_plain"], st["v_plain"]):
        pages[there_] = torch.where(keep, pages[here], pages[there_])
    i32 = torch.int32
    lens = torch.where(served, ln, torch.where(there, torch.full_like(ln, -1), torch.zeros_like(ln)))
    return {"table_out": table.to(i32), "seq_len_out": lens.to(i32),
            "free_state_out": torch.stack([(first + took) % n, count - took + free.sum()]).to(i32), "free_pages": ring[:n],
            "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _plain_attention(q, k, v, seen):
    """q [B,Hkv,R,D], k and v [B,Hkv,N,D], all binary32; seen broadcasts to [B,Hkv,R,N].  Rows that see nothing: zeros."""
    D = q.shape[-1]
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(D))
    s = s.masked_fill(~seen, -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    return torch.matmul(e, v) / e.sum(-1, keepdim=True).clamp(min=1e-30)


def _plain_shared(st):
    Q, table, p = st["Q"], st["page_table"].long().clamp(min=0), st["case"]["page"]
    B, Hq, D = Q.shape
    Hkv = st["case"]["Hkv"]
    k, v = (st[x][table].permute(0, 2, 1, 3, 4).reshape(B, Hkv, table.shape[1] * p, D).float()
            for x in ("k_pages", "v_pages"))
    seen = torch.arange(k.shape[2], device=Q.device) < st["lens"][:, None]
    o = _plain_attention(Q.float().view(B, Hkv, Hq // Hkv, D), k, v, seen[:, None, None, :])
    return {"O": o.view(B, Hq, D).to(Q.dtype)}


def _plain_window(st):
    Q, K, V, W = st["Q"], st["K"], st["V"], st["window"]
    B, Hq, S, D = Q.shape
    Hkv = K.shape[1]
    t, j = torch.arange(S, device=Q.device)[:, None], torch.arange(S, device=Q.device)
    seen = (j <= t) & ((j > t - W) | (j < st["sinks"])) & (j < st["lens"][:, None, None])      # [B,S,S]
    o = _plain_attention(Q.float().view(B, Hkv, Hq // Hkv * S, D), K.float(), V.float(),
                         seen[:, None, None].expand(B, Hkv, Hq // Hkv, S, S).reshape(B, Hkv, Hq // Hkv * S, S))
    return {"O": torch.where((st["row_sel"] >= 0)[:, None, None, None], st["O"], o.view(B, Hq, S, D).to(Q.dtype))}


def _plain_window_step(st):
    Q, p, W, s = st["Q"], st["case"]["page"], st["window"], st["sinks"]
    B, Hq, D = Q.shape
    Hkv = st["case"]["Hkv"]
    n = st["lens"].long()[:, None]
    i = torch.arange(s + W, device=Q.device)
    at = torch.where(i < s, i, (n - W).clamp(min=s) + i - s)     # the first tokens, then the window
    seen = at < n
    at = torch.where(seen, at, torch.zeros_like(at))
    page = torch.gather(st["page_table"].long(), 1, at // p).clamp(min=0)
    k, v = (st[x][page, :, at % p].transpose(1, 2).float() for x in ("k_pages", "v_pages"))
    o = _plain_attention(Q.float().view(B, Hkv, Hq // Hkv, D), k, v, seen[:, None, None, :])
    return {"O": o.view(B, Hq, D).to(Q.dtype)}


# ------------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    h, kind = _host(case, seed), case["kind"]
    if kind == "window" and case["B"] * case["Hq"] * case["S"] ** 2 > 1.2 * _MAX_SCORES:
        return None
    st = _inputs(case, seed)
    return {"rotate": _exact_rotate, "fork": _exact_fork, "shared": _exact_pages, "window": _exact_window,
            "window_step": _exact_pages}[kind](case, h, st)


def _exact_rotate(case, h, st):
    B, S, Hq, Hkv, D, rot = (case[x] for x in ("B", "S", "Hq", "Hkv", "D", "rot"))
    x = st["X"].double().view(B, S, Hq + 2 * Hkv, D).permute(2, 0, 1, 3)
    turn = torch.polar(torch.full_like(st["freq"], st["amp"]).expand(B, S, -1).contiguous(), st["pos"].double()[..., None] * st["freq"])
    real = [[(b, t) for t in range(S) if h["pos"][b][t] >= 0] for b in range(B)]
    ok = st["pos"] >= 0

    def heads(part, weight):
        if weight is not None:
            part = part * torch.rsqrt(part.square().mean(-1, keepdim=True) + 1e-6) * weight.double()
        r = part[..., :rot]
        pairs = r.unflatten(-1, (rot // 2, 2)) if case["interleaved"] else r.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z if case["interleaved"] else z.transpose(-1, -2)
        return torch.cat([z.flatten(-2), part[..., rot:]], -1)

    parts = {"Q": heads(x[:Hq], st["q_weight"]), "K": heads(x[Hq:Hq + Hkv], st["k_weight"]), "V": x[Hq + Hkv:]}
    out = {}
    for name, y in parts.items():          # y [H,B,S,D]
        if st[name] is not None:
            out[name] = torch.where(ok[:, None, :, None], y.permute(1, 0, 2, 3), torch.zeros((), dtype=torch.float64, device="cuda"))
    if case["page"]:
        p = case["page"]
        for name, pages in (("K", "k_pages"), ("V", "v_pages")):
            to = st[pages].double()
            for b in range(B):
                at = torch.tensor(h["slot"][b][:len(real[b])], device="cuda")
                to[at // p, :, at % p, :] = parts[name][:, b, :len(real[b])].transpose(0, 1)
            out[pages] = to
    return out


def _exact_fork(case, h, st):
    p, n, B = case["page"], h["n"], len(h["seq"])
    out = [[-1] * h["max_pages"] for _ in range(B)]
    lens, taken, moves = [0] * B, 0, []
    queue = 0
    for b, s in enumerate(h["from_"]):
        if s < 0:
            continue
        m = h["seq"][s]
        pages = h["table"][s][:-(-m // p)]
        keeper = s if h["from_"][s] == s else h["from_"].index(s)
        if m % p and keeper != b:
            queue += 1
            if queue > h["count"]:
                lens[b] = -1
                continue
            fresh = h["free"][(h["first"] + taken) % n]
            taken += 1
            moves.append((pages[-1], fresh, m % p))
            pages = pages[:-1] + [fresh]
        lens[b] = m
        for j, q in enumerate(pages):
            dead = case["window"] > 0 and (j + 1) * p <= m - case["window"] and j * p >= case["sinks"]
            out[b][j] = -1 if dead else q
    had = {q for b in range(B) for q in h["table"][b][:-(-h["seq"][b] // p)] if q >= 0}
    has = {q for b in range(B) for q in out[b] if q >= 0}
    ring = h["free"][:]
    gone = sorted(had - has)
    for i, q in enumerate(gone):
        ring[(h["first"] + h["count"] + i) % n] = q
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    res = {"table_out": i32(out), "seq_len_out": i32(lens),
           "free_state_out": i32([(h["first"] + taken) % n, h["count"] - taken + len(gone)]), "free_pages": i32(ring)}
    for pages in ("k_pages", "v_pages"):
        to = st[pages].double()
        for a, b, m in moves:
            to[b, :, :m] = st[pages][a, :, :m].double()
        res[pages] = to
    return res


def _weighted(q, k, v, hidden=None):
    q, k, v = q.double(), k.double(), v.double()
    s = q @ k.t() / math.sqrt(q.shape[-1])
    if hidden is not None:
        s[hidden] = -math.inf
    return torch.nan_to_num(torch.softmax(s, -1)) @ v


def _exact_pages(case, h, st):
    """One token of each request over its pages: all of them, or those that the window leaves."""
    Hq, Hkv, D, p = (case[x] for x in ("Hq", "Hkv", "D", "page"))
    lens = h["seq"] if case["kind"] == "shared" else h["lens"]
    g = Hq // Hkv
    out = torch.zeros(len(lens), Hq, D, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        if n == 0:
            continue
        if case["kind"] == "shared":
            js, pages = list(range(-(-n // p))), h["table"][b][:-(-n // p)]
        else:
            js, pages = (list(x) for x in zip(*h["alive"][b]))
        at = (torch.tensor(js, device="cuda")[:, None] * p + torch.arange(p, device="cuda")).flatten()
        seen = at < n
        if case["kind"] != "shared":
            seen &= (at >= n - case["window"]) | (at < case["sinks"])
        k, v = (st[x][torch.tensor(pages, device="cuda")].transpose(0, 1).flatten(1, 2)[:, seen] for x in ("k_pages", "v_pages"))
        for hk in range(Hkv):
            out[b, hk * g:(hk + 1) * g] = _weighted(st["Q"][b, hk * g:(hk + 1) * g], k[hk], v[hk])
    return {"O": out}


def _exact_window(case, h, st):
    B, Hq, Hkv, S, D = (case[x] for x in ("B", "Hq", "Hkv", "S", "D"))
    g = Hq // Hkv
    out = torch.zeros(B, Hq, S, D, dtype=torch.float64, device="cuda")
    j = torch.arange(S, device="cuda")
    back = j[:, None] - j
    for b in range(B):
        if b in h["skip"]:
            continue
        hidden = (back < 0) | ((back >= case["window"]) & (j >= case["sinks"])) | (j >= h["lens"][b])
        for q in range(Hq):
            out[b, q] = _weighted(st["Q"][b, q], st["K"][b, q // g], st["V"][b, q // g], hidden)
    return {"O": out}
