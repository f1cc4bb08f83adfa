"""Generation after the prefill, as cases that can be timed and compared: the page plan of a step, K and V rows into
their pages, attention of one new token over the pages, and attention to an encoder's states of another length.

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
        # The bookkeeping of one generated token: 64 requests, one token each, a few of them at their end.
        dict(name="plan-step", kind="plan", B=64, S=1, page=16, max_pages=128, lo=100, hi=2000, fresh=False, ended=3,
             short=False, spare=64),
        # The bookkeeping of a large batch of new prompts of ragged length.
        dict(name="plan-prompts", kind="plan", B=256, S=1024, page=16, max_pages=128, lo=16, hi=1024, fresh=True, ended=0,
             short=False, spare=500),
        # One layer's K and V of one generated token of each request.
        dict(name="append-step", kind="append", B=128, H=8, S=1, D=128, dt="bf16", page=16, lo=1, hi=1, n_pages=1024),
        # K and V of a batch of ragged prompts, all layers of a 1B-shaped model folded into the heads.
        dict(name="append-prompts", kind="append", B=64, H=128, S=128, D=64, dt="bf16", page=16, lo=32, hi=128,
             n_pages=640),
        # The same in binary32 with pages and lengths of odd sizes.
        dict(name="append-fp32", kind="append", B=16, H=8, S=94, D=80, dt="f32", page=10, lo=1, hi=94, n_pages=200),
        # A few requests with short contexts: latency counts.
        dict(name="paged-few", kind="paged", B=4, Hq=32, Hkv=8, D=64, dt="bf16", page=16, L=1, lo=50, hi=1000),
        # A full serving batch of an 8B-shaped layer, contexts from short to long.
        dict(name="paged-batch", kind="paged", B=128, Hq=32, Hkv=8, D=128, dt="bf16", page=16, L=1, lo=128, hi=4096),
        # Few requests with very long contexts.
        dict(name="paged-long", kind="paged", B=4, Hq=32, Hkv=8, D=128, dt="bf16", page=64, L=1, lo=30000, hi=131072),
        # Binary32, three query heads on one K and V, pages of odd size, contexts from one token on.
        dict(name="paged-fp32", kind="paged", B=16, Hq=24, Hkv=8, D=128, dt="f32", page=10, L=1, lo=1, hi=1500),
        # A generated token of each request attends to its encoder's padded states.
        dict(name="cross-step", kind="cross", B=32, Hq=12, Hkv=12, Sq=1, Sk=1000, D=64, dt="bf16", lo=200, hi=1000),
        # A decoder's prompts attend to long encoder states of odd length.
        dict(name="cross-long", kind="cross", B=16, Hq=32, Hkv=32, Sq=1024, Sk=2047, D=128, dt="bf16", lo=2047, hi=2047),
        # The same in binary32, the precision of the paper's models, small and ragged.
        dict(name="cross-fp32", kind="cross", B=8, Hq=24, Hkv=8, Sq=94, Sk=333, D=128, dt="f32", lo=100, hi=333),
    ]


# ------------------------------------------------------------------------------- drawn cases
_MAX_BYTES = 1.1e9       # one pass, and what a state holds
_MAX_FLOPS = 5.4e11      # matrix cores
_MAX_FLOPS_F32 = 8.0e9


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _fit(case):
    """Halve the batch, then the lengths, until a pass and its state fit the limits above."""
    while True:
        w = work(case)
        state = _SIZE[case["dt"]] * 2 * case["D"] * (
            case["n_pages"] * case["page"] * case["H"] if case["kind"] == "append" else
            case["B"] * (case["hi"] + case.get("page", 0)) * case["Hkv"] * case.get("L", 1))
        if max(w["bytes"], state / 4) <= _MAX_BYTES and w["flops"] <= (
                _MAX_FLOPS_F32 if case["dt"] == "f32" else _MAX_FLOPS):
            return case
        if case["B"] > 1:
            case["B"] //= 2
        else:
            case["hi"] = max(1, case["hi"] // 2)
            case["lo"] = min(case["lo"], case["hi"])
            if "Sk" in case:
                case["Sk"] = case["hi"]


def draw(rng):
    kind = rng.choice(["plan", "append", "paged", "paged", "paged", "cross", "cross", "cross"])
    page = rng.choice([1, 8, 10, 16, 16, 16, 32, 48, 64, 128])
    if kind == "plan":
        B, fresh = _log_int(rng, 8, 1000), rng.random() < 0.5
        S = _log_int(rng, 1, min(2048, max(1, 300000 // B))) if fresh else rng.choice([1, 1, 1, 2, 5])
        hi = S if fresh else _log_int(rng, 1, 8000)
        return dict(kind=kind, B=B, S=S, page=page, max_pages=-(-(hi + S) // page) + rng.randrange(4),
                    lo=_log_int(rng, 1, hi), hi=hi, fresh=fresh, ended=0 if fresh else rng.randrange(B // 4 + 1),
                    short=rng.random() < 0.25, spare=rng.choice([8, 30, B, 4 * B]))
    f32 = rng.random() < 0.25
    dt = "f32" if f32 else "bf16"
    D = rng.choice([32, 64, 80, 100, 128, 199, 256]) if f32 else rng.choice([64, 128])
    hkv = rng.choice([1, 2, 4, 8, 12])
    g = rng.choice([1, 1, 2, 3, 4, 8])
    if kind == "append":
        S = rng.choice([1, 1, _log_int(rng, 1, 1024)])
        c = dict(kind=kind, B=_log_int(rng, 1, 256), H=hkv * rng.choice([1, 1, 4, 16]), S=S, D=D, dt=dt, page=page,
                 lo=_log_int(rng, 1, S), hi=S, n_pages=0)
        while True:
            c["n_pages"] = c["B"] * (-(-S // page)) + 5
            B = c["B"]
            _fit(c)
            if c["B"] == B:
                return c
    if kind == "paged":
        hi = _log_int(rng, 1, 100000)
        return _fit(dict(kind=kind, B=_log_int(rng, 1, 256), Hq=hkv * g, Hkv=hkv, D=D, dt=dt, page=page,
                         L=rng.choice([1, 1, 3]), lo=_log_int(rng, 1, hi), hi=hi))
    Sk = _log_int(rng, 1, 4096)
    return _fit(dict(kind=kind, B=_log_int(rng, 1, 64), Hq=hkv * g, Hkv=hkv, Sq=rng.choice([1, _log_int(rng, 1, 2048)]),
                     Sk=Sk, D=D, dt=dt, lo=_log_int(rng, 1, Sk), hi=Sk))


# ------------------------------------------------------------------------------- sizes
def _lengths(case):
    """B lengths spread over [lo, hi] by their logarithm; the seed only says which request has which."""
    n, lo, hi = case["B"], case["lo"], case["hi"]
    return [max(lo, min(hi, int(round(math.exp(math.log(lo) + (i + 0.5) / n * (math.log(hi) - math.log(lo)))))))
            for i in range(n)]


def work(case):
    kind, B = case["kind"], case["B"]
    lens = _lengths(case)
    if kind == "plan":
        fresh, p = case["fresh"], case["page"]
        pages = sum(-(-n // p) for n in lens) if fresh else B // p
        return {"bytes": 4.0 * (2 * B + pages) + 4.0 * (B * case["S"] + 2 * B + pages + 4), "flops": 0.0}
    size = _SIZE[case["dt"]]
    if kind == "append":
        return {"bytes": 4.0 * sum(lens) * case["H"] * case["D"] * size + 4.0 * B * case["S"], "flops": 0.0}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    Sq = case.get("Sq", 1)
    bytes_ = size * D * (2.0 * sum(lens) * Hkv + 2.0 * B * Sq * Hq) + 4.0 * B
    if kind == "paged":
        bytes_ += 4.0 * sum(-(-n // case["page"]) for n in lens)
    return {"bytes": bytes_, "flops": 4.0 * Sq * sum(lens) * Hq * D}


# ------------------------------------------------------------------------------- inputs
def _host(case, seed):
    """Lengths and pages as Python lists: the same for prepare() and exact()."""
    rng = random.Random(seed * 7919 + 17)
    lens = _lengths(case)
    rng.shuffle(lens)
    h = {"lens": lens}
    if case["kind"] == "plan":
        B, p = case["B"], case["page"]
        h["seq"] = [0] * B if case["fresh"] else lens
        h["new"] = lens if case["fresh"] else [case["S"]] * B
        for b in rng.sample(range(B), case["ended"]):
            h["new"][b] = -1
        held = [-(-n // p) for n in h["seq"]]
        want = sum(max(0, -(-(s + max(n, 0)) // p) - q) for s, n, q in zip(h["seq"], h["new"], held))
        n = sum(held) + (want // 2 if case["short"] else want) + case["spare"] + 1
        pages = list(range(n))
        rng.shuffle(pages)
        h["table"] = [[-1] * case["max_pages"] for _ in range(B)]
        for b, q in enumerate(held):
            for j in range(q):
                h["table"][b][j] = pages.pop()
        h["first"] = rng.randrange(n)
        h["free"] = [-1] * n
        for i, q in enumerate(pages):
            h["free"][(h["first"] + i) % n] = q
        h["count"] = len(pages)
    elif case["kind"] == "append":
        n, p = case["n_pages"], case["page"]
        pages = list(range(n))
        rng.shuffle(pages)
        h["slot"] = []
        for b, m in enumerate(lens):
            start = rng.randrange(p) if case["S"] == 1 else 0
            mine = [pages.pop() for _ in range(-(-(start + m) // p))]
            h["slot"].append([mine[(start + t) // p] * p + (start + t) % p for t in range(m)] + [-1] * (case["S"] - m))
    elif case["kind"] == "paged":
        p = case["page"]
        held = [-(-n // p) for n in lens]
        h["n_pages"] = sum(held) + 3
        pages = list(range(h["n_pages"]))
        rng.shuffle(pages)
        width = -(-case["hi"] // p)
        h["table"] = [[pages.pop() for _ in range(q)] + [-1] * (width - q) for q in held]
    return h


def _randn(gen, dt, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).to(_DT[dt])


def _inputs(case, seed):
    h, kind, B = _host(case, seed), case["kind"], case["B"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    st = dict(kind=kind, case=case)
    if kind == "plan":
        st.update(seq_len=i32(h["seq"]), new_len=i32(h["new"]), free_state=i32([h["first"], h["count"]]),
                  free_pages=i32(h["free"]), page_table=i32(h["table"]), page=case["page"],
                  seq_len_out=torch.zeros(B, dtype=torch.int32, device="cuda"),
                  added=torch.zeros(B, dtype=torch.int32, device="cuda"),
                  free_state_out=torch.zeros(2, dtype=torch.int32, device="cuda"),
                  slot=torch.zeros(B, case["S"], dtype=torch.int32, device="cuda"))
        return st
    D, dt = case["D"], case["dt"]
    if kind == "append":
        shape = (case["n_pages"] + 1, case["H"], case["page"], D)
        st.update(K=_randn(gen, dt, B, case["H"], case["S"], D), V=_randn(gen, dt, B, case["H"], case["S"], D),
                  slot=i32(h["slot"]), k_plain=_randn(gen, dt, *shape), v_plain=_randn(gen, dt, *shape))
        st.update(k_pages=st["k_plain"][:-1], v_pages=st["v_plain"][:-1])
        return st
    Hq, Hkv, Sq = case["Hq"], case["Hkv"], case.get("Sq", 1)
    st["lens"] = i32(h["lens"])
    if kind == "paged":
        L = case["L"]
        cache = [_randn(gen, dt, h["n_pages"], L * Hkv, case["page"], D) for _ in range(2)]
        # one layer of a cache that holds L
        st.update(Q=_randn(gen, dt, B, Hq, D), k_pages=cache[0][:, (L - 1) * Hkv:], v_pages=cache[1][:, (L - 1) * Hkv:],
                  page_table=i32(h["table"]))
    else:
        st.update(Q=_randn(gen, dt, B, Hq, Sq, D), K=_randn(gen, dt, B, Hkv, case["Sk"], D),
                  V=_randn(gen, dt, B, Hkv, case["Sk"], D))
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own and case["kind"] in ("paged", "cross"):
        from paper_2510_25979_amd import binding as ac
        B, Hq, Hkv, D = (case[x] for x in ("B", "Hq", "Hkv", "D"))
        st["O"] = torch.empty_like(st["Q"])
        need = (ac.attention_paged_workspace_bytes(B, Hq, Hkv, D) if case["kind"] == "paged" else
                ac.attention_cross_workspace_bytes(B, Hq, Hkv, case["Sq"], case["Sk"], D))
        st["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------------------- one pass
def run(st):
    if own:
        return _run_own(st)
    return {"plan": _plain_plan, "append": _plain_append, "paged": _plain_paged, "cross": _plain_cross}[st["kind"]](st)


def _run_own(st):
    from paper_2510_25979_amd import binding as ac
    kind = st["kind"]
    if kind == "plan":
        ac.attncache_page_plan(st["seq_len"], st["new_len"], st["free_state"], st["free_pages"], st["page_table"],
                               st["seq_len_out"], st["added"], st["free_state_out"], st["slot"], page_size=st["page"])
        return {n: st[n] for n in ("seq_len_out", "added", "free_state_out", "free_pages", "page_table", "slot")}
    if kind == "append":
        ac.attncache_page_append(st["K"], st["V"], st["slot"], st["k_pages"], st["v_pages"])
        return {"k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if kind == "paged":
        ac.attention_paged(st["Q"], st["k_pages"], st["v_pages"], st["page_table"], st["lens"], st["O"], st["ws"])
    else:
        ac.attention_cross(st["Q"], st["K"], st["V"], st["O"], st["ws"], key_len=st["lens"])
    return {"O": st["O"]}


def _plain_plan(st):
    seq, new, p = st["seq_len"].long(), st["new_len"].long(), st["page"]
    table, n = st["page_table"].clone(), st["free_pages"].numel()
    ring = torch.cat([st["free_pages"], st["free_pages"][:1]])
    (B, width), S = table.shape, st["slot"].shape[1]
    first, count = st["free_state"].long().unbind()
    dev = seq.device
    ended = new < 0
    new = new.clamp(0, S)
    held = (seq + p - 1) // p
    need = (seq + new + p - 1) // p - held
    fits = (seq + new <= width * p) & ~ended
    need = torch.where(fits, need, torch.zeros_like(need))
    upto = torch.cumsum(need, 0)
    served = fits & ((need == 0) | (upto <= count))
    added = torch.where(served, new, torch.zeros_like(new))
    # new pages: entry j of a row is the (upto - need + j - held)-th free one
    j = torch.arange(width, device=dev)
    fresh = served[:, None] & (j >= held[:, None]) & (j < (held + need)[:, None])
    at = (first + (upto - need - held)[:, None] + j) % n
    # pages of requests that have ended go to the end of the ring
    given = torch.where(ended, held, torch.zeros_like(held))
    back = ended[:, None] & (j < held[:, None])
    to = (first + count + (torch.cumsum(given, 0) - given)[:, None] + j) % n
    old = st["page_table"]
    table = torch.where(fresh, st["free_pages"][at], table)
    ring.scatter_(0, torch.where(back, to, torch.full_like(to, n)).flatten(), old.flatten())   # [n]: nobody's
    taken = torch.where(served, need, torch.zeros_like(need)).sum()
    t = torch.arange(S, device=dev)
    pos = seq[:, None] + t
    page = torch.gather(table, 1, (pos // p).clamp(max=width - 1)).long()
    slot = torch.where(t < added[:, None], page * p + pos % p, torch.full_like(pos, -1))
    i32 = torch.int32
    return {"seq_len_out": torch.where(ended, torch.zeros_like(seq), seq + added).to(i32), "added": added.to(i32),
            "free_state_out": torch.stack([(first + taken) % n, count - taken + given.sum()]).to(i32),
            "free_pages": ring[:n], "page_table": table, "slot": slot.to(i32)}


def _plain_append(st):
    n, H, p, D = st["k_pages"].shape
    slot = st["slot"].long().flatten()
    slot = torch.where(slot < 0, torch.full_like(slot, n * p), slot)       # the page behind the last is nobody's
    for rows, pages in (("K", "k_plain"), ("V", "v_plain")):
        st[pages][slot // p, :, slot % p] = st[rows].transpose(1, 2).reshape(-1, H, D)
    return {"k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _plain_attention(q, k, v, lens):
    """q [B,Hkv,R,D], k and v [B,Hkv,N,D], all binary32; keys from lens[b] on are hidden."""
    D = q.shape[-1]
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(D))
    seen = torch.arange(k.shape[2], device=q.device) < lens[:, None]
    s = s.masked_fill(~seen[:, None, None, :], -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - m)
    return torch.matmul(e, v) / e.sum(-1, keepdim=True)


def _plain_paged(st):
    Q, table = st["Q"], st["page_table"].long().clamp(min=0)
    B, Hq, D = Q.shape
    n, Hkv, p, _ = st["k_pages"].shape
    k, v = (st[x][table].permute(0, 2, 1, 3, 4).reshape(B, Hkv, table.shape[1] * p, D).float()
            for x in ("k_pages", "v_pages"))
    o = _plain_attention(Q.float().view(B, Hkv, Hq // Hkv, D), k, v, st["lens"])
    return {"O": o.view(B, Hq, D).to(Q.dtype)}


def _plain_cross(st):
    Q, K, V = st["Q"], st["K"], st["V"]
    B, Hq, Sq, D = Q.shape
    Hkv = K.shape[1]
    o = _plain_attention(Q.float().view(B, Hkv, Hq // Hkv * Sq, D), K.float(), V.float(), st["lens"])
    return {"O": o.view(B, Hq, Sq, D).to(Q.dtype)}


# ------------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    h, kind, B = _host(case, seed), case["kind"], case["B"]
    if kind == "plan":
        return _exact_plan(case, h)
    st = _inputs(case, seed)
    if kind == "append":
        p = case["page"]
        out = {}
        for rows, pages in (("K", "k_pages"), ("V", "v_pages")):
            to, src = st[pages].double(), st[rows].double()
            for b in range(B):
                m = h["lens"][b]
                at = torch.tensor(h["slot"][b][:m], device="cuda")
                to[at // p, :, at % p, :] = src[b, :, :m].transpose(0, 1)
            out[pages] = to
        return out
    Hq, Hkv, D, Sq = case["Hq"], case["Hkv"], case["D"], case.get("Sq", 1)
    g = Hq // Hkv
    out = torch.zeros(B, Hq, Sq, D, dtype=torch.float64, device="cuda")
    Q = st["Q"].view(B, Hq, Sq, D)
    for b in range(B):
        n = h["lens"][b]
        if kind == "paged":
            p = case["page"]
            pages = torch.tensor(h["table"][b][:-(-n // p)], device="cuda")
            k, v = (st[x][pages].transpose(0, 1).flatten(1, 2)[:, :n] for x in ("k_pages", "v_pages"))
        else:
            k, v = st["K"][b, :, :n], st["V"][b, :, :n]
        for hk in range(Hkv):
            kk, vv = k[hk].double(), v[hk].double()
            q = Q[b, hk * g:(hk + 1) * g].double().reshape(g * Sq, D)
            w = torch.softmax(q @ kk.t() / math.sqrt(D), -1)
            out[b, hk * g:(hk + 1) * g] = (w @ vv).view(g, Sq, D)
    return {"O": out.view(B, Hq, D) if kind == "paged" else out}


def _exact_plan(case, h):
    p, S, n = case["page"], case["S"], len(h["free"])
    table, ring = [r[:] for r in h["table"]], h["free"][:]
    seq_out, added, slots, queue, freed = [], [], [], 0, []
    taken = 0
    for b, (s, new) in enumerate(zip(h["seq"], h["new"])):
        mine, took = table[b], 0
        held = -(-s // p)
        if new < 0:
            freed += mine[:held]
            seq_out.append(0)
        else:
            new = min(new, S)
            need = -(-(s + new) // p) - held
            if s + new <= case["max_pages"] * p:
                queue += need
                if need == 0 or queue <= h["count"]:
                    took = new
                    for k in range(need):
                        mine[held + k] = h["free"][(h["first"] + taken + k) % n]
                    taken += need
            seq_out.append(s + took)
        added.append(took)
        slots.append([mine[(s + t) // p] * p + (s + t) % p if t < took else -1 for t in range(S)])
    for i, q in enumerate(freed):
        ring[(h["first"] + h["count"] + i) % n] = q
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    return {"seq_len_out": i32(seq_out), "added": i32(added),
            "free_state_out": i32([(h["first"] + taken) % n, h["count"] - taken + len(freed)]),
            "free_pages": i32(ring), "page_table": i32(table), "slot": i32(slots)}
