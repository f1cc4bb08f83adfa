"""What the operators of generation refuse, before anything is launched.  Host code, no GPU: the pointers are never followed."""
import ctypes

import pytest
import torch

OK, NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, MEMSPACE = 0, -1, -2, -3, -4, -6, -9
P, F32, F16, BF16 = 1 << 20, 0, 1, 2
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    from paper_2510_25979_amd import binding
    return binding.lib()


def _call(fn, names, given, **change):
    values = dict(zip(names.split(), given))
    assert not set(change) - set(values), change
    values.update(change)
    return fn(*values.values())


def _plan(L, **change):
    return _call(L.attncache_page_plan, "seq new state ring table seq_out added state_out slot B S max_pages page n stream",
                 [P] * 9 + [4, 2, 8, 16, 100, None], **change)


def _append(L, **change):
    return _call(L.attncache_page_append, "K V slot kp vp B H S D n page stride dtype stream",
                 [P] * 5 + [4, 2, 3, 64, 10, 16, 2 * 16 * 64, BF16, None], **change)


def _paged(L, **change):
    return _call(L.attention_paged, "Q kp vp table len O B Hq Hkv D n page max_pages stride dtype scale ws ws_bytes stream",
                 [P] * 6 + [4, 8, 2, 64, 10, 16, 8, 2 * 16 * 64, BF16, 0.0, P, BIG, None], **change)


def _cross(L, **change):
    return _call(L.attention_cross, "Q K V O sel len B Hq Hkv Sq Sk D dtype scale ws ws_bytes stream",
                 [P] * 6 + [4, 8, 2, 3, 50, 64, BF16, 0.0, P, BIG, None], **change)


@pytest.mark.parametrize("call,change,status", [
    *[(_plan, {n: None}, NULL) for n in "seq new state ring table seq_out added state_out slot".split()],
    *[(_plan, {n: 0}, SHAPE) for n in "S max_pages page n".split()],
    (_plan, dict(B=-1), SHAPE), (_plan, dict(n=1 << 27), SHAPE), (_plan, dict(max_pages=1 << 27, B=1), SHAPE),
    (_plan, dict(max_pages=1 << 20, B=1 << 11), SHAPE), (_plan, dict(S=(1 << 25) + 1), SHAPE), (_plan, dict(max_pages=(1 << 26) + 1, B=1), SHAPE), (_plan, dict(B=(1 << 22) + 1), SHAPE),
    (_plan, dict(max_pages=((1 << 31) - 4096) // 3 + 1, B=3, page=1), SHAPE),
    (_plan, dict(B=0), OK), (_plan, dict(B=0, seq=None), OK),
    *[(_append, {n: None}, NULL) for n in "K V slot kp vp".split()],
    *[(_append, {n: P + 8}, ALIGN) for n in "K V kp vp".split()],
    *[(_append, {n: 0}, SHAPE) for n in "H S D n page".split()],
    (_append, dict(B=-1), SHAPE), (_append, dict(D=96), SHAPE), (_append, dict(D=257, dtype=F32, stride=BIG), SHAPE),
    (_append, dict(dtype=F16), DTYPE), (_append, dict(dtype=7), DTYPE), (_append, dict(stride=2 * 16 * 64 - 1), SHAPE),
    (_append, dict(stride=2 * 16 * 64 + 4), ALIGN), (_append, dict(D=100, dtype=F32, stride=2 * 16 * 100 + 2), ALIGN),
    (_append, dict(n=1 << 27), SHAPE), (_append, dict(stride=1 << 60), SHAPE), (_append, dict(B=1 << 20, S=1 << 11), SHAPE),
    (_append, dict(H=2**31 - 1, page=2**31 - 1, n=1, stride=2**63 - 1), SHAPE), (_append, dict(B=0), OK),
    *[(_paged, {n: None}, NULL) for n in "Q kp vp table len O ws".split()],
    *[(_paged, {n: P + 8}, ALIGN) for n in "Q kp vp O ws".split()],
    *[(_paged, {n: 0}, SHAPE) for n in "Hq Hkv D n page max_pages".split()],
    (_paged, dict(Hq=9), SHAPE), (_paged, dict(B=-1), SHAPE), (_paged, dict(D=32), SHAPE), (_paged, dict(dtype=F16), DTYPE),
    (_paged, dict(scale=-1.0), SHAPE), (_paged, dict(scale=float("nan")), SHAPE), (_paged, dict(ws_bytes=1000), WORKSPACE),
    (_paged, dict(max_pages=1 << 27), SHAPE), (_paged, dict(max_pages=(1 << 26) + 1, B=1, Hq=1, Hkv=1), SHAPE), (_paged, dict(B=1 << 16, max_pages=1 << 20), SHAPE),
    (_paged, dict(stride=2 * 16 * 64 - 8), SHAPE), (_paged, dict(stride=2 * 16 * 64 + 4), ALIGN), (_paged, dict(B=0), OK),
    *[(_cross, {n: None}, NULL) for n in "Q K V O ws".split()],
    *[(_cross, {n: P + 8}, ALIGN) for n in "Q K V O ws".split()],
    *[(_cross, {n: 0}, SHAPE) for n in "Hq Hkv Sq Sk D".split()],
    (_cross, dict(Hq=9), SHAPE), (_cross, dict(B=-1), SHAPE), (_cross, dict(D=96), SHAPE), (_cross, dict(dtype=F16), DTYPE),
    (_cross, dict(dtype=F32, D=257), SHAPE), (_cross, dict(scale=-1.0), SHAPE), (_cross, dict(ws_bytes=1000), WORKSPACE),
    (_cross, dict(Sq=1 << 23), SHAPE), (_cross, dict(Sk=(1 << 30) + 1, B=1, Hq=1, Hkv=1), SHAPE), (_cross, dict(dtype=F32, Sq=1 << 20, Sk=1 << 20), SHAPE), (_cross, dict(B=0), OK),
], ids=lambda x: x.__name__[1:] if callable(x) else str(x))
def test_refusals(L, call, change, status):
    assert call(L, **change) == status


def test_workspace_sizes():
    from paper_2510_25979_amd import binding as ac
    paged, cross = ac.attention_paged_workspace_bytes, ac.attention_cross_workspace_bytes
    assert paged(0, 8, 2, 64) == paged(1, 8, 3, 64) == paged(1, 8, 0, 64) == paged(1, 8, 2, -64) == 0
    assert paged(1, 8, 2, 64) == paged(1000, 8, 2, 64) < paged(1, 8, 1, 64) < paged(1, 8, 1, 128)
    assert cross(1, 8, 2, 1, 100, 64, torch.bfloat16) == paged(1, 8, 2, 64) == cross(1, 8, 2, 1, 100, 64)
    assert cross(64, 32, 8, 256, 1000, 64, torch.bfloat16) == cross(64, 32, 8, 256, 1000, 64, torch.float32) == 0
    assert cross(8, 32, 8, 25, 1000, 64, torch.float32) == 0 < cross(8, 32, 8, 25, 1000, 64, torch.bfloat16) == cross(8, 32, 8, 25, 1000, 64)
    assert cross(0, 8, 2, 1, 100, 64) == cross(1, 8, 3, 1, 100, 64) == cross(1, 8, 2, 1, 100, 65, torch.bfloat16) == 0


def test_the_binding_names_what_is_wrong():
    from paper_2510_25979_amd import binding as ac
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q, pages, kv = torch.zeros(2, 4, 64).bfloat16(), torch.zeros(5, 2, 16, 64).bfloat16(), torch.zeros(2, 2, 3, 64).bfloat16()
    for call, what in (
            (lambda: ac.attention_paged(q, pages, pages, i32(2, 3), i32(2), q, q), "Q must be a CUDA tensor"),
            (lambda: ac.attention_paged(q[0], pages, pages, i32(2, 3), i32(2), q, q), "Q must be"),
            (lambda: ac.attention_paged(q.half(), pages, pages, i32(2, 3), i32(2), q, q), "unsupported dtype"),
            (lambda: ac.attncache_page_append(kv[0], kv, i32(2, 3), pages, pages), "K and V must be"),
            (lambda: ac.attncache_page_append(kv, kv, i32(2, 3), pages, pages), "K must be a CUDA tensor"),
            (lambda: ac.attncache_page_plan(i32(2), i32(2), i32(2), i32(9), i32(2), i32(2), i32(2), i32(2), i32(2, 1), page_size=4),
             "page_table must be"),
            (lambda: ac.attncache_page_plan(i32(2), i32(2), i32(2), i32(9), i32(2, 3), i32(2), i32(2), i32(2), i32(2, 1), page_size=4),
             "seq_len must be a CUDA tensor"),
            (lambda: ac.attention_cross(kv, kv[0], kv, kv), "Q must be"), (lambda: ac.attention_cross(kv, kv, kv, kv), "Q must be a CUDA"),
            (lambda: ac._pages(pages, pages[:4], pages.dtype, 2, 64), "k_pages and v_pages must be"),
            (lambda: ac._pages(pages, pages, pages.dtype, 3, 64), "k_pages and v_pages must be"),
            (lambda: ac._pages(pages.transpose(1, 2), pages.transpose(1, 2), pages.dtype, 16, 64), "contiguous within a page"),
            (lambda: ac._pages(pages[::2], pages[:3], pages.dtype, 2, 64), "one page stride"),
            (lambda: ac._pages(pages[:1].expand(5, -1, -1, -1), pages[:1].expand(5, -1, -1, -1), pages.dtype, 2, 64), "contiguous within"),
            (lambda: ac._pages(pages, pages, pages.dtype, 2, 64), "k_pages must be a CUDA tensor")):
        with pytest.raises(ValueError, match=what):
            call()


def test_host_memory_is_refused_where_there_is_a_gpu(L):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU to tell memory apart")
    host = (ctypes.c_char * 4096)()
    at = ctypes.addressof(host) + 15 & ~15
    for call in (_plan, _append, _paged, _cross):
        assert call(L, **{"slot" if call in (_plan, _append) else "O": at}) == MEMSPACE
