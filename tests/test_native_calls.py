"""Entry points of many arguments called by the native module: the same statuses as by ctypes, numbers that do not fit are refused (no GPU)."""
import ctypes

import pytest
import torch  # noqa: F401  (before the native module, which needs its libraries)

from paper_2510_25979_amd import binding, _tensor_arg
from tests.test_answers_arguments import BF16, P

BIG = 1 << 60
# refused for one reason each, so that every argument is looked at before any launch: (entry, arguments, status)
CALLS = [("attncache_rotate", [P] * 11 + [2, 3, 4, 2, 64, 64, 3 * 8 * 64, 8 * 64, 5, 16, 2 * 16 * 64, BF16, 0, 1e-6, 1.0, None]),
         ("attncache_page_fork", [P] * 10 + [2, 2, 64, 4, 20, 16, 2 * 16 * 64, 0, 0, BF16, P, 0, None]),
         ("attention_paged_shared", [P] * 8 + [2, 4, 2, 64, 1, 20, 16, 4, 2 * 16 * 64, BF16, 0.0, P, 0, None]),
         ("attention_window", [P] * 4 + [None, None, 2, 4, 2, 30, 64, BF16, 7, 1, 0.0, None]),
         ("attention_paged_window", [P] * 6 + [2, 4, 2, 64, 20, 16, 4, 2 * 16 * 64, BF16, 7, 1, 0.0, P, 0, None])]


@pytest.mark.parametrize("name,args", CALLS, ids=[c[0] for c in CALLS])
def test_every_argument_arrives(name, args):
    """B = 0 and every other argument in turn out of range: what the library says, by either way."""
    L = binding.lib()
    by_ctypes, native = getattr(L, name), binding._call(name)
    assert native.func is getattr(_tensor_arg, name)
    batch = next(i for i, a in enumerate(args) if a == 2)
    seen = set()
    for i in range(len(args) - 1):
        for odd in (None, P + 8) if args[i] == P or args[i] is None else (-1, 0, 3, 1 << 30, BIG if args[i] == 2 * 16 * 64 else 77):
            if isinstance(args[i], float):
                odd = float("nan") if odd is None or odd < 0 else float("inf") if odd == 0 else -1.0
            call = args[:batch] + [0] + args[batch + 1:]
            call[i] = odd
            if i == batch and odd > 0 or args[i + 1:] == [None] and args[i] == 0 and odd < 0:     # (a size of a workspace has no sign)
                continue
            status = native(*call)
            assert status == by_ctypes(*call)
            seen.add(status)
    assert len(seen) > 1 and 0 in seen


@pytest.mark.parametrize("name,args", CALLS, ids=[c[0] for c in CALLS])
def test_what_does_not_fit_is_refused(name, args):
    native, ints = binding._call(name), [i for i, a in enumerate(args) if isinstance(a, int) and a != P]
    for wrong in (args[:-1], args + [0], []):
        with pytest.raises(TypeError):
            native(*wrong)
    for i in ints:
        with pytest.raises(OverflowError):
            native(*args[:i], 1 << 70, *args[i + 1:])
        with pytest.raises(TypeError):
            native(*args[:i], 1.5, *args[i + 1:])
    with pytest.raises(OverflowError):     # 32 bits
        native(*args[:ints[0]], 1 << 31, *args[ints[0] + 1:])
    with pytest.raises(TypeError):
        native("x", *args[1:])
    with pytest.raises(ValueError):
        getattr(_tensor_arg, name)(None, *args)


def test_without_the_native_module(monkeypatch):
    monkeypatch.setattr(binding, "_native", None)
    monkeypatch.setattr(binding.lib(), "calls", {})
    for name, args in CALLS:
        f = binding._call(name)
        assert isinstance(f, ctypes._CFuncPtr) and f(*args[:10], *[0] * (len(args) - 10)) < 0
