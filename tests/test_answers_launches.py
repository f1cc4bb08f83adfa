"""The launches of the operators of several answers to long prompts (host code on a recorder, no GPU): every kernel is reached by the GPU
tests' cases, the rules choose what measured best, and grids that do not fit one launch are split."""
import pytest

from tests import answers_launches as al
from tests import test_gpu_page_fork as fork
from tests import test_gpu_rotate as rotate
from tests import test_gpu_shared_attention as shared
from tests import test_gpu_window_attention as window
from tests import test_gpu_window_step as step
from tests.test_launch_coverage import _kernels


def _pages(lens, page):
    return max(1, max(-(-n // page) for n in lens))


def _shared(groups, alone, Hq, Hkv, D, dt, page, n=100, stride=None):
    lens = [p + (n_ or 0) for p, rows in groups for n_ in rows] + list(alone)
    return ("shared", len(lens), Hq, Hkv, D, len(groups), n, page, max(_pages(lens, page), shared.width(len(lens), Hkv, D, dt, page)), stride, dt)


def test_every_kernel_is_reached(tmp_path):
    calls = [("rotate", B, S, Hq, Hkv, D, rot, i, n, (Hq + 2 * Hkv) * D, dt) for B, S, Hq, Hkv, D, dt, rot in rotate.SIZES for i in (0, 1) for n in (0, 1)]
    calls += [("fork", B, 2, 4, -(-hi // p) + 1, p, B * (-(-hi // p) + 1) + 20, i, "f32") for B, p, hi in fork.PLACES for i in (True, False)]
    calls += [("fork", 12, H, D, 8, 16, 116, False, dt) for H, D, dt, _ in fork.TYPES]
    calls += [("fork", B, 1, D, width, page, n, False, dt) for B, page, width, n in fork.LARGE for D, dt in ((64, "bf16"), (33, "f32"))]
    calls += [_shared(shared.EDGES, [0, 1, 50], 6, 2, D, dt, 16) for D, dt in shared.TYPES]
    calls += [_shared(*c) for c in shared.CASES]
    calls += [_shared(*c) for c in shared.MANY]
    calls += [("shared", 8, 4, 2, D, 2002, 100, 16, shared.width(8, 2, D, dt, 16), None, dt) for D, dt in shared.TYPES]
    calls += [_shared(shared.FAR, [], Hq, Hkv, D, "bf16", 16, 300, 1 << 24) for Hq, Hkv, D in shared.FAR_HEADS]
    calls += [_shared(shared.FAR_MANY, [], Hq, Hkv, D, "bf16", 16, 4400, 1 << 20) for Hq, Hkv, D in shared.FAR_HEADS]
    calls += [("window", *size, D, 7, 3, dt) for size in window.SIZES + window.MANY for D, dt in window.TYPES]
    calls += [("window_step", len(step.EDGES), 6, 2, D, 100, 16, _pages(step.EDGES, 16), 50, 9, dt) for D, dt in step.TYPES]
    calls += [("window_step", 5, 6, 2, D, 400, 16, _pages([2500], 16), 1000, 9, dt) for D, dt in step.TYPES]
    calls += [("window_step", len(c[0]), c[1], c[2], c[3], 100, c[5], _pages(c[0], c[5]), c[6], c[7], c[4]) for c in step.RUNS]
    calls += [("window_step", len(step.LENS), 32, 16, D, 100, 16, _pages(step.LENS, 16), 20, 5, dt) for D, dt in step.TYPES]
    calls += [("window_step", len(step.LENS), 8, 4, D, 100, 16, _pages(step.LENS, 16), 200, 5, dt) for D, dt in step.TYPES]
    calls += [("shared", 1203, 4, 1, D, 100, 100, 16, 2, None, dt) for D, dt in shared.TYPES]
    seen = set()
    for call, (status, ls) in zip(calls, al.record(calls, tmp_path)):
        assert status == 0, call
        seen |= {la[0] for la in ls}
    missing = _kernels("rotate_", "fork_", "shared_", "window_") - seen
    assert not missing, "\n".join(sorted(missing))


@pytest.mark.parametrize("call,kernels", [
    (("fork", 32, 8, 128, 127, 16, 5000, False, "bf16"), ["fork_small_kernel", "fork_copy_kernel"]),
    (("fork", 1025, 8, 128, 10, 16, 5000, False, "bf16"), ["fork_rows_kernel", "fork_flat_kernel", "fork_ring_kernel"]),
    (("fork", 16, 8, 128, 1025, 16, 5000, False, "bf16"), ["fork_rows_kernel", "fork_flat_kernel", "fork_ring_kernel"]),
    (("fork", 16, 8, 128, 10, 16, 65537, False, "bf16"), ["fork_rows_kernel", "fork_tables_kernel", "fork_ring_kernel"]),
    (("shared", 64, 32, 8, 128, 1, 1100, 16, 1100, None, "bf16"), ["shared_both_kernel<128, false, true>", "shared_join_kernel<false, 32, 1>"]),
    (("shared", 4, 32, 8, 128, 1, 1100, 16, 1100, None, "bf16"), ["shared_run_kernel<SharedBf16<128>, true>", "shared_join_kernel<false, 32, 4>"]),
    (("shared", 300, 32, 8, 128, 1, 1100, 16, 1100, None, "bf16"), ["shared_plan_kernel<32, 32, 1024, true>", "shared_both_kernel<128, false, false>", "shared_rows_kernel<false, 32>"]),
    (("shared", 64, 32, 8, 64, 1, 1100, 16, 1100, 1 << 22, "bf16"), ["shared_both_kernel<64, true, true>", "shared_join_kernel<false, 16, 1>"]),
    (("shared", 17, 24, 8, 128, 4, 1100, 10, 200, None, "f32"), ["shared_run_kernel<SharedF32<2, true>, true>", "shared_join_kernel<true, 32, 4>"]),
    (("shared", 61, 8, 8, 128, 1, 1100, 16, 16, None, "bf16"), ["decode_unit_kernel"]),
    (("shared", 10000, 8, 8, 128, 1, 1100, 16, 8, None, "bf16"), ["shared_wave_kernel"]),
    (("shared", 100, 8, 8, 128, 1, 1100, 16, 8, None, "bf16"), ["decode_unit_kernel"]),
    (("window_step", 256, 32, 8, 64, 300, 16, 600, 100, 16, "bf16"), ["window_step_wave_kernel"]),
    (("shared", 8, 8, 1, 128, 1, 1100, 16, 900, None, "bf16"), ["decode_run_kernel", "decode_join_kernel"]),
    (("shared", 64, 32, 8, 128, 0, 1100, 16, 1100, None, "bf16"), ["decode_run_kernel", "decode_join_kernel"]),
    (("window", 4, 32, 8, 4096, 128, 1024, 4, "bf16"), ["window_bf16_kernel<128>"]),
    (("window_step", 4, 32, 8, 64, 300, 16, 600, 500, 16, "bf16"), ["window_step_unit_kernel"]),
    (("window_step", 128, 32, 8, 128, 300, 16, 12500, 4096, 4, "bf16"), ["window_step_run_kernel", "window_step_join_kernel"]),
], ids=lambda x: "-".join(map(str, x)) if isinstance(x, tuple) else None)
def test_the_kernels_that_measured_best_serve_the_call(tmp_path, call, kernels):
    (status, ls), = al.record([call], tmp_path)
    assert status == 0 and len(ls) == len(kernels) and all(la[0].startswith(k) for la, k in zip(ls, kernels)), ls


@pytest.mark.parametrize("call,kernel,covered", [
    (("rotate", 1 << 20, 1 << 10, 2, 1, 128, 128, 0, 0, 512, "bf16"), "rotate_kernel", 1 << 28),
    (("window", 1 << 18, 64, 64, 200, 64, 10, 0, "bf16"), "window_bf16_kernel", (1 << 24) * 2),
    (("window", 1 << 18, 64, 64, 40, 64, 10, 0, "f32"), "window_f32_kernel", 1 << 24),
    (("window", 1, 1 << 20, 1, 1, 64, 10, 0, "bf16"), "window_bf16_kernel", 1 << 18),
    (("window", 9, 1 << 20, 1, 1, 64, 10, 0, "f32"), "window_f32_kernel", 9 << 18),
    (("window", 64, 64, 1, 1 << 18, 64, 10, 0, "bf16"), "window_bf16_kernel", 64 << 17),
], ids=lambda x: "-".join(map(str, x)) if isinstance(x, tuple) else None)
def test_a_grid_that_does_not_fit_is_split(tmp_path, call, kernel, covered):
    (status, ls), = al.record([call], tmp_path)
    assert status == 0 and all(la[0].startswith(kernel) for la in ls)
    assert sum(la[1] * la[2] for la in ls) >= covered and all(la[1] * la[4] < 2**32 for la in ls)


def test_the_most_rows_of_shared_prefixes_fit_a_launch(tmp_path):
    (status, ls), = al.record([("shared", 1 << 20, 32, 1, 64, 1, 10, 16, 1, None, "bf16")], tmp_path)
    assert status == 0 and all(la[1] * la[4] < 2**32 for la in ls)
