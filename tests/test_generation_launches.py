"""The launches of the operators of generation (host code on a recorder, no GPU): every kernel is reached by the GPU tests' cases, the
rules choose what measured best, and grids that do not fit one launch are split."""
import pytest

from tests import generation_launches as gl
from tests import test_gpu_cross_attention as cross
from tests import test_gpu_paged_attention as paged
from tests import test_gpu_pages as pages
from tests.test_launch_coverage import _kernels


def _paged(lens, Hq, Hkv, D, dt, page):
    width = max(1, max(-(-n // page) for n in lens))
    return ("paged", len(lens), Hq, Hkv, D, 100, page, width, dt)


def test_every_kernel_is_reached(tmp_path):
    calls = [("plan", B, S, width, page, n, in_place) for B, S, page, width, n, _ in pages.PLANS for in_place in (True, False)]
    calls += [("append", B, H, S, D, n, page, dt) for B, H, S, D, dt, n, page, _ in pages.APPENDS]
    calls += [_paged(paged.EDGES, 6, 2, D, dt, page) for D, dt in paged.TYPES for page in paged.PAGES]
    calls += [_paged(paged.EDGES * 5, 6, 2, D, dt, 16) for D, dt in paged.TYPES]
    calls += [_paged([70, 1, 600, 33], *h, 64, dt, 16) for h in paged.HEADS for dt in ("bf16", "f32")]
    calls += [_paged(lens, *t, 16) for lens in paged.RAGGED for t in paged.RAGGED_TYPES]
    calls += [_paged(*c) for c in paged.RUNS]
    calls += [("cross", *size, D, dt) for size in cross.SIZES for D, dt in cross.TYPES]
    seen = set()
    for call, (status, ls) in zip(calls, gl.record(calls, tmp_path)):
        assert status == 0, call
        seen |= {la[0] for la in ls}
    missing = _kernels("page_", "decode_", "cross_") - seen
    assert not missing, sorted(missing)


@pytest.mark.parametrize("call,kernels", [
    # us, the other way / this one
    (("plan", 64, 1, 128, 16, 5000, True), ["page_plan_kernel<256"]),                                # 1,024 threads 5.0 / 4.3
    (("plan", 300, 1, 128, 16, 5000, True), ["page_plan_kernel<1024"]),
    (("plan", 256, 1024, 128, 16, 5000, False), ["page_plan_kernel<256"]),                           # 10.6 / 5.3
    (("plan", 256, 1024, 128, 16, 5000, True), ["page_plan_kernel<256", "page_plan_kernel<1024"]),
    (("paged", 4, 32, 8, 64, 300, 16, 63, "bf16"), ["decode_unit_kernel"]),                          # 8.8 / 8.4
    (("paged", 4, 32, 8, 128, 300, 16, 63, "bf16"), ["decode_run_kernel", "decode_join_kernel"]),    # 13.8 / 10.1
    (("paged", 4, 32, 8, 128, 300, 16, 32, "bf16"), ["decode_unit_kernel"]),                         # 9.9 / 9.3
    (("paged", 8, 32, 8, 128, 300, 16, 63, "bf16"), ["decode_run_kernel", "decode_join_kernel"]),    # 19.1 / 17.1
    (("paged", 16, 32, 8, 128, 300, 16, 63, "bf16"), ["decode_unit_kernel"]),                        # 21.2 / 19.4
    (("paged", 4, 24, 8, 128, 300, 10, 50, "f32"), ["decode_run_kernel", "decode_join_kernel"]),     # 19.1 / 13.4
    (("paged", 4, 32, 8, 64, 300, 16, 125, "bf16"), ["decode_run_kernel", "decode_join_kernel"]),    # 12.3 / 9.8
    (("paged", 32, 32, 8, 128, 300, 16, 125, "bf16"), ["decode_unit_kernel"]),                       # 65.9 / 49.4
    (("paged", 128, 32, 8, 128, 9000, 16, 256, "bf16"), ["decode_run_kernel", "decode_join_kernel"]),   # 156 / 129
    (("cross", 32, 12, 12, 1, 1000, 64, "bf16"), ["decode_unit_kernel"]),                            # 17.8 / 15.6
    (("cross", 16, 8, 8, 32, 1000, 128, "bf16"), ["decode_unit_kernel"]),                            # 25.5 / 18.4
    (("cross", 16, 8, 8, 64, 1000, 128, "bf16"), ["cross_bf16_kernel<128, true"]),                   # 32.5 / 25.9
    (("cross", 64, 8, 8, 32, 1000, 64, "bf16"), ["cross_bf16_kernel<64"]),                           # 33.9 / 27.6
    (("cross", 8, 24, 8, 94, 333, 256, "f32"), ["cross_f32_kernel<4, 1, 2>"]),                       # 110 / 77
    (("cross", 8, 24, 8, 94, 333, 128, "f32"), ["cross_f32_kernel<2, 2, 2>"]),                       # 37.5 / 33.2
    (("cross", 2, 24, 8, 94, 333, 128, "f32"), ["decode_unit_kernel"]),                              # 16.9 / 16.5
    (("cross", 16, 8, 8, 64, 500, 128, "f32"), ["cross_f32_kernel<2, 2, 2>"]),                       # 45.4 / 32.0
    (("cross", 64, 8, 8, 20, 500, 128, "f32"), ["cross_f32_kernel<2, 2, 2>"]),                       # 68 / 54
    (("cross", 64, 8, 8, 40, 300, 128, "f32"), ["cross_f32_kernel<2, 2, 1>"]),                       # 67.4 / 55.8
    (("cross", 8, 24, 8, 1000, 1000, 128, "f32"), ["cross_f32_kernel<2, 2, 1>"]),                    # 382 / 340
], ids=str)
def test_the_kernels_that_measured_best_serve_the_call(tmp_path, call, kernels):
    (status, ls), = gl.record([call], tmp_path)
    assert status == 0 and len(ls) == len(kernels) and all(la[0].startswith(k) for la, k in zip(ls, kernels)), ls


@pytest.mark.parametrize("call,kernel,covered", [
    (("append", 1 << 20, 256, 7, 64, 9, 16, "bf16"), "page_append_kernel", (1 << 28) * 7 // 64),
    (("append", 1 << 20, 64, 31, 199, 9, 16, "f32"), "page_append_kernel", (1 << 26) * 31 // 2),
    (("cross", 1 << 20, 16, 16, 129, 5, 64, "bf16"), "cross_bf16_kernel", 2 << 24),
    (("cross", 1 << 10, 8, 1, 1 << 21, 100, 64, "bf16"), "cross_bf16_kernel", 1 << 27),
    (("cross", 1 << 16, 256, 256, 40, 3, 64, "f32"), "cross_f32_kernel", 1 << 24),
], ids=str)
def test_a_grid_that_does_not_fit_is_split(tmp_path, call, kernel, covered):
    (status, ls), = gl.record([call], tmp_path)
    assert status == 0 and len(ls) > 1 and all(la[0].startswith(kernel) for la in ls)
    assert sum(la[1] for la in ls) >= covered and all(la[1] * la[4] < 2**32 for la in ls)


@pytest.mark.parametrize("call", [
    ("plan", 1 << 22, 1, 500, 16, 1000, False), ("plan", 1, 1 << 25, 1 << 10, 1 << 17, 16000, False), ("plan", 1 << 22, 4000, 500, 16, 1000, True),
    ("paged", 1 << 23, 1, 1, 64, 9, 1, 1, "bf16"), ("paged", 1 << 23, 4, 4, 64, 9, 16, 1, "f32"), ("paged", 4096, 64, 8, 128, 9, 16, 60000, "bf16"),
    ("cross", 1 << 24, 16, 1, 1, 7, 64, "bf16"), ("cross", 1 << 20, 9, 1, 1, 30, 2, "f32"), ("cross", 1, 1, 1, 1 << 24, 1, 64, "bf16"),
], ids=str)
def test_the_largest_calls_fit(tmp_path, call):
    (status, ls), = gl.record([call], tmp_path)
    assert status == 0 and ls and all(la[2] < 65536 for la in ls)
