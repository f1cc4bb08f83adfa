"""The index arithmetic of the generation kernels at the largest sizes that the entry points accept, against Python's integers: host
code, no GPU."""
import ctypes
import os
import subprocess

import pytest

from tests import generation_launches as gl

HERE = os.path.dirname(os.path.abspath(__file__))
TOP = 2**31 - 1


@pytest.fixture(scope="module")
def index(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("index") / "libgeneration_index.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fwrapv", "-shared", "-fPIC",
                    os.path.join(HERE, "generation_index.cpp"), "-o", out], check=True)
    return ctypes.CDLL(out)


@pytest.mark.parametrize("n", [1, 2, 1000, 2**30, 2**30 + 1, 1_200_000_000, 1_500_000_000, TOP])
def test_the_first_entry_of_a_ring(index, n):
    """A ring of pages of one token has up to 2^31 - 1 entries."""
    for first in (0, 1, n - 1, n // 2 + 1, n // 2 - 1, 1_100_000_000, TOP, -1, -n, 1 - n, -TOP - 1):
        assert index.ring_first(first, n) == first % n, first


RUN_WAVES = {"f32": 1024, "bf16": 2048}     # of decode_run_kernel
KEYS = {"f32": 16, "bf16": 32}              # of a block
MOST = 2**31 - 65536                        # what blocks of 16 keys add up to, two more a unit, has to stay below


def _units(call):
    """Units of 16 rows of a call, and keys of each."""
    kind, *c = call
    if kind == "paged":
        B, Hq, Hkv, _, _, page, width, dt = c
        rows, keys = Hq // Hkv, page * width
    else:
        B, Hq, Hkv, rows, keys, _, dt = c
        rows *= Hq // Hkv
    return B * Hkv * -(-rows // 16), keys, dt


@pytest.mark.parametrize("waves", sorted(RUN_WAVES.values()))
def test_runs_cover_all_blocks_and_no_more_than_their_waves(index, waves):
    for total in (1, waves // 2, waves // 2 + 1, waves, waves + 1, 2 * waves, 2 * waves + 1, 10**6, 2**30 - 1, 2**30, 2**30 + 1, 1_073_774_592,
                  1_082_130_432, 1_077_936_128, 1_500_000_000, MOST - 1):
        per = index.run_length(total, waves)
        assert per == (1 if 2 * total <= waves else max(2, -(-total // waves))), total
        assert per * waves >= total and (waves - 1) * per <= TOP
        assert (total - 1) // per < waves


# calls whose blocks number more than 2^30: shared pages of many tokens, many rows over few keys, many requests; the last two end just
# below what is refused
LARGEST = [("paged", 2048, 8, 8, 1, 1, 1 << 20, 1, "f32"), ("cross", 64, 1, 1, 1 << 20, 4096, 2, "f32"),
           ("paged", 1 << 19, 8, 8, 64, 9, 16, 509, "bf16"), ("paged", 4095, 8, 8, 64, 9, 1, (1 << 20) - 64, "f32"),
           ("cross", 1 << 10, 128, 128, 1, 262_080, 2, "f32")]


@pytest.mark.parametrize("call", LARGEST, ids=str)
def test_partial_results_of_the_largest_calls_lie_in_the_workspace(index, tmp_path, call):
    (status, ls), = gl.record([call], tmp_path)
    assert status == 0 and [la[0].split("<")[0] for la in ls] == ["decode_run_kernel", "decode_join_kernel"]
    units, keys, dt = _units(call)
    cost = -(-keys // KEYS[dt]) + 2
    waves, total = RUN_WAVES[dt], units * cost
    assert 2**30 < total and units * (-(-keys // 16) + 2) < MOST
    per = index.run_length(total, waves)
    for u in sorted({0, 1, units // 3, units // 2, units - 2, units - 1} | {min(units - 1, w * per // cost) for w in (1, waves // 2, waves - 1)}):
        start, end = u * cost, u * cost + cost - 3
        w0, w1 = start // per, end // per
        assert w1 < waves, u
        for w in range(w0, w1 + 1):
            assert index.partial_of(w, per, start) == 2 * w + (w * per <= start) < 2 * waves


JOIN_WAVES = 4 * 8192


@pytest.mark.parametrize("rows", [1025, JOIN_WAVES - 1, JOIN_WAVES, JOIN_WAVES + 1, 2 * JOIN_WAVES, 10**6, 10**8 + 1, 2**30, MOST - JOIN_WAVES, MOST - 1])
def test_each_row_of_the_join_is_one_waves(index, rows):
    """Rows are dealt in one piece each, so that a wave looks through the items once; the numbers of idle waves stay in 31 bits, too."""
    each = index.rows_of_a_wave(rows, JOIN_WAVES)
    waves = -(-rows // each)
    assert each >= 1 and waves <= JOIN_WAVES and (rows > JOIN_WAVES or each == 1)
    assert -(-waves // 4) * 4 * each <= TOP


@pytest.mark.parametrize("call", [
    ("paged", 1 << 23, 1, 1, 64, 9, 1, 1, "bf16"), ("paged", 1 << 23, 4, 4, 64, 9, 16, 1, "f32"), ("cross", 1 << 24, 16, 1, 1, 7, 64, "bf16"),
    ("paged", 1 << 19, 8, 8, 64, 9, 16, 509, "bf16"), ("paged", 3000, 16, 4, 64, 9, 16, 200, "bf16")], ids=str)
def test_lengths_are_looked_through_once_a_wave(index, tmp_path, call):
    """As many waves are launched as have a piece of the rows: each goes on from item to item, and none looks through the lengths again."""
    (status, ls), = gl.record([call], tmp_path)
    run, join = ls
    assert status == 0 and run[0].startswith("decode_run_kernel") and join[0].startswith("decode_join_kernel")
    rows = call[1] * call[2]
    waves = -(-rows // index.rows_of_a_wave(rows, JOIN_WAVES))
    assert join[1] * join[4] // 64 == -(-waves // 4) * 4 <= JOIN_WAVES


@pytest.mark.parametrize("S", [1, 2, 3, 4, 5, 100, 511, 512, 513, 1023, 1024, 1025, 4000, 10**5, 1 << 25])
def test_rows_of_a_workgroup_of_the_page_plan(index, S):
    """At most 16,384 workgroups sum the requests before their own, as far as slots of all requests fit any memory (2^40 of them)."""
    for B in (1, 2, 300, 4097, 16384, 16385, 100_000, (1 << 22) - 1, 1 << 22):
        rows = index.plan_rows(B, S)
        assert 1 <= rows <= 256 and rows * S <= TOP
        assert -(-B // rows) <= 16384 or B * S > 2**40


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,S", [(1 << 22, 4000), (1 << 22, 1), (40_000, 1500), (256, 1024), (2, 5000)])
def test_workgroups_of_the_page_plan(tmp_path, B, S, in_place):
    (status, ls), = gl.record([("plan", B, S, 500, 16, 1000, in_place)], tmp_path)
    assert status == 0 and len(ls) == 1 + in_place
    assert ls[0][1] <= 16384 + 1 and (B > 2 or ls[0][2] == 5)       # a row of its own is shared
