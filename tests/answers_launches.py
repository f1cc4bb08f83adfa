"""Which kernels the operators of several answers to long prompts launch: host code on a recorder, no GPU.

record(calls) -> one (status, [(kernel, grid_x, grid_y, grid_z, block, lds), ...]) per call.  A call is
("rotate", B, S, Hq, Hkv, D, rot, interleaved, norm, row_stride, dtype), ("fork", B, H, D, max_pages, page, n, in_place, dtype),
("shared", B, Hq, Hkv, D, G, n, page, max_pages, page_stride or None, dtype), ("window", B, Hq, Hkv, S, D, window, sinks, dtype) or
("window_step", B, Hq, Hkv, D, n, page, max_pages, window, sinks, dtype)."""
import ctypes
import json
import os
import subprocess
import sys

from tests import launches


def record(calls, build_dir, lib=launches.LIB):
    launches.record([], build_dir)      # the recorder is built
    out = subprocess.run([sys.executable, "-m", "tests.answers_launches", f"{build_dir}/liblaunch_recorder.so", lib],
                         input=json.dumps(calls), text=True, capture_output=True, check=True, cwd=os.path.dirname(launches.HERE)).stdout
    got = json.loads(out)
    names = sorted({la[0] for _, ls in got for la in ls})
    nice = dict(zip(names, launches.plain(names)))
    return [(st, [(nice[la[0]], *la[1:]) for la in ls]) for st, ls in got]


def _main(rec, path):
    R = ctypes.CDLL(rec, mode=ctypes.RTLD_GLOBAL)
    R.recorded.restype = ctypes.c_char_p
    L = ctypes.CDLL(path)
    p, q, i64, f32 = ctypes.c_void_p(launches.PTR), ctypes.c_void_p(2 * launches.PTR), ctypes.c_int64, ctypes.c_float
    sz = ctypes.c_size_t(launches.HUGE)
    code = {"bf16": launches.BF16, "f32": launches.F32}
    out = []
    for fn, *c in json.load(sys.stdin):
        R.forget()
        if fn == "rotate":
            B, S, Hq, Hkv, D, rot, inter, norm, stride, dt = c
            w = p if norm else None
            st = L.attncache_rotate(p, w, w, p, p, None, p, p, p, None, None, B, S, Hq, Hkv, D, rot, i64(S * stride), i64(stride), 0, 0, i64(0),
                                    code[dt], inter, f32(0), f32(1), None)
        elif fn == "fork":
            B, H, D, width, page, n, in_place, dt = c
            o = p if in_place else q
            st = L.attncache_page_fork(q, p, p, q, p, o, o, o, q, q, B, H, D, width, n, page, i64(H * page * D), 0, 0, code[dt], p, sz, None)
        elif fn == "shared":
            B, Hq, Hkv, D, G, n, page, width, stride, dt = c
            st = L.attention_paged_shared(p, p, p, p, p, p, p, p, B, Hq, Hkv, D, G, n, page, width, i64(stride or Hkv * page * D), code[dt], f32(0), p, sz, None)
        elif fn == "window":
            B, Hq, Hkv, S, D, window, sinks, dt = c
            st = L.attention_window(p, p, p, p, None, None, B, Hq, Hkv, S, D, code[dt], window, sinks, f32(0), None)
        else:
            B, Hq, Hkv, D, n, page, width, window, sinks, dt = c
            st = L.attention_paged_window(p, p, p, p, p, p, B, Hq, Hkv, D, n, page, width, i64(Hkv * page * D), code[dt], window, sinks, f32(0), p, sz, None)
        rows = [r.split(" ") for r in R.recorded().decode().splitlines()]
        out.append((st, [(r[0], *map(int, r[1:])) for r in rows]))
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main(*sys.argv[1:])
