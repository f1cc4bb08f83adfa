"""Which kernels the operators of generation launch, as launches.py has it for the others: host code on a recorder, no GPU.

record(calls) -> one (status, [(kernel, grid_x, grid_y, grid_z, block, lds), ...]) per call.  A call is
("plan", B, S, max_pages, page, n, in_place), ("append", B, H, S, D, n, page, "bf16"|"f32"),
("paged", B, Hq, Hkv, D, n, page, max_pages, dtype) or ("cross", B, Hq, Hkv, Sq, Sk, D, dtype)."""
import ctypes
import json
import subprocess
import sys

from tests import launches


def record(calls, build_dir, lib=launches.LIB):
    launches.record([], build_dir)      # the recorder is built
    rec = f"{build_dir}/liblaunch_recorder.so"
    out = subprocess.run([sys.executable, "-m", "tests.generation_launches", rec, lib], input=json.dumps(calls), text=True,
                         capture_output=True, check=True, cwd=launches.os.path.dirname(launches.HERE)).stdout
    got = json.loads(out)
    names = sorted({la[0] for _, ls in got for la in ls})
    nice = dict(zip(names, launches.plain(names)))
    return [(st, [(nice[la[0]], *la[1:]) for la in ls]) for st, ls in got]


def _main(rec, path):
    R = ctypes.CDLL(rec, mode=ctypes.RTLD_GLOBAL)
    R.recorded.restype = ctypes.c_char_p
    L = ctypes.CDLL(path)
    p, i64, f32, sz = ctypes.c_void_p(launches.PTR), ctypes.c_int64, ctypes.c_float(0), ctypes.c_size_t(launches.HUGE)
    code = {"bf16": launches.BF16, "f32": launches.F32}
    out = []
    for fn, *c in json.load(sys.stdin):
        R.forget()
        if fn == "plan":
            B, S, width, page, n, in_place = c
            other = p if in_place else ctypes.c_void_p(2 * launches.PTR)
            st = L.attncache_page_plan(p, p, p, p, p, other, other, other, p, B, S, width, page, n, None)
        elif fn == "append":
            B, H, S, D, n, page, dt = c
            st = L.attncache_page_append(p, p, p, p, p, B, H, S, D, n, page, i64(H * page * D), code[dt], None)
        elif fn == "paged":
            B, Hq, Hkv, D, n, page, width, dt = c
            st = L.attention_paged(p, p, p, p, p, p, B, Hq, Hkv, D, n, page, width, i64(Hkv * page * D), code[dt], f32, p, sz, None)
        else:
            B, Hq, Hkv, Sq, Sk, D, dt = c
            st = L.attention_cross(p, p, p, p, None, None, B, Hq, Hkv, Sq, Sk, D, code[dt], f32, p, sz, None)
        rows = [r.split(" ") for r in R.recorded().decode().splitlines()]
        out.append((st, [(r[0], *map(int, r[1:])) for r in rows]))
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main(*sys.argv[1:])
