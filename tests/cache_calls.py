"""What the decode-step calls answer, found without a GPU: libkvc.so on top of a HIP runtime that launches nothing (tests/cache_recorder.cpp), in a
process of its own, called with addresses nobody looks at.

    answers([call, ...]) -> [(code, launches, pool_out and desc_out of the last compaction), ...]

A call is a dict: op "compact" with pool, desc, pool_out, desc_out, used, work (addresses), pool_bytes, out_bytes, pages (descriptors) and work_bytes; op
"adopt" with pool, desc, pool_bytes and pages; or op "attend" with N, d, ppb and fields of kvc_attend_t by their names."""
import ctypes as C
import json
import os
import subprocess
import sys
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HOST, UNREACHABLE, SEEN_LOWER = 1 << 45, 1 << 46, 1 << 44


def _recorder(at):
    versions, out = os.path.join(at, "v"), os.path.join(at, "rec.so")
    with open(versions, "w") as f:
        f.write("hip_4.2 { global: *; };\n")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-Wno-attributes",
                    "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2512_11920_amd", "csrc"),
                    "-Wl,-soname,libamdhip64.so.7", f"-Wl,--version-script={versions}", "-o", out, os.path.join(ROOT, "tests", "cache_recorder.cpp")], check=True)
    return out


def answers(calls):
    from paper_2512_11920_amd import build

    with tempfile.TemporaryDirectory() as at:
        p = subprocess.run([sys.executable, os.path.abspath(__file__), _recorder(at), build.LIB], input=json.dumps(calls), capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr[-3000:]
    return [tuple(x) for x in json.loads(p.stdout)]


def _main(recorder, lib):
    sys.path.insert(0, ROOT)
    from paper_2512_11920_amd.kvc import Attend  # (the record alone: the library is not loaded by it)

    rec = C.CDLL(recorder, mode=C.RTLD_GLOBAL)
    rec.rec_pool_out.restype = rec.rec_desc_out.restype = C.c_void_p
    L = C.CDLL(lib)
    L.kvc_attend_workspace.restype = L.kvc_compact_workspace.restype = C.c_uint64
    vp, u64, out = C.c_void_p, C.c_uint64, []
    for c in json.load(sys.stdin):
        ctx = vp()
        assert L.kvc_create(C.byref(ctx), (C.c_int32 * 4)(c.get("N", 16), c.get("d", 128), c.get("ppb", 1), 3)) == 0
        rec.rec_clear()
        if c["op"] == "attend":
            a = Attend(**{k: v for k, v in c.items() if k not in ("op", "N", "d", "ppb")})
            code = L.kvc_attend(ctx, C.byref(a), None)
        elif c["op"] == "adopt":
            code = L.kvc_adopt_pool(ctx, vp(c["pool"]), u64(c["pool_bytes"]), vp(c["desc"]), u64(c["pages"]), vp(1 << 20), None)
        else:
            assert L.kvc_bind_pool(ctx, vp(c["pool"]), u64(c["pool_bytes"]), vp(c["desc"]), u64(c["pages"])) == 0
            work_bytes = c.get("work_bytes", L.kvc_compact_workspace(u64(c["pool_bytes"])))
            code = L.kvc_compact_pool(ctx, vp(c["pool_out"]), u64(c["out_bytes"]), vp(c["desc_out"]), vp(c["used"]), vp(c["work"]), u64(work_bytes), None)
        out.append((code, rec.rec_count(), rec.rec_pool_out(), rec.rec_desc_out()))
        L.kvc_destroy(ctx)
    print(json.dumps(out))


if __name__ == "__main__":
    _main(*sys.argv[1:])
