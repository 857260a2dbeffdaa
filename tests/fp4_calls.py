"""What the calls on small caches answer, found without a GPU, as tests/cache_calls.py does for the others: libkvc.so on top of a HIP runtime that launches nothing, in a process of its own.

    answers([call, ...]) -> [(code, launches), ...]

A call is a dict: op "append_fp4", "attend_fp4", "weigh" or "evict" with N, d, ppb and fields of the argument records by their names, or op "unpack_fp4" with the call's arguments in a list."""
import ctypes as C
import json
import os
import subprocess
import sys
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def answers(calls):
    from cache_calls import _recorder
    from paper_2512_11920_amd import build

    with tempfile.TemporaryDirectory() as at:
        p = subprocess.run([sys.executable, os.path.abspath(__file__), _recorder(at), build.LIB], input=json.dumps(calls), capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr[-3000:]
    return [tuple(x) for x in json.loads(p.stdout)]


def _main(recorder, lib):
    sys.path.insert(0, ROOT)
    from paper_2512_11920_amd import kvc  # (the records alone: the library is not loaded by it)

    rec = C.CDLL(recorder, mode=C.RTLD_GLOBAL)
    L = C.CDLL(lib)
    records = {"append_fp4": kvc.Append, "attend_fp4": kvc.Attend, "weigh": kvc.Weigh, "evict": kvc.Evict}
    L.kvc_unpack_fp4.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
    out = []
    for c in json.load(sys.stdin):
        ctx = C.c_void_p()
        assert L.kvc_create(C.byref(ctx), (C.c_int32 * 4)(c.pop("N", 16), c.pop("d", 128), c.pop("ppb", 2), 3)) == 0
        rec.rec_clear()
        op = c.pop("op")
        if op == "unpack_fp4":
            code = L.kvc_unpack_fp4(ctx, *c["args"], None)
        else:
            a = records[op](**{k: tuple(v) if isinstance(v, list) else v for k, v in c.items()})
            code = getattr(L, "kvc_" + op)(ctx, C.byref(a), None)
        out.append((code, rec.rec_count()))
        L.kvc_destroy(ctx)
    print(json.dumps(out))


if __name__ == "__main__":
    _main(*sys.argv[1:])
