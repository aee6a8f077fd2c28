"""What the calls over the 8-bit cache and the 4-bit weights enqueue, without a GPU: launch_recorder.py's stand-in for the HIP runtime,
with the allocations counted too.

`record(calls)` runs them in a process of its own and returns [{"rc", "launches": [{"kernel", "grid", "block"}], "mallocs"}]."""
import ctypes
import json
import os
import subprocess
import sys
import tempfile

from launch_recorder import LIB, STAND_IN

MIB = 1 << 20
_stand_in = {}


def attn(H, Hkv, d, prefix, c, workspace_bytes=128 * MIB):
    return {"fn": "attn", "args": [H, Hkv, d, prefix, c, workspace_bytes]}


def append(H, Hkv, d, prefix, c):
    return {"fn": "append", "args": [H, Hkv, d, prefix, c]}


def linear(m, n, k, form="plain"):
    return {"fn": "linear", "args": [m, n, k, form]}


def pack(n, k):
    return {"fn": "pack", "args": [n, k]}


def names(result):
    """The launched kernels' names with their template arguments, in order."""
    assert result["rc"] == 0, result
    return [x["kernel"].split("::", 1)[1].split("(")[0] for x in result["launches"]]


def record(calls):
    if not _stand_in:
        tmp = _stand_in["folder"] = tempfile.TemporaryDirectory()   # goes with the process
        src, _stand_in["so"] = os.path.join(tmp.name, "stand_in.cpp"), os.path.join(tmp.name, "stand_in.so")
        with open(src, "w") as f:
            f.write(STAND_IN + '\nextern "C" int recorder_mallocs() { return n_mallocs; }\n')
        subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", src, "-o", _stand_in["so"], "-ldl"], check=True)
    job = {"so": _stand_in["so"], "calls": calls}
    r = subprocess.run([sys.executable, os.path.abspath(__file__)], input=json.dumps(job), capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    return json.loads(r.stdout)


def _serve():
    job = json.load(sys.stdin)
    i64, i32, f32, vp = ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_void_p
    rec = ctypes.CDLL(job["so"], mode=ctypes.RTLD_GLOBAL)
    lib = ctypes.CDLL(LIB)

    class Launch(ctypes.Structure):
        _fields_ = [("name", ctypes.c_char * 512), ("grid", ctypes.c_uint * 3), ("block", ctypes.c_uint * 3)]

    rec.recorder_launch.restype = ctypes.POINTER(Launch)
    lib.kvra_append_kv_q8.argtypes = [vp] * 8 + [i64, i64, i64, i32, i32, i32, f32, vp]
    lib.kvra_chunk_attn_q8.argtypes = [vp] * 5 + [i64, i64, i32, i32, i32, f32, vp, vp, i64, vp]
    lib.kvra_linear_w4.argtypes = [vp] * 7 + [i64, i64, i64, vp]
    lib.kvra_pack_w4.argtypes = lib.kvra_unpack_w4.argtypes = [vp, vp, vp, i64, i64, vp]
    P, out = 1 << 20, []   # (addresses are never read)

    def do_append(H, Hkv, d, prefix, c):
        return lib.kvra_append_kv_q8(*[P] * 8, prefix, c, prefix + c, H, Hkv, d, 1e4, None)

    def do_attn(H, Hkv, d, prefix, c, workspace_bytes):
        return lib.kvra_chunk_attn_q8(*[P] * 5, prefix, c, H, Hkv, d, 0.1, P, P, workspace_bytes, None)

    def do_linear(m, n, k, form):
        second = P if form == "swiglu" else None
        return lib.kvra_linear_w4(P, P, P, second, second, P if form == "residual" else None, P, m, n, k, None)

    def do_pack(n, k):
        return lib.kvra_pack_w4(P, P, P, n, k, None) or lib.kvra_unpack_w4(P, P, P, n, k, None)

    for c in job["calls"]:
        rec.recorder_reset(0, 0, 0)
        rc = locals()["do_" + c["fn"]](*c["args"])
        launches = []
        for i in range(rec.recorder_count()):
            la = rec.recorder_launch(i).contents
            launches.append({"kernel": la.name.decode(), "grid": list(la.grid), "block": list(la.block)})
        out.append({"rc": rc, "launches": launches, "mallocs": rec.recorder_mallocs()})
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _serve()
