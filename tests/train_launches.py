"""launches.py for the calls whose arguments are structs: ``norm(post, pre, ...)`` and ``grads((data, rows, cols, ld, out, ld_out, count, dtype), ...)``
stand for them; ``mx`` as there."""
import ctypes as C
import json
import os
import subprocess
import sys

import launches
from launches import FAKE, LIB, Launch, mx  # noqa: F401


def norm(post, pre, gate=None, eps=1e-5):
    return {"norm": [post, pre, gate, eps]}


def grads(*items):
    return {"grads": [list(i) for i in items]}


def would_launch(calls):
    command = [sys.executable, os.path.abspath(__file__), launches._recorder(), LIB]
    out = json.loads(subprocess.run(command, input=json.dumps(calls), stdout=subprocess.PIPE, text=True, check=True).stdout)
    clear = launches._readable({l[0] for _, ls in out for l in ls})
    return [(rc, [Launch(clear[n], tuple(s[:3]), tuple(s[3:6]), s[6], bool(s[7])) for n, s in ls]) for rc, ls in out]


class _Norm(C.Structure):
    _fields_ = [("post", C.c_int32), ("pre", C.c_int32), ("vectors", C.c_void_p * 5), ("res_scale", C.c_float), ("post_eps", C.c_float), ("pre_eps", C.c_float)]


class _Grad(C.Structure):
    _fields_ = [("data", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("out", C.c_void_p), ("ld_out", C.c_int64),
                ("count", C.c_void_p), ("dtype", C.c_int32)]


def _argument(a):
    if isinstance(a, dict) and "norm" in a:
        post, pre, gate, eps = a["norm"]
        n = _Norm(post, pre, res_scale=1.0, post_eps=eps, pre_eps=eps)
        n.vectors[2] = gate
        return C.byref(n)
    if isinstance(a, dict) and "grads" in a:
        return (_Grad * max(len(a["grads"]), 1))(*[_Grad(*i) for i in a["grads"]])
    return launches._argument(a)


def _main():
    recorder = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
    library = C.CDLL(sys.argv[2])
    recorder.recorded_name.restype = C.c_char_p
    out = []
    for name, *args in json.load(sys.stdin):
        recorder.forget_launches()
        f = getattr(library, name)
        f.restype = C.c_size_t if name.endswith("_bytes") else C.c_int32
        rc = f(*[_argument(a) for a in args])
        made = []
        for i in range(recorder.recorded_launches()):
            shape = (C.c_uint * 8)()
            recorder.recorded_shape(i, shape)
            made.append((recorder.recorded_name(i).decode(), list(shape)))
        out.append((rc, made))
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main()
