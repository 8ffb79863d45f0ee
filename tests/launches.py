"""What the library would launch, found out without a GPU.

``would_launch(calls)`` makes C calls in a process of its own in which the HIP runtime's launch calls are those of launch_recorder.cpp: the
library's host side runs as it is, and every kernel is written down instead of run.  A call is ``(name, *arguments)``: whole numbers (pointers
among them; nothing is dereferenced), floats, ``None``, and ``mx(rows, cols)`` for an MXFP4 matrix.
"""
import atexit
import ctypes as C
import functools
import json
import os
import re
import shutil
import subprocess
import sys
import tempfile
from typing import NamedTuple, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(HERE), "paper_2410_20046_amd", "libdqrm.so")
FAKE = 0x10000  # non-null, aligned, never dereferenced


class Launch(NamedTuple):
    kernel: str
    grid: Tuple[int, int, int]
    block: Tuple[int, int, int]
    shared: int
    failed: bool


def mx(rows, cols, codes=FAKE, scales=FAKE):
    return {"mx": [rows, cols, codes, scales]}


@functools.lru_cache(maxsize=None)
def _recorder():
    folder = tempfile.mkdtemp()
    atexit.register(shutil.rmtree, folder, ignore_errors=True)
    out = os.path.join(folder, "recorder.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", out, os.path.join(HERE, "launch_recorder.cpp")], check=True)
    return out


def would_launch(calls):
    """[(return code, [Launch, ...])] of the calls."""
    out = _ask(calls)["calls"]
    clear = _readable({l[0] for _, ls in out for l in ls})
    return [(rc, [Launch(clear[n], tuple(s[:3]), tuple(s[3:6]), s[6], bool(s[7])) for n, s in ls]) for rc, ls in out]


def library_kernels():
    """The names of all kernels that the library has."""
    return set(_readable(set(_ask([])["kernels"])).values())


def _ask(calls):
    command = [sys.executable, os.path.abspath(__file__), _recorder(), LIB]
    return json.loads(subprocess.run(command, input=json.dumps(calls), stdout=subprocess.PIPE, text=True, check=True).stdout)


def _readable(names):
    """Without types of arguments and namespaces; element types as they are in C (the demangler may not know the 16-bit ones)."""
    names = sorted(names)
    if not names:
        return {}
    known = "\n".join(n.replace("IDF16b", "I4bf16").replace("IDF16_", "I4half") for n in names)
    plain = subprocess.run(["c++filt"], input=known, stdout=subprocess.PIPE, text=True, check=True).stdout.splitlines()
    short = [re.sub(r"^void ", "", re.sub(r"\([^()]*\)$", "", p)) for p in plain]
    return {n: p.replace("dqrm_mx::", "").replace("(anonymous namespace)::", "").replace("(FewSource)", "") for n, p in zip(names, short)}


class _Mx(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("codes", C.c_void_p), ("scales", C.c_void_p)]


def _argument(a):
    if isinstance(a, dict):
        return C.byref(_Mx(*a["mx"]))
    return C.c_float(a) if isinstance(a, float) else C.c_int64(a or 0)


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
        launches = []
        for i in range(recorder.recorded_launches()):
            shape = (C.c_uint * 8)()
            recorder.recorded_shape(i, shape)
            launches.append((recorder.recorded_name(i).decode(), list(shape)))
        out.append((rc, launches))
    recorder.known_kernel.restype = C.c_char_p
    json.dump({"calls": out, "kernels": [recorder.known_kernel(i).decode() for i in range(recorder.known_kernels())]}, sys.stdout)


if __name__ == "__main__":
    _main()
