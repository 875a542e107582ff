"""Runs checks of tests/token_cases.py on the CPU build of the kernels, whose library is argv[1]; the rest of the
arguments name the checks as function or function:case.  Started by test_tokens_emulated.py with AddressSanitizer preloaded."""
import ctypes
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path[:0] = [ROOT, os.path.join(ROOT, "tests")]
sys.modules["torch"] = None  # the binding does without it

import numpy as np  # noqa: E402

import paper_2411_19114_amd.binding as prep  # noqa: E402

libc = ctypes.CDLL(None)
libc.memalign.restype = ctypes.c_void_p
libc.memalign.argtypes = [ctypes.c_size_t, ctypes.c_size_t]


class Library(ctypes.CDLL):
    """The CPU build lacks the sources that it cannot compile; nobody here calls what they define."""

    def __getattr__(self, name):
        try:
            return super().__getattr__(name)
        except AttributeError:
            f = ctypes.CFUNCTYPE(ctypes.c_int)()
            setattr(self, name, f)
            return f


class Backend:
    """Buffers of exactly their size on the heap, so that the sanitizer sees what lies outside."""
    stream = 0

    def put(self, a):
        a = np.ascontiguousarray(a)
        p = libc.memalign(16, max(a.nbytes, 1))
        ctypes.memmove(p, a.tobytes(), a.nbytes)
        return p, a.shape, a.dtype

    def ptr(self, b):
        return b[0]

    def get(self, b):
        p, shape, dtype = b
        return np.frombuffer(ctypes.string_at(p, int(np.prod(shape)) * dtype.itemsize), dtype=dtype).reshape(shape).copy()

    def sync(self):
        pass


def main():
    prep.lib_path = lambda: sys.argv[1]
    ctypes.CDLL = Library
    prep.lib()
    import token_cases
    for what in sys.argv[2:]:
        name, _, case = what.partition(":")
        print(what, flush=True)
        args = [] if not case else [case == "True"] if case in ("True", "False") else [case]
        getattr(token_cases, name)(Backend(), *args)
    print("all passed", flush=True)


if __name__ == "__main__":
    main()
