"""Test infrastructure: makes the linear layers of tests/layers_layouts.py on the built libogq_layers.so, with record_launches.cpp preloaded in place of the HIP runtime, and prints which kernels they launched.
Run as a child process by test_layers_dispatch_of_linear.py; argument: the stand-in's path."""
import ctypes
import json
import sys

from paper_2002_11082_amd import layers as l
from tests.layers_layouts import LINEAR

A = 0x10000  # aligned; never looked at


def main():
    lib, stub = l.layers_lib(), ctypes.CDLL(sys.argv[1])
    stub.recorded_name.restype = ctypes.c_char_p
    stub.recorded_launches_of.restype = ctypes.c_uint64
    stub.recorded_kernels.restype = ctypes.c_size_t

    def counts():
        return {stub.recorded_name(i).decode(): stub.recorded_launches_of(i) for i in range(stub.recorded_kernels())}

    calls = []
    for tokens, outs, cols, pad in LINEAR:
        for dtype in (0, 1, 2):
            for transposed in (0, 1):
                before = counts()
                need = lib.ogq_linear_workspace(tokens, outs, cols, dtype, transposed)
                status = lib.ogq_linear(A, cols + pad, A, (outs if transposed else cols) + pad, transposed, tokens, outs, cols, dtype, A, 1, None, 0, A, outs, None, 0, A, need, None)
                made = [name for name, n in counts().items() if n != before.get(name, 0)]
                calls.append({"tokens": tokens, "outs": outs, "cols": cols, "pad": pad, "dtype": dtype, "transposed": transposed, "status": status, "kernels": made})
    print(json.dumps({"calls": calls, "kernels": list(counts())}))


main()
