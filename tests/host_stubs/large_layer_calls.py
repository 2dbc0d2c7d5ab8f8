"""Test infrastructure: calls of the built libogq_layers.so whose grids are next to a launch's limits and beyond what one dimension takes, with limited_launches.cpp preloaded in place of the
HIP runtime; prints what became of them.  Run as a child process by test_layers_dispatch.py; argument: the stand-in's path."""
import ctypes
import json
import sys

from paper_2002_11082_amd import layers as l

A = 0x10000  # aligned; never looked at
MOST, BIG = (1 << 31) - 1, 1 << 60


def main():
    stub, lib = ctypes.CDLL(sys.argv[1]), l.layers_lib()
    for name in ("recorded_launches", "recorded_refused", "recorded_last_threads_in_all"):
        getattr(stub, name).restype = ctypes.c_uint64
    calls, wrong = 0, []

    def call(what, threads, f, *arguments):
        """threads: as many as the work of the call's last launch needs at least."""
        nonlocal calls
        before = stub.recorded_launches()
        status = f(*arguments)
        calls += 1
        if status != 0 or stub.recorded_launches() == before or stub.recorded_last_threads_in_all() < threads:
            wrong.append([what, status, stub.recorded_last_threads_in_all()])

    for dtype in (0, 1, 2):
        for rows, cols in ((MOST, 1), (MOST, 300), (1, MOST), (3, MOST), (1 << 22, 20000), ((1 << 22) + 1, 20000), (1 << 20, (1 << 20) - 200), (1 << 23, 100000)):
            at = f"{rows} {cols} {dtype}"
            call(f"norm {at}", rows * 64, lib.ogq_layer_norm_forward, A, cols, rows, cols, dtype, A, A, 1e-5, A, cols, A, A, None)
            call(f"norm backward {at}", 1, lib.ogq_layer_norm_backward, A, cols, A, cols, rows, cols, dtype, A, A, A, A, cols, A, A, 0, A, BIG, None)
            call(f"norm backward alone {at}", 1, lib.ogq_layer_norm_backward, A, cols, A, cols, rows, cols, dtype, None, A, A, A, cols, None, None, 0, None, 0, None)
            call(f"linear backward {at}", 1, lib.ogq_linear_backward, A, cols, rows, cols, dtype, 1, A, cols, A, cols, A, 1, A, BIG, None)
            call(f"embedding {at}", rows, lib.ogq_embedding_forward, A, 0, rows, A, cols, 100, cols, dtype, 1.0, A, cols, None)
            call(f"embedding gradient {at}", 64, lib.ogq_embedding_gradient, A, 1, 100, A, cols, rows, cols, dtype, 1.0, 0, A, cols, A, BIG, None)
            call(f"embedding gradient, sorted, {at}", 64, lib.ogq_embedding_gradient, A, 1, 300, A, cols, rows, cols, dtype, 1.0, 0, A, cols, A, BIG, None)
            call(f"embedding of nothing {at}", rows * cols // 16, lib.ogq_embedding_gradient, None, 1, 0, None, cols, rows, cols, dtype, 1.0, 0, A, cols, None, 0, None)
            call(f"distill {at}", rows * 256, lib.ogq_distill_gradient, A, cols, rows, cols, dtype, A, 0, A, 10, 1.0, None, A, A, cols, A, BIG, None)
        for number, cols in (((1 << 30) - 1, 1), ((1 << 30) - 1, 800), (1 << 29, 1900)):
            call(f"many tokens {number} {cols} {dtype}", 64, lib.ogq_embedding_gradient, A, 1, number, A, cols, 1000, cols, dtype, 1.0, 1, A, cols, A, BIG, None)
        for tokens, outs, cols in ((1, MOST - 127, 1), (1, MOST - 127, 300), (8, MOST - 127, 1), (9, (1 << 31) - 128, 1), (9, (1 << 31) - 128, 100), (1 << 19, (1 << 19) - 128, 1), ((1 << 19) - 129, 1 << 19, 1000),
                                   (MOST - 127, 64, 100), (1 << 19, 1 << 18, 100000)):
            for transposed in (0, 1):
                need = lib.ogq_linear_workspace(tokens, outs, cols, dtype, transposed)
                call(f"linear {tokens} {outs} {cols} {dtype} {transposed}", 1, lib.ogq_linear, A, cols, A, outs if transposed else cols, transposed, tokens, outs, cols, dtype, A, 1, None, 0,
                     A, outs, None, 0, A, need, None)
        for tokens, outs, cols in ((1, MOST, 1), (129, MOST - 127, 1), (1 << 19, 1 << 19, 1)):
            if lib.ogq_linear(A, cols, A, cols, 0, tokens, outs, cols, dtype, A, 1, None, 0, A, outs, None, 0, A, BIG, None) != -9:
                wrong.append([f"linear {tokens} {outs} {cols}", "not refused"])
    print(json.dumps({"calls": calls, "refused": stub.recorded_refused(), "wrong": wrong[:20]}))


main()
