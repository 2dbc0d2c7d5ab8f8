"""Test infrastructure: makes the calls below on the built libogq_layers.so, with record_launches.cpp preloaded in place of the HIP runtime, and
prints what they launched.  Run as a child process by test_layers_dispatch.py; argument: the stand-in's path."""
import ctypes
import json
import sys

from paper_2002_11082_amd import layers as l

A = 0x10000  # aligned; never looked at
SIZES = (1, 2, 7, 31, 33, 128, 200, 400, 513, 900, 1500, 2049, 4097, 6000, 8192, 12000, 16384, 25000, 33000, 60000, 100000, 140000)
BIG = 1 << 50


def main():
    lib, size = l.layers_lib(), ctypes.c_size_t
    stub = ctypes.CDLL(sys.argv[1])
    stub.recorded_name.restype = ctypes.c_char_p
    for name in ("recorded_launches", "recorded_launches_of", "recorded_unknown"):
        getattr(stub, name).restype = ctypes.c_uint64
    stub.recorded_kernels.restype = size
    calls, wrong = 0, []

    def call(what, least, most, f, *arguments):
        nonlocal calls
        before = stub.recorded_launches()
        status = f(*arguments)
        made = stub.recorded_launches() - before
        calls += 1
        if status != 0 or not least <= made <= most or stub.recorded_last_threads() > 1024 or stub.recorded_last_blocks() == 0:
            wrong.append([what, status, made])

    for dtype in (0, 1, 2):
        for rows in (1, 7, 200, 1000, 8192, 100000):
            for cols in SIZES:
                at = f"{rows} {cols} {dtype}"
                call(f"norm {at}", 1, 1, lib.ogq_layer_norm_forward, A, cols, rows, cols, dtype, A, A, 1e-5, A, cols, A, A, None)
                call(f"norm backward {at}", 1, 3, lib.ogq_layer_norm_backward, A, cols, A, cols, rows, cols, dtype, A, A, A, A, cols, A, A, 0, A, BIG, None)
                call(f"norm backward alone {at}", 1, 1, lib.ogq_layer_norm_backward, A, cols, A, cols, rows, cols, dtype, None, A, A, A, cols, None, None, 0, None, 0, None)
                call(f"linear backward {at}", 1, 2, lib.ogq_linear_backward, A, cols, rows, cols, dtype, 1, A, cols, A, cols, A, 1, A, BIG, None)
                call(f"sums {at}", 1, 2, lib.ogq_linear_backward, A, cols, rows, cols, dtype, 4, None, 0, None, 0, A, 0, A, BIG, None)
                call(f"embedding {at}", 1, 1, lib.ogq_embedding_forward, A, 0, rows, A, cols, 1000, cols, dtype, 1.0, A, cols, None)
                for accumulate in (0, 1):
                    call(f"embedding gradient {at}", 1 if rows <= 256 else 2, 1 if rows <= 256 else 5, lib.ogq_embedding_gradient, A, 1, rows, A, cols, 1000, cols, dtype, 1.0, accumulate, A, cols, A, BIG, None)
                call(f"distill {at}", 1, 2, lib.ogq_distill_loss, A, cols, rows, cols, dtype, A, 0, A, 10, 1.0, None, A, A, BIG, None)
                call(f"distill gradient {at}", 1, 2, lib.ogq_distill_gradient, A, cols, rows, cols, dtype, A, 0, A, 10, 1.0, None, A, A, cols, A, BIG, None)
        for tokens in (1, 2, 3, 4, 5, 6, 7, 8, 9, 16, 33, 64, 65, 100, 300, 1000, 5000, 20000):
            for outs in (1, 17, 300, 2500, 4096, 20000):
                for cols in (0, 1, 100, 512, 1000, 4096, 25088):
                    for transposed in (0, 1):
                        stride = outs if transposed else cols
                        for gap in (0, 3, 1 << 23):
                            need = lib.ogq_linear_workspace(tokens, outs, cols, dtype, transposed)
                            call(f"linear {tokens} {outs} {cols} {dtype} {transposed} {gap}", 2 if need else 1, 2 if need else 1, lib.ogq_linear, A, cols + gap, A, stride + gap, transposed,
                                 tokens, outs, cols, dtype, A, 1, None, 0, A, outs, A, outs, A, need, None)
        call("no tokens", 1, 1, lib.ogq_embedding_gradient, A, 1, 0, A, 8, 1000, 8, dtype, 1.0, 0, A, 8, None, 0, None)
        call("no rows", 1, 1, lib.ogq_layer_norm_backward, None, 8, None, 8, 0, 8, dtype, None, None, None, None, 8, A, A, 0, None, 0, None)
        call("many tokens", 5, 6, lib.ogq_embedding_gradient, A, 1, 5000000, A, 8, 1000, 8, dtype, 1.0, 0, A, 8, A, BIG, None)
    print(json.dumps({"calls": calls, "wrong": wrong[:20], "unknown": stub.recorded_unknown(),
                      "launches": {stub.recorded_name(i).decode(): stub.recorded_launches_of(i) for i in range(stub.recorded_kernels())}}))


main()
