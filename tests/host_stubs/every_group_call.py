"""Test infrastructure: makes the calls below on the built libogq_groups.so, with record_launches.cpp preloaded in place of the HIP runtime, and
prints what they launched.  Run as a child process by test_groups_dispatch.py; argument: the stand-in's path."""
import ctypes
import json
import sys

from paper_2002_11082_amd import groups as g

A = 0x10000  # aligned; never looked at
SIZES = (1, 2, 31, 33, 128, 200, 513, 1000, 4097, 16384, 100000)
BIG = ctypes.c_size_t(1 << 50)


def main():
    stub, lib = ctypes.CDLL(sys.argv[1]), g.groups_lib()
    stub.recorded_name.restype = ctypes.c_char_p
    for name in ("recorded_launches", "recorded_launches_of", "recorded_unknown"):
        getattr(stub, name).restype = ctypes.c_uint64
    stub.recorded_kernels.restype = ctypes.c_size_t
    calls, wrong = 0, []

    def call(what, most, f, *arguments):
        nonlocal calls
        before = stub.recorded_launches()
        status = f(*arguments)
        made = stub.recorded_launches() - before
        calls += 1
        if status != 0 or not 1 <= made <= most or stub.recorded_last_threads() > 1024 or stub.recorded_last_blocks() == 0:
            wrong.append([what, status, made])

    for group in (32, 64, 128):
        p8, p4 = g.make_group_params(group, 8), g.make_group_params(group, 4)
        for dtype in (0, 1, 2):
            for rows in SIZES:
                for cols in SIZES:
                    for gap in (0, 5):
                        s = cols + gap
                        for p in (p8, p4):
                            call(f"quantize {rows} {cols} {dtype}", 1, lib.ogq_group_quantize, A, s, rows, cols, dtype, p, A, A, None)
                            call(f"dequantize {rows} {cols} {dtype}", 1, lib.ogq_group_dequantize, A, A, rows, cols, p, A, s, dtype, None)
                        for up in (None, A):
                            call(f"forward {rows} {cols} {dtype}", 1, lib.ogq_activation_forward, A, s, up, s, rows, cols, dtype, 3, p8, A, s, A, A, up, up, None)
                            call(f"backward {rows} {cols} {dtype}", 1, lib.ogq_activation_backward, A, s, A, A, up, up, rows, cols, dtype, 3, p8, A, s, up, s, None)
                    for outs in (1, 17, 300, 4096, 20000):
                        need = lib.ogq_weight_gradient_workspace(rows, outs, cols, dtype, p8)
                        call(f"gradient {rows} {outs} {cols} {dtype}", 2 if need else 1, lib.ogq_weight_gradient, A, outs, dtype, A, A, rows, outs, cols, p8, 0, A, cols,
                             A, need, None)
                for tokens in (1, 2, 3, 4, 5, 16, 17, 33, 64, 100, 1000):
                    for cols in (0,) + SIZES:
                        need = lib.ogq_group_matvec_workspace(tokens, rows, cols, dtype, p4)
                        call(f"matvec {tokens} {rows} {cols} {dtype}", 2 if need else 1, lib.ogq_group_matvec, A, A, rows, cols, p4, A, cols, tokens, dtype, A, rows, A, need,
                             None)
    print(json.dumps({"calls": calls, "wrong": wrong[:20], "unknown": stub.recorded_unknown(),
                      "launches": {stub.recorded_name(i).decode(): stub.recorded_launches_of(i) for i in range(stub.recorded_kernels())}}))


main()
