"""Test infrastructure: calls of the built libogq_groups.so whose grids are next to a launch's limits and beyond what one dimension takes, with limited_launches.cpp preloaded in place of the
HIP runtime; prints what became of them.  Run as a child process by test_groups_launch_limits.py; argument: the stand-in's path."""
import ctypes
import json
import sys

from paper_2002_11082_amd import groups as g

A = 0x10000  # aligned; never looked at


def main():
    stub, lib = ctypes.CDLL(sys.argv[1]), g.groups_lib()
    for name in ("recorded_launches", "recorded_refused", "recorded_last_threads_in_all"):
        getattr(stub, name).restype = ctypes.c_uint64
    calls, wrong = 0, []

    def call(what, threads, f, *arguments):
        """threads: as many as the call's work needs at least."""
        nonlocal calls
        before = stub.recorded_launches()
        status = f(*arguments)
        calls += 1
        if status != 0 or stub.recorded_launches() == before or stub.recorded_last_threads_in_all() < threads:
            wrong.append([what, status])

    for group in (32, 64, 128):
        p8, p4 = g.make_group_params(group, 8), g.make_group_params(group, 4)
        for dtype in (0, 1, 2):
            # values in whole groups, eight to a thread: 2^32 threads and their neighbours, and the largest tensors there are
            for rows, cols in ((1, (1 << 31) - 1), (1 << 18, 1 << 17), ((1 << 18) - 1, 1 << 17), ((1 << 18) + 1, 1 << 17), (1 << 28, 1), ((1 << 28) + 1, 1), ((1 << 31) - 1, 1),
                               ((1 << 31) - 1, 300), (1 << 20, (1 << 20) - 200)):
                threads, what = rows * (-(-cols // group) * group) // 8, f"{rows} {cols} {dtype} {group}"
                for p in (p8, p4):
                    call("quantize " + what, threads, lib.ogq_group_quantize, A, cols, rows, cols, dtype, p, A, A, None)
                    call("dequantize " + what, threads, lib.ogq_group_dequantize, A, A, rows, cols, p, A, cols, dtype, None)
                for up in (None, A):
                    call("forward " + what, threads, lib.ogq_activation_forward, A, cols, up, cols, rows, cols, dtype, 3, p8, A, cols, A, A, up, up, None)
                    call("backward " + what, threads, lib.ogq_activation_backward, A, cols, A, A, up, up, rows, cols, dtype, 3, p8, A, cols, up, cols, None)
            # four outputs to a wavefront; tiles of 128 x 128 sums, or of 128 outputs and 64 tokens, to 256 threads, where 2^32 threads are an error of the arguments
            for rows, outs, cols in ((1, (1 << 31) - 128, 1), (1, 1, (1 << 31) - 128), (700, (1 << 30) - 1, 100), (1, 1 << 19, (1 << 19) - 200)):
                need = lib.ogq_weight_gradient_workspace(rows, outs, cols, dtype, p8)
                call(f"gradient {rows} {outs} {cols} {dtype}", outs * cols // 256, lib.ogq_weight_gradient, A, outs, dtype, A, A, rows, outs, cols, p8, 0, A, cols, A, need, None)
            for rows, outs, cols in ((1, (1 << 31) - 127, 1), (1, 1, (1 << 31) - 127), (700, (1 << 30) - 1, 800), (1, 1 << 19, (1 << 19) - 100)):
                if lib.ogq_weight_gradient_workspace(rows, outs, cols, dtype, p8) != 0 or \
                   lib.ogq_weight_gradient(A, outs, dtype, A, A, rows, outs, cols, p8, 0, A, cols, A, 1 << 50, None) != -9:
                    wrong.append([f"gradient {rows} {outs} {cols} {dtype}", "not refused"])
            for tokens, outs, cols in ((2, (1 << 31) - 127, 1), (1 << 20, (1 << 20) - 200, 40), (1 << 18, (1 << 19) - 100, 40)):
                if lib.ogq_group_matvec_workspace(tokens, outs, cols, dtype, p4) != 0 or \
                   lib.ogq_group_matvec(A, A, outs, cols, p4, A, cols, tokens, dtype, A, outs, A, 1 << 50, None) != -9:
                    wrong.append([f"matvec {tokens} {outs} {cols} {dtype}", "not refused"])
            for tokens, outs, cols in ((1, (1 << 31) - 1, 1), (1, 1 << 28, 32), (1, (1 << 26) + 1, 8192), (16, (1 << 31) - 128, 1), (1 << 18, (1 << 19) - 200, 40), ((1 << 17) + 1, 1 << 19, 40)):
                need = lib.ogq_group_matvec_workspace(tokens, outs, cols, dtype, p4)
                threads = outs * 16 if tokens == 1 else outs * tokens // 32
                call(f"matvec {tokens} {outs} {cols} {dtype}", threads if cols > 1 else 1, lib.ogq_group_matvec, A, A, outs, cols, p4, A, cols, tokens, dtype, A, outs, A, need, None)
    print(json.dumps({"calls": calls, "refused": stub.recorded_refused(), "wrong": wrong}))


main()
