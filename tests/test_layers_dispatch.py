"""libogq_layers without a GPU: every accepted call is as many launches as it should be, every kernel is reached, no accepted size passes a launch's limits, no kernel but those named below uses scratch
memory, and the argument checks run clean under AddressSanitizer and UndefinedBehaviorSanitizer."""
import json
import os
import re
import struct
import subprocess
import sys

import pytest

from tests.test_resources import _notes
from tests.test_sanitizers import SAN, _child_env, _run_pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUBS = os.path.join(ROOT, "tests", "host_stubs")


def _calls(tmp_path, stub_source, script):
    from paper_2002_11082_amd import build, layers
    if not os.path.exists(layers.LAYERS_LIB_PATH):
        build.build()
    stub = str(tmp_path / "stub.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", os.path.join(STUBS, stub_source), "-o", stub], check=True)
    env = dict(os.environ)
    env["LD_PRELOAD"] = ":".join(x for x in (stub, env.get("LD_PRELOAD")) if x)
    env["PYTHONPATH"] = ROOT + os.pathsep + env.get("PYTHONPATH", "")
    res = subprocess.run([sys.executable, os.path.join(STUBS, script), stub], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    return json.loads(res.stdout)


@pytest.fixture(scope="module")
def recorded(tmp_path_factory):
    return _calls(tmp_path_factory.mktemp("record"), "record_launches.cpp", "every_layer_call.py")


def test_every_accepted_call_is_launched(recorded):
    assert recorded["calls"] > 9000
    assert recorded["wrong"] == [] and recorded["unknown"] == 0


def test_every_kernel_of_the_library_is_reached(recorded):
    assert len(recorded["launches"]) > 100
    assert [name for name, launches in recorded["launches"].items() if launches == 0] == []


def test_no_accepted_call_is_refused_by_the_runtime(tmp_path):
    made = _calls(tmp_path, "limited_launches.cpp", "large_layer_calls.py")
    assert made["calls"] > 200 and made["refused"] == 0 and made["wrong"] == [], made


def test_scratch_memory():
    """Registers that spill cost trips to memory.  fp32 rows of more than 32768 logits leave too few registers for their gradient."""
    from paper_2002_11082_amd import build, layers
    if not os.path.exists(layers.LAYERS_LIB_PATH):
        build.build()
    data, magic, found = open(layers.LAYERS_LIB_PATH, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__", {}
    at = data.find(magic)
    while at >= 0:
        number, = struct.unpack_from("<Q", data, at + len(magic))
        entry = at + len(magic) + 8
        for _ in range(number):
            offset, size, name = struct.unpack_from("<QQQ", data, entry)
            if b"gfx950" in data[entry + 24:entry + 24 + name]:
                for note in _notes(data[at + offset:at + offset + size]):
                    found.update((kernel[".name"], kernel) for kernel in note["amdhsa.kernels"])
            entry += 24 + name
        at = data.find(magic, at + 1)
    assert len(found) > 100
    spilled = [name for name, k in found.items() if k[".private_segment_fixed_size"]]
    assert [name for name in spilled if not re.search(r"distill_kernelIfLi1024ELi16E", name)] == []


def test_argument_checks_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    hip_include = "/opt/rocm/include"
    if not os.path.isdir(os.path.join(hip_include, "hip")):
        pytest.skip("HIP headers not found")
    lib = str(tmp_path / "libogq_layers_host_san.so")
    csrc = os.path.join(ROOT, "paper_2002_11082_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I" + hip_include, "-I" + os.path.join(ROOT, "include"), "-I" + csrc, "-shared",
                    "-fPIC", "-x", "c++", os.path.join(csrc, "layers_api.hip"), os.path.join(STUBS, "layers_launch_stubs.cpp"), "-o", lib], check=True)
    env = _child_env({"OGQ_LAYERS_LIBRARY": lib})
    probe = (
        "import paper_2002_11082_amd as ogq\n"
        "A, L = 0x10000, ogq.layers_lib()\n"
        "assert L.ogq_layer_norm_forward(A, 64, 4, 64, 0, A, A, 1e-5, A, 64, A, A, None) == -8 and L.ogq_layers_last_hip_error() != 0\n"
        "assert L.ogq_layer_norm_backward(A, 64, A, 64, 2000, 64, 0, A, A, A, A, 64, A, A, 0, A, 4096, None) == -8\n"
        "assert L.ogq_linear(A, 64, A, 64, 0, 4, 8, 64, 1, A, 1, None, 0, A, 8, None, 0, None, 0, None) == -8\n"
        "assert L.ogq_linear_backward(A, 8, 4, 8, 1, 4, None, 0, None, 0, A, 0, None, 0, None) == -8\n"
        "assert L.ogq_embedding_forward(A, 1, 4, A, 8, 10, 8, 1, 2.0, A, 8, None) == -8\n"
        "assert L.ogq_embedding_gradient(A, 1, 4, A, 8, 10, 8, 1, 2.0, 1, A, 8, A, 64, None) == -8\n"
        "assert L.ogq_distill_loss(A, 64, 4, 64, 1, A, 1, A, 3, 2.0, None, A, None, 0, None) == -8\n"
        "assert L.ogq_distill_gradient(A, 64, 4, 64, 1, A, 1, A, 3, 2.0, None, None, A, 64, None, 0, None) == -8\n"
        "print('refused launches reported')\n")
    res = subprocess.run([sys.executable, "-c", probe], cwd=ROOT, env=env, capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "refused launches reported" in res.stdout, res.stdout + res.stderr
