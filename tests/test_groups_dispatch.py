"""libogq_groups without a GPU: every accepted call is a launch (or two, with a workspace), every kernel is reached, and the argument checks run clean under
AddressSanitizer and UndefinedBehaviorSanitizer."""
import json
import os
import subprocess
import sys

import pytest

from tests.test_sanitizers import SAN, _child_env, _run_pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUBS = os.path.join(ROOT, "tests", "host_stubs")


@pytest.fixture(scope="module")
def recorded(tmp_path_factory):
    from paper_2002_11082_amd import build, groups
    if not os.path.exists(groups.GROUPS_LIB_PATH):
        build.build()
    stub = str(tmp_path_factory.mktemp("record") / "record_launches.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", os.path.join(STUBS, "record_launches.cpp"), "-o", stub], check=True)
    env = dict(os.environ)
    env["LD_PRELOAD"] = ":".join(x for x in (stub, env.get("LD_PRELOAD")) if x)
    env["PYTHONPATH"] = ROOT + os.pathsep + env.get("PYTHONPATH", "")
    res = subprocess.run([sys.executable, os.path.join(STUBS, "every_group_call.py"), stub], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    return json.loads(res.stdout)


def test_every_accepted_call_is_launched(recorded):
    assert recorded["calls"] > 5000
    assert recorded["wrong"] == [] and recorded["unknown"] == 0


def test_every_kernel_of_the_library_is_reached(recorded):
    assert len(recorded["launches"]) > 40
    assert [name for name, launches in recorded["launches"].items() if launches == 0] == []


def test_argument_checks_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    hip_include = "/opt/rocm/include"
    if not os.path.isdir(os.path.join(hip_include, "hip")):
        pytest.skip("HIP headers not found")
    lib = str(tmp_path / "libogq_groups_host_san.so")
    csrc = os.path.join(ROOT, "paper_2002_11082_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I" + hip_include, "-I" + os.path.join(ROOT, "include"), "-I" + csrc, "-shared",
                    "-fPIC", "-x", "c++", os.path.join(csrc, "groups_api.hip"), os.path.join(STUBS, "groups_launch_stubs.cpp"), "-o", lib], check=True)
    env = _child_env({"OGQ_GROUPS_LIBRARY": lib})
    files = [os.path.join(ROOT, "tests", "test_groups_abi.py")]
    assert " passed" in _run_pytest(files, env)
    probe = (
        "import paper_2002_11082_amd as ogq\n"
        "A, L = 0x10000, ogq.groups_lib()\n"
        "p8, p4 = ogq.make_group_params(64, 8), ogq.make_group_params(64, 4)\n"
        "assert L.ogq_group_quantize(A, 64, 4, 64, 0, p8, A, A, None) == -8 and L.ogq_groups_last_hip_error() != 0\n"
        "assert L.ogq_group_dequantize(A, A, 4, 64, p4, A, 64, 1, None) == -8\n"
        "assert L.ogq_activation_forward(A, 64, A, 64, 4, 64, 2, 3, p8, A, 64, A, A, A, A, None) == -8\n"
        "assert L.ogq_activation_backward(A, 64, A, A, None, None, 4, 64, 2, 3, p8, A, 64, None, 0, None) == -8\n"
        "assert L.ogq_weight_gradient(A, 8, 0, A, A, 4, 8, 64, p8, 1, A, 64, None, 0, None) == -8\n"
        "assert L.ogq_weight_gradient(A, 8, 0, A, A, 2000, 8, 64, p8, 1, A, 64, A, 4096, None) == -8\n"
        "assert L.ogq_group_matvec(A, A, 8, 64, p4, A, 64, 3, 1, A, 8, None, 0, None) == -8\n"
        "print('refused launches reported')\n")
    res = subprocess.run([sys.executable, "-c", probe], cwd=ROOT, env=env, capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "refused launches reported" in res.stdout, res.stdout + res.stderr
