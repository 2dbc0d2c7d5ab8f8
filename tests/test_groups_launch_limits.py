"""libogq_groups on tensors whose grids pass what HIP takes along one dimension, 2^32 threads."""
import json
import os
import subprocess
import sys

import pytest
import torch

import paper_2002_11082_amd as ogq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUBS = os.path.join(ROOT, "tests", "host_stubs")
DEV = "cuda:0"


def test_no_accepted_call_is_refused_by_the_runtime(tmp_path):
    from paper_2002_11082_amd import build, groups
    if not os.path.exists(groups.GROUPS_LIB_PATH):
        build.build()
    stub = str(tmp_path / "limited_launches.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", os.path.join(STUBS, "limited_launches.cpp"), "-o", stub], check=True)
    env = dict(os.environ)
    env["LD_PRELOAD"] = ":".join(x for x in (stub, env.get("LD_PRELOAD")) if x)
    env["PYTHONPATH"] = ROOT + os.pathsep + env.get("PYTHONPATH", "")
    res = subprocess.run([sys.executable, os.path.join(STUBS, "large_group_calls.py"), stub], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    made = json.loads(res.stdout)
    assert made["calls"] > 700 and made["refused"] == 0 and made["wrong"] == [], made


def numbers(n, dtype, period):
    """Whole numbers that a group of 8 bits holds exactly."""
    return (torch.arange(n, dtype=torch.int32, device=DEV) % period - period // 2).to(dtype)


@pytest.mark.gpu
def test_more_groups_than_threads_along_a_dimension():
    rows = (1 << 28) + 5
    print("[groups] many rows", rows, flush=True)
    p = ogq.make_group_params(128, 8)
    x, up = numbers(rows, torch.bfloat16, 201).view(rows, 1), numbers(rows, torch.bfloat16, 127).view(rows, 1)
    codes, exponents = ogq.ogq_group_quantize(x, p)
    assert torch.equal(ogq.ogq_group_dequantize(codes, exponents, 1, p, torch.bfloat16), x)
    y, codes, exponents, up_codes, up_exponents = ogq.ogq_activation_forward(x, ogq.RELU, p, up, codes=codes, exponents=exponents)
    assert torch.equal(y, x.relu() * up)
    dx, dup = ogq.ogq_activation_backward(up, ogq.RELU, codes, exponents, p, up_codes, up_exponents)
    assert torch.equal(dx, torch.where(x > 0, up * up, torch.zeros_like(x))) and torch.equal(dup, up * x.relu())


@pytest.mark.gpu
def test_more_outputs_than_threads_along_a_dimension():
    outs, period = (1 << 28) + 9, 1 << 12
    print("[groups] many outputs", outs, flush=True)
    p = ogq.make_group_params(32, 4)
    few_codes, few_exponents = ogq.ogq_group_quantize(torch.randn(period, 32, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV), p)
    x = torch.randn(1, 32, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).bfloat16()
    few = ogq.ogq_group_matvec(few_codes, few_exponents, 32, p, x)
    # the same rows again and again (by repetition: torch's indexing has given wrong rows of as many bytes)
    many = -(-outs // period)
    y = ogq.ogq_group_matvec(few_codes.repeat(many, 1)[:outs], few_exponents.repeat(many, 1)[:outs], 32, p, x)
    assert torch.equal(y[0], few[0].repeat(many)[:outs])


@pytest.mark.gpu
def test_as_many_sums_as_a_launch_takes():
    outs = (1 << 31) - 128
    print("[groups] many sums", outs, flush=True)
    p = ogq.make_group_params(32, 8)
    codes, exponents = ogq.ogq_group_quantize(torch.full((1, 1), 3.0, device=DEV), p)
    dy = numbers(outs, torch.bfloat16, 251).view(1, outs)
    dw = ogq.ogq_weight_gradient(dy, codes, exponents, 1, p)
    for at in range(0, outs, 1 << 28):
        part = slice(at, min(outs, at + (1 << 28)))
        assert torch.equal(dw[part, 0], dy[0, part].float() * 3.0)
