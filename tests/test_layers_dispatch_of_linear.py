"""The sizes at which linear layers are compared on the GPU reach every kernel that they have on the matrix cores: a rule that sends a size elsewhere would leave a kernel untested."""
import re

import pytest

from tests.layers_layouts import LINEAR
from tests.test_layers_dispatch import _calls


@pytest.fixture(scope="module")
def made(tmp_path_factory):
    return _calls(tmp_path_factory.mktemp("layouts"), "record_launches.cpp", "linear_layouts.py")


def test_compared_sizes_reach_every_kernel_on_the_matrix_cores(made):
    assert len(made["calls"]) == 6 * len(LINEAR) and all(c["status"] == 0 for c in made["calls"])
    reached = {name for c in made["calls"] for name in c["kernels"]}
    kernels = [name for name in made["kernels"] if re.search(r"linear_kernel|join_parts", name)]
    assert len(kernels) == 2 * 2 + 2 * 2 * (3 + 2) + 2 * 2 * 2 + 3  # fp32 tiles; 16 bits' with one team and two; 256 x 256 two ways; joined parts
    assert [name for name in kernels if name not in reached] == []


def test_tiles_of_256_x_256_are_compared(made):
    """Both ways, in both orientations, with more tiles than workgroups that stay."""
    for kernel in ("large_linear_kernel", "direct_linear_kernel"):
        for transposed in (0, 1):
            calls = [c for c in made["calls"] if c["transposed"] == transposed and c["dtype"] != 0 and any(kernel in name for name in c["kernels"])]
            tiles = [-(-c["tokens"] // 256) * -(-c["outs"] // 256) for c in calls]
            assert min(tiles) <= 256 < max(tiles), (kernel, transposed, tiles)
