"""Sums of libogq_groups (weight gradients, products with 4-bit weights) where layouts, values and types are at their limits, on the GPU against the
definitions in 64 bits.  Bounds as in test_groups_gpu.py: n terms summed in 32 bits are off by at most n * 2^-23 times the sum of their magnitudes."""
import pytest
import torch

import paper_2002_11082_amd as ogq
from tests.test_groups_gpu import DEV, TYPES, check_gradient, say, values

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------------------------------------------------
# the order of a sum
# ----------------------------------------------------------------------------------------------------------------------
def layouts(x):
    """The same values with rows next to each other, apart by little, and far apart."""
    rows, cols = x.shape
    yield "contiguous", x
    for stride in (cols + 1, cols + 8, 64 + cols, 1 << 24):
        if rows * stride < 1 << 31:
            wide = torch.empty((rows - 1) * stride + cols, dtype=x.dtype, device=DEV).as_strided((rows, cols), (stride, 1))
            wide.copy_(x)
            yield f"stride {stride}", wide


@pytest.mark.parametrize("rows,outs,cols", [(200, 10, 1000), (97, 10, 33), (129, 130, 260), (190, 7, 222), (255, 128, 128), (1300, 13, 150), (2300, 12, 1030), (700, 3, 4000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_the_order_of_a_gradients_sum_does_not_depend_on_strides(dtype, rows, outs, cols):
    p = ogq.make_group_params(32, 8)
    codes, exponents = ogq.ogq_group_quantize(values(rows, cols, TYPES[dtype], 1), p)
    dy = values(rows, outs, TYPES[dtype], 2, scale=0.05).contiguous()
    first = check_gradient(dy, codes, exponents, cols, p, "order")
    for name, view in layouts(dy):
        say("order", dtype, rows, outs, cols, name)
        assert torch.equal(ogq.ogq_weight_gradient(view, codes, exponents, cols, p), first), name
    one = dy[rows // 3:rows // 3 + 1].expand(rows, outs)
    assert torch.equal(ogq.ogq_weight_gradient(one, codes, exponents, cols, p), ogq.ogq_weight_gradient(one.contiguous(), codes, exponents, cols, p))


# ----------------------------------------------------------------------------------------------------------------------
# fp16 gradients
# ----------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,outs,cols", [(1, 16, 32), (40, 48, 96), (33, 200, 333), (200, 10, 1000), (129, 257, 129), (4100, 33, 65), (1300, 140, 150), (641, 4100, 2570)])
@pytest.mark.parametrize("held_as", ["bf16", "fp32"])
def test_fp16_gradients_with_a_checkpoint_of_another_type(held_as, rows, outs, cols):
    """Inputs beyond what fp16 holds, at both ends, beside ordinary ones."""
    p = ogq.make_group_params(32, 8)
    x = values(rows, cols, torch.float32, 1)
    powers = torch.tensor([2.0 ** 20, 1.0, 2.0 ** -30, 2.0 ** 8, 2.0 ** 60, 2.0 ** -100])
    for n, column in enumerate(range(0, cols, 32)):
        x[:, column:column + 32] *= float(powers[n % 6])
    x[rows // 2, :32] = 3.0 * 2.0 ** 12  # (one group of a column alone)
    codes, exponents = ogq.ogq_group_quantize(x.to(TYPES[held_as]), p)
    dy = values(rows, outs, torch.float16, 2, scale=0.05)
    check_gradient(dy, codes, exponents, cols, p, "other type")
    x = values(rows, cols, torch.float32, 1) * 0.01
    x[-1, -1] = 1e6  # one value in the whole checkpoint
    codes, exponents = ogq.ogq_group_quantize(x.to(TYPES[held_as]), p)
    check_gradient(dy, codes, exponents, cols, p, "one group")
