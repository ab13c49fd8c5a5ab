"""Root-mean-square norm, its gradient and rows in 8 bits where a workgroup goes over the rows more than once, the last time with fewer rows than it takes: against the definitions in 64 bits, with the
weight's gradient, a residual and outputs in the place of inputs, as tests/test_gpu_rms.py has them for one round and with its bounds."""
import pytest

import paper_2507_05508_amd as P
import test_gpu_rms as one

pytestmark = pytest.mark.gpu
# rows, width, pad, shift: every number of threads a row has, 8 and 16 entries a thread; more rows than two rounds of all workgroups take, forward (two of a CU where a thread has one load a round) and backward
SIZES = [(9001, 40, 0, 0), (8997, 511, 1, 0), (4500, 520, 0, 0), (4501, 1021, 3, 1), (2300, 1100, 0, 0), (1100, 2100, 4, 0), (601, 8191, 0, 0), (601, 9000, 0, 0), (529, 16384, 0, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad,shift", SIZES)
def test_forward(n, d, pad, shift, dtype):
    one.test_rms_norm(n, d, pad, shift, dtype)


@pytest.mark.parametrize("dtype,grad_dtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,d,pad,shift", SIZES)
def test_backward(n, d, pad, shift, dtype, grad_dtype):
    assert P.mlmc_rms_norm_workspace(n, d) == 256 * d * 4     # a partial sum of each of 256 workgroups
    one.test_rms_norm_backward(n, d, pad, shift, dtype, grad_dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad,shift", SIZES)
def test_quantize(n, d, pad, shift, dtype):
    one.test_quantize_to_the_bit(n, d, pad, shift, dtype)
