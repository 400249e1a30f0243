"""What is no number, in ts_quantize_fp8 and ts_matmul_fp8: it hides no other value, and reaches its own row or column alone."""
import numpy as np
import pytest
import torch

from oracle import operators as op
from paper_1905_04035_amd import binding as ts
from tests.test_fp8_gpu import BF16, E4M3, E5M2, FP32, quantized, same_codes

pytestmark = pytest.mark.gpu

# NaNs that signal, the smallest and a negative one; that are quiet; infinities
BITS = [0x7F800001, 0xFFA00000, 0x7FC00000, 0xFFFFFFFF, 0x7F800000, 0xFF800000]


def beside_the_largest(bits, rows, cols):
    """[rows, cols] fp32: the largest value of each block of 128 of every row has `bits` beside it, at each distance and place in turn."""
    rng = np.random.default_rng(bits & 0xFFFF)
    x = rng.standard_normal((rows, cols)).astype(np.float32)
    for r in range(rows):
        for b in range(0, cols, 128):
            width = min(128, cols - b)
            at = (5 * r + b // 128) % width
            other = [at ^ 1, at ^ 2, at ^ 4, at ^ 8, at ^ 16, at ^ 64][r // 2 % 6]
            x[r, b + at] = (-1.0) ** r * 1000.0 * (1 + r % 7)
            if other < width:
                x.view(np.uint32)[r, b + other] = bits
    return x


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("fmt", [E4M3, E5M2])
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("rows,cols", [(256, 384), (150, 203)])
def test_what_is_no_number_hides_no_largest_value(bits, fmt, dtype, rows, cols):
    x = torch.from_numpy(beside_the_largest(bits, rows, cols).view(np.int32))
    # bf16: the upper half of the bits, and the NaN whose bits lie below it keeps one
    x = x.view(FP32) if dtype == FP32 else ((x >> 16) | ((x & 0x7FFFFFFF) == 0x7F800001).int()).to(torch.int16).view(BF16)
    for turned in (False, True):
        y = x.t().contiguous() if turned else x
        h = y.float().numpy()
        q, s, qt, st = quantized(y, fmt)
        for codes, scales, of in ((q, s, h), (qt, st, h.T)):
            want, want_scales = op.quantize(of, fmt)
            assert np.array_equal(scales.cpu().numpy(), want_scales)
            same_codes(codes, want, fmt)
