"""Sizes that reach every kernel of the point-wise product, and how far fp32 results may be off in all: below what any lost term of a factor would cost.

What is off, each part by half a step (2^-24) or a share of it and independent of the others, so that the 2-norms add up in squares at most and here, for the
bound, as they are:
  terms left out    2^-21 of a product at most, of either sign: 2^-21 of the 2-norm
  sums              an addition is off by 2^-23 of the partial sum at most (the matrix cores need not round to nearest); partial sums are no larger than the
                    result in the mean, `adds` of them in a row: sqrt(adds) 2^-23
  the slope         silu'(pre): an exponential, a sum, a reciprocal and two products, each within 2^-23, pre's own sum and terms as above, weighed by
                    |silu''| <= 1/2: 2^-21
"""
import math

import torch

F32, BF16 = 0, 1
NAMES = ("f32", "bf16")
# dtype, N, K, M, H, W, act
CASES = [(F32, 1, 16, 20, 30, 30, "silu"), (F32, 1, 16, 65, 180, 320, "silu"), (F32, 1, 64, 70, 30, 30, "silu"), (F32, 1, 100, 60, 30, 30, "silu"),
         (F32, 1, 150, 200, 64, 64, "silu"), (F32, 1, 200, 200, 64, 64, "silu"), (F32, 1, 260, 130, 64, 64, "silu"), (F32, 3, 16, 200, 150, 301, "none"),
         (F32, 3, 40, 20, 150, 301, "silu"), (F32, 3, 40, 200, 150, 301, "none"), (F32, 3, 170, 20, 150, 301, "silu"), (F32, 3, 170, 40, 150, 301, "silu"),
         (F32, 20, 24, 200, 31, 33, "none"), (F32, 60, 190, 20, 31, 33, "silu"), (F32, 70, 32, 20, 7, 9, "silu"), (BF16, 1, 16, 20, 30, 30, "silu"),
         (BF16, 1, 16, 65, 400, 400, "none"), (BF16, 1, 16, 129, 30, 30, "none"), (BF16, 1, 24, 60, 30, 30, "none"), (BF16, 1, 40, 65, 180, 320, "silu"),
         (BF16, 1, 40, 200, 400, 400, "none"), (BF16, 1, 60, 65, 30, 30, "silu"), (BF16, 1, 90, 33, 30, 30, "silu"), (BF16, 1, 90, 210, 400, 400, "none"),
         (BF16, 1, 128, 128, 30, 30, "silu"), (BF16, 1, 150, 129, 180, 320, "silu"), (BF16, 1, 200, 260, 64, 64, "silu"), (BF16, 1, 210, 20, 180, 320, "silu"),
         (BF16, 1, 210, 65, 100, 130, "none"), (BF16, 1, 210, 260, 180, 320, "silu"), (BF16, 1, 260, 210, 180, 320, "silu"), (BF16, 2, 16, 20, 301, 255, "none"),
         (BF16, 2, 210, 33, 301, 255, "silu"), (BF16, 3, 16, 32, 150, 301, "silu"), (BF16, 3, 16, 129, 150, 301, "none"), (BF16, 3, 16, 200, 150, 301, "none"),
         (BF16, 3, 24, 40, 150, 301, "none"), (BF16, 3, 40, 32, 150, 301, "silu"), (BF16, 3, 100, 20, 150, 301, "silu"), (BF16, 3, 210, 20, 150, 301, "silu"),
         (BF16, 20, 16, 129, 31, 33, "none"), (BF16, 20, 16, 200, 31, 33, "silu"), (BF16, 20, 16, 210, 31, 33, "none"), (BF16, 20, 40, 210, 31, 33, "none"),
         (BF16, 20, 170, 20, 31, 33, "none"), (BF16, 20, 170, 20, 31, 33, "silu"), (BF16, 60, 16, 70, 31, 33, "silu"), (BF16, 70, 24, 20, 7, 9, "none"),
         (BF16, 70, 100, 65, 7, 9, "silu")]
# the least that a result's 2-norm is off by where a factor loses its third term (test_product_accuracy.py)
LOST = 3.8e-6
# results rounded to bf16 that are not the nearest to the definition's: two terms of a weight leave 2^-17 of a product at most, half of a typical element's 2^-8 step
# times 2^-8; small elements have smaller steps, gp's two terms double it.  With one term left a third of all are others.
OTHERS = 2.0 ** -6


def bars(case):
    """{result: how far its 2-norm may be off} of the results that are fp32."""
    dt, N, K, M, H, W, act = case
    pixels, products = N * H * W, 6 if dt == F32 else 3 if act != "none" else 1

    def bar(adds, slope):
        return 2.0 ** -21 + 2.0 ** -23 * math.sqrt(adds) + (2.0 ** -21 if slope and act != "none" else 0)

    # grad_w's tiles, and the shares of the pixels that fill 512 blocks; the shares' sums come in 32 or fewer steps
    side_m = 128 if M > 64 else 64
    side_k = 128 if K > 64 and not (dt == F32 and M > 64) else 64
    shares = max(1, min(512 // (-(-M // side_m) * -(-K // side_k)), pixels // 64))
    res = {n: bar(products * pixels / 16 / shares + 32, True) for n in ("grad_w", "grad_b")}
    if dt == F32:
        res.update(out=bar(6 * K / 16 + 8, False), grad_x=bar(6 * M / 16 + 8, True))
    return res


def off(a, b):
    return ((a.double() - b.double()).norm() / b.double().norm()).item()


def two_of_three(t):
    """fp32 values without the third of three bf16 terms (truncated ones)."""
    first = (t.view(torch.int32) & -65536).view(torch.float32)
    second = ((t - first).view(torch.int32) & -65536).view(torch.float32)
    return first.double() + second.double()


def one_of_two(t):
    return t.bfloat16().double()
