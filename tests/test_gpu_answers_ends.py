"""Products whose last columns end anywhere in what a kernel reads at a time, against 64 bits.  What follows the matrix in memory is
no part of it (bytes of 255: scales that are NaN); tests/test_message_reads.py goes through the reads themselves.

Tolerance: as in test_gpu_answers.py, every code counted as 31, 8 U of the sum of such terms, and the rounding to the output's type; for
the gradient in 16-bit dtypes 2^-17 of them besides."""
import numpy as np
import pytest
import torch

from paper_1907_07346_amd import binding as b
from tests import answers_plain as plain

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def close(got, want, size, dtype, pieces, what):
    tol = (8 * U + (2.0 ** -17 if pieces and dtype != F32 else 0.0)) * 31.0 * size + plain.rounding(want, dtype)
    bad = ~((got.cpu().double() - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}"


def check_products(tokens, rows, cols, block, dtype, gradient=True):
    rng = np.random.default_rng(tokens * 7919 + rows * 31 + cols + block)
    msg, codes, scales = plain.random_message(rows, cols, block, rng)
    m = plain.dense(codes, scales, block)
    unit = torch.from_numpy(np.repeat(scales.astype(np.float64), block, axis=1)[:, :cols] / 15.0)
    big = torch.full((msg.numel() + 256,), 255, dtype=torch.uint8)
    big[:msg.numel()] = msg
    here = big.cuda()[:msg.numel()]
    x = torch.from_numpy(rng.standard_normal((tokens, cols))).to(dtype)
    close(b.ds_product(here, x.cuda(), rows, block), x.double() @ m.t().contiguous(), x.double().abs() @ unit.t().contiguous(), dtype, False, "y")
    if gradient:
        dy = torch.from_numpy(rng.standard_normal((tokens, rows))).to(dtype)
        close(b.ds_product_gradient(here, dy.cuda(), cols, block), dy.double() @ m, dy.double().abs() @ unit, dtype, True, "dx")


# One token, widths around 16384 columns, which a workgroup takes at a time: one to four words are left, or a few lanes' worth.
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("block", [64, 256, 2048])
@pytest.mark.parametrize("cols", [16384, 16385, 16392, 16393, 16400, 16401, 16408, 16409, 16416, 16417, 32769, 32792])
def test_one_token_through_wide_rows(cols, block, dtype):
    check_products(1, 37, cols, block, dtype, gradient=False)


# Few tokens, 256 columns at a time: a row ends with them, or a word, two or more behind them; rows below, at and above the 128 of a workgroup;
# 66 tokens: the last two are a launch of their own.
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("block", [64, 128, 256, 512])
@pytest.mark.parametrize("tokens,rows,cols", [(2, 100, 257), (8, 128, 264), (16, 129, 265), (8, 131, 513), (3, 300, 4100), (2, 40, 256), (5, 7, 520),
                                              (8, 260, 521), (66, 130, 260)])
def test_few_tokens_and_the_columns_behind_a_stage(tokens, rows, cols, block, dtype):
    check_products(tokens, rows, cols, block, dtype)
