"""The operators that serve the sub-block where the tolerances of random operands say little: scales beyond fp16's range,
operands of whole numbers whose results are known to the last bit, and every kernel that a size chooses.

Tolerances.  u is a type's unit roundoff, eps / 2 (bf16 2^-8, fp16 2^-11, e4m3 2^-4).  Sums of n products in fp32 are off by
at most (n + 16) 2^-23 of the sum of the products' sizes.  A result's own rounding adds u of its size; below the
type's normal range half of its smallest step.
"""
import pytest
import torch

from paper_1802_06905_b200 import block
from test_gpu_block import BF16, FP16, FP32, TINY, U, close, gen, normal, poisoned, sum_err
from test_gpu_block_serve import Int4

pytestmark = pytest.mark.gpu


# ---- 4-bit weights beyond fp16's range -------------------------------------------------------------

def check_fp16(c, out, what):
    """Against 64 bits: weights rounded to fp16's precision with more than 64 tokens, a row's smallest ones to 2^-31 of its
    largest scale; results beyond fp16's largest number (65504, from 65520 on) are infinite.  Tokens that hold an infinity
    (x beyond that number) give nothing finite; the others are compared."""
    q, z, s = c.weights()
    x, there = c.x.double(), torch.isfinite(c.x).all(1)
    assert not torch.isfinite(out[~there]).any(), what
    x, out = x[there], out[there]
    w = s * (q - z)
    exact = x @ w.T
    size = x.abs() @ (s.abs() * (32 + q + z) if c.M <= 64 else w.abs()).T
    tol = 1.01 * ((sum_err(c.K) + (U[FP16] if c.M > 64 else 0)) * size + U[FP16] * exact.abs()) + TINY[FP16]
    if c.M > 64:
        tol = tol + 2.0 ** -30 * x.abs().sum(1, keepdim=True) * c.scale.double().abs().amax(1)
    out = out.double()
    big = torch.isinf(out)
    assert ((exact.abs() + tol)[big] >= 65520).all() and (torch.sign(out[big]) == torch.sign(exact[big])).all(), what
    assert ((exact.abs() - tol)[~big] < 65520).all(), what
    close(out[~big], exact[~big], tol[~big], what)


# (scale of x, scale of the groups' scales): results of common size from scales that fp16 weights cannot hold
RANGES = [(2.0 ** -10, 1e5), (2e4, 1e-9), (3e4, 1e-7), (1.0, 1e-3), (2.0 ** -14, 1e7), (5e3, 1e-8), (1e4, 1e-9)]


@pytest.mark.parametrize("M,N,K", [(64, 72, 256), (65, 72, 256), (65, 131, 1000), (100, 40, 264), (300, 513, 320), (2100, 1300, 256)])
@pytest.mark.parametrize("scale", [FP32, BF16])
def test_int4_scales_that_fp16_cannot_hold(M, N, K, scale):
    for i, (xs, ss) in enumerate(RANGES):
        for group, zero in ((32, False), (64, True), (128, i % 2 == 0)):
            c = Int4(M, N, K, group, FP16, scale, zero, seed=i)
            c.x = (c.x.double() * xs).to(FP16)
            c.scale = (c.scale.double() * (ss * 5 * K ** 0.5)).to(scale)
            check_fp16(c, c.run(), f"{M}x{N}x{K} group {group}: x {xs}, scales {ss}")
    assert block.status() == (0, 0)


@pytest.mark.parametrize("M", [64, 65, 200])
def test_int4_rows_of_every_size_in_fp16(M):
    """A row of each power of ten from 1e-12 to 1e12, rows of zeros among them, negative scales; and fp16's own scales to their ends."""
    N, K = 25 * 4, 512
    c = Int4(M, N, K, 128, FP16, FP32, zero=True)
    size = 10.0 ** (torch.arange(N, device="cuda", dtype=torch.float64) // 4 - 12)
    c.scale = (c.scale.double() * size[:, None]).to(FP32)
    c.scale[::7] *= -1
    c.scale[5] = 0
    c.scale[9, 1:3] = 0
    # tokens small and large, so that each row has results in range
    c.x = (c.x.double() * 2.0 ** (torch.arange(M, device="cuda", dtype=torch.float64) % 28 - 14)[:, None]).to(FP16)
    check_fp16(c, c.run(), "rows of every size")
    c.scale = torch.tensor([6e-8, 1e-6, 6.1e-5, 1.0, 4000.0, 4400.0, 30000.0, 65504.0], device="cuda", dtype=FP16).repeat(13)[:N, None].repeat(1, 4)
    check_fp16(c, c.run(), "scales in fp16")


@pytest.mark.parametrize("scale", [FP32, FP16])
def test_int4_a_row_s_small_groups_beside_large_ones(scale):
    c = Int4(80, 64, 1024, 128, FP16, scale)
    c.scale = (c.scale.double() * 2.0 ** -(3.0 * (torch.arange(8, device="cuda", dtype=torch.float64)))).to(scale)
    # the large groups meet tokens of zeros: what is left is the small groups' part
    c.x[:40, :512] = 0
    check_fp16(c, c.run(), "small groups")


def test_int4_infinities_and_nan_of_scales_in_fp16():
    """They stay with their row, and the row's other groups do not change what it is divided by."""
    c = Int4(70, 64, 512, 128, FP16, FP32)
    exp = c.run()
    c.scale[9, 2], c.scale[12, 0] = float("nan"), float("inf")
    out = c.run()
    rows = [n for n in range(64) if n not in (9, 12)]
    assert torch.equal(out[:, rows], exp[:, rows])
    assert torch.isnan(out[:, 9]).all() and not torch.isfinite(out[:, 12]).any()


def test_int4_in_fp16_into_strided_results():
    for M, N in ((65, 77), (65, 1024), (700, 333)):
        c = Int4(M, N, 384, 64, FP16, FP32, zero=True)
        c.scale *= 1e4
        c.x = (c.x.double() * 1e-3).to(FP16)
        big = torch.full((M + 2, N + 11), 7.0, device="cuda", dtype=FP16)
        check_fp16(c, c.run(out=big[1:M + 1, 3:N + 3]), "inside")
        big[1:M + 1, 3:N + 3] = 7.0
        assert (big == 7.0).all()
        wide = poisoned((N, M), FP16)
        check_fp16(c, c.run(out=wide.t()), "transposed")


def test_int4_in_fp16_with_more_rows_than_a_launch_has_blocks():
    c = Int4(66, 4 * 65535 + 90, 48, 32, FP16, FP32, zero=True)
    c.scale = (c.scale.double() * 10.0 ** (torch.arange(c.N, device="cuda", dtype=torch.float64) % 9 - 5)[:, None]).to(FP32)
    check_fp16(c, c.run(), "many rows")
