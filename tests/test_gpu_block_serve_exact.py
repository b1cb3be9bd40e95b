"""The operators that serve the sub-block where the tolerances of random operands say little: scales beyond fp16's range,
operands of whole numbers whose results are known to the last bit, and every kernel that a size chooses.

Tolerances.  u is a type's unit roundoff, eps / 2 (bf16 2^-8, fp16 2^-11, e4m3 2^-4).  Sums of n products in fp32 are off by
at most (n + 16) 2^-23 of the sum of the products' sizes.  A result's own rounding adds u of its size; below the
type's normal range half of its smallest step.
"""
import pytest
import torch

import test_gpu_block_serve as serve
from paper_1802_06905_b200 import block
from test_gpu_block import BF16, FP16, FP32, TINY, U, close, gen, normal, poisoned, sum_err
from test_gpu_block_serve import Int4, Moe

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


def test_int4_in_fp16_captured_and_on_two_streams():
    """The rows' powers of two are the workspace's, of each call its own; a workspace of just the size, whatever it holds."""
    cs = []
    for i, (M, N, K) in enumerate(((65, 333, 520), (300, 1024, 512), (80, 77, 2050))):
        c = Int4(M, N, K, 64, FP16, FP32, zero=True, seed=i)
        c.scale = (c.scale.double() * 10.0 ** (torch.arange(N, device="cuda", dtype=torch.float64) % 7 - 4)[:, None]).to(FP32)
        cs.append(c)
    want = [c.run() for c in cs]
    for c, w in zip(cs, want):
        check_fp16(c, w, "alone")
        n = block.int4_product_workspace(c.x, c.q, c.scale, w, zero=c.zero, group=64)
        for byte in (0, 255):
            space = torch.full((n + 4096,), byte, device="cuda", dtype=torch.uint8)
            assert torch.equal(c.run(workspace=space[:n]), w) and (space[n:] == byte).all()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    torch.cuda.synchronize()
    for i in range(30):
        with torch.cuda.stream(streams[i % 2]):
            got.append((i % 3, cs[i % 3].run()))
    torch.cuda.synchronize()
    assert all(torch.equal(out, want[i]) for i, out in got)
    graphs = []
    for c in cs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[0]):
            graphs.append((g, c.run()))
    for c in cs:
        c.scale.mul_(1e-3)
    torch.cuda.synchronize()
    for _ in range(2):
        for (g, out), c in zip(graphs, cs):
            g.replay()
    torch.cuda.synchronize()
    for (g, out), c in zip(graphs, cs):
        assert torch.equal(out, c.run())


# ---- 4-bit products known to the last bit ------------------------------------------------------------

def integers(g, low, high, shape, dtype):
    return torch.randint(low, high + 1, shape, generator=g, device="cuda").to(dtype)


def exact_int4(M, N, K, group, dtype, scale, zero):
    """Tokens of whole numbers up to 3 and scales that are powers of two from 1/8 to 1: in units of 1/8, sums of (q - z) s x
    are whole numbers below 45 8 K (K up to 16416: 2^22.5), and a group's of (16 + q) x below 2^14, so that fp32 holds each
    without rounding in whatever order they are added up; and weights are numbers of 4 bits and a sign."""
    c = Int4(M, N, K, group, dtype, scale, zero)
    g = gen(M + N + K + group)
    c.x = integers(g, -3, 3, (M, K), dtype)
    c.scale = (2.0 ** -integers(g, 0, 3, c.scale.shape, FP32)).to(scale)
    return c


# own tokens: one tile a block and several (more than 296 tiles of 16 or 32 rows), rows that begin at multiples of 16, 8 and 4
# bytes; 3 to 8 tokens shared; every number of token tiles; few and many units for a cluster; expanded
EXACT = [(1, 20011, 256), (2, 20011, 264), (1, 20011, 272), (2, 9500, 1040), (1, 20011, 4096), (8, 12000, 128), (1, 300, 8192), (2, 77, 16416),
         (3, 300, 4096), (7, 4096, 4096), (8, 5000, 5120), (4, 129, 8192), (5, 40, 16416), (3, 1000, 5130), (6, 2000, 2056),
         (9, 700, 4096), (16, 1000, 5120), (17, 129, 8192), (23, 5000, 4200), (31, 64, 1024), (40, 129, 16416), (48, 700, 4100), (64, 31, 16416),
         (64, 1030, 2048), (65, 130, 4096), (300, 513, 1000), (2060, 300, 264)]


@pytest.mark.parametrize("M,N,K", EXACT)
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_int4_products_of_whole_numbers(M, N, K, dtype):
    for group in (32, 64, 128):
        for scale, zero in ((dtype, False), (FP32, True)):
            c = exact_int4(M, N, K, group, dtype, scale, zero)
            out = c.run()
            q, z, s = c.weights()
            exact = c.x.double() @ (s * (q - z)).T
            assert torch.equal(out, exact.to(FP32).to(dtype)), (group, scale, zero)
    assert block.status() == (0, 0)


@pytest.mark.parametrize("M,N,K", [(1, 1000, 8192), (2, 20011, 1024), (5, 1000, 5120), (8, 300, 4096), (23, 1000, 4200), (64, 100, 16416),
                                   (65, 1000, 4096), (400, 300, 4096), (1, 100, 60000), (2, 64, 40000), (8, 64, 60000)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_int4_errors_are_the_result_s_rounding(M, N, K, dtype):
    """Of random operands, relative to the result's norm: a result rounded once is off by r, the sums' errors are far below
    it (K 2^-24 of their terms' root sum of squares at worst, which 16 + q makes five times as large: 2^-8 r in fp16 at
    K = 4096) and add a tenth at most; with more than 64 tokens each weight is rounded as well, by the same share: r sqrt 2."""
    for group, zero in ((32, True), (128, False)):
        c = Int4(M, N, K, group, dtype, None, zero)
        out = c.run().double()
        q, z, s = c.weights()
        exact = c.x.double() @ (s * (q - z)).T
        rounding = (exact.to(dtype).double() - exact).norm()
        assert (out - exact).norm() <= (1.1 if M <= 64 else 1.55) * rounding


# ---- mixtures known to the last bit ----------------------------------------------------------------------

def exact_moe(T, D, F, E, k, dtype):
    """Whole numbers as tokens (up to 2) and as weights of gate and up (up to 1), sixteenths as weights of down, relu, and
    powers of two from 1/4 to 1 as the choices' weights: h is a whole number, of more bits than the type has, but for
    |h| <= 65504 no more than two numbers of it hold; everything else is a whole number in units of 1/64."""
    m = Moe(T, D, F, E, k, dtype, "relu")
    g = gen(T + D + F + E)
    m.x = integers(g, -2, 2, (T, D), dtype)
    thin = min(1.0, 700.0 / D)  # (the share of weights that are not zeros, which keeps h in range)
    keep = lambda t: t * (torch.rand(t.shape, generator=g, device="cuda") < thin)  # noqa: E731
    m.wg, m.wu = (keep(integers(g, -1, 1, (E, F, D), dtype)) for _ in range(2))
    m.wd = integers(g, -1, 1, (E, D, F), dtype) / 16
    ids = torch.stack([torch.randperm(E, generator=g, device="cuda")[:k] for _ in range(T)]).to(torch.int32)
    weights = 2.0 ** -integers(g, 0, 2, (T, k), FP32) * integers(g, 0, 1, (T, k), FP32).mul_(2).sub_(1)
    return m, ids, weights


def exact_moe_result(m, ids, weights):
    x = m.x.double()
    y, size, h_most, h_bits = torch.zeros((m.T, m.D), device="cuda", dtype=torch.float64), 0, 0, False
    for e in range(m.E):
        w = (weights.double() * (ids == e)).sum(1, keepdim=True)
        h = (x @ m.wg[e].double().T).clamp(min=0) * (x @ m.wu[e].double().T)
        h_most = max(h_most, h.abs().max().item())
        h_bits |= bool((h.to(m.dtype).double() != h).any())
        y += w * (h @ m.wd[e].double().T)
        size = size + w.abs() * (h.abs() @ m.wd[e].double().abs().T)
    assert h_most <= 65504 and size.max().item() * 64 < 2 ** 24  # nothing on the way is rounded
    return y, h_bits


# every number of columns and of warps a team, tiles shared by 8, 4, 2 and 1 blocks, rows that begin at multiples of 16 and of 2
# bytes, lists of up to 32 pairs and of more, several launches
EXACT_MOE = [(1, 2048, 1024, 64, 8), (5, 1000, 1304, 10, 3), (32, 2048, 256, 32, 4), (33, 1024, 136, 4, 2), (40, 1001, 66, 4, 3), (64, 4096, 72, 8, 2),
             (20, 2400, 64, 2, 2), (20, 2401, 63, 2, 2), (33, 1300, 136, 4, 2), (33, 1301, 65, 4, 2), (40, 200, 33, 3, 2), (64, 700, 200, 8, 2),
             (16, 2500, 96, 40, 6), (64, 904, 264, 128, 4), (9, 4801, 40, 16, 2), (130, 1000, 200, 4, 2), (70, 1001, 65, 4, 2), (64, 8, 8, 1, 1),
             (17, 1, 1, 2, 2), (4, 2047, 1023, 8, 2), (64, 1500, 1100, 2, 1), (12, 800, 2048, 64, 8),
             (64, 64, 16, 1024, 32), (64, 65, 17, 300, 32), (64, 2401, 9, 300, 32)]


@pytest.mark.parametrize("T,D,F,E,k", EXACT_MOE)
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_moe_of_whole_numbers(T, D, F, E, k, dtype):
    m, ids, weights = exact_moe(T, D, F, E, k, dtype)
    out = m.run(ids=ids, weights=weights)[0]
    y, h_bits = exact_moe_result(m, ids, weights)
    assert torch.equal(out, y.to(FP32).to(dtype))
    # the second part of h counts (fp16 holds whole numbers up to 2048 in one)
    assert h_bits or D < 500 or dtype is FP16


@pytest.mark.parametrize("T,D,F,E,k", [(9, 1000, 64, 4, 2), (40, 1024, 72, 4, 2), (33, 136, 2000, 5, 2)])
def test_moe_of_whole_numbers_whose_elements_lie_apart(T, D, F, E, k):
    m, ids, weights = exact_moe(T, D, F, E, k, BF16)
    y, _ = exact_moe_result(m, ids, weights)
    for names in (("wg",), ("wu",), ("wd",), ("wg", "wu", "wd")):
        h, _, _ = exact_moe(T, D, F, E, k, BF16)
        for name in names:
            setattr(h, name, getattr(m, name).transpose(1, 2).contiguous().transpose(1, 2))
        assert torch.equal(h.run(ids=ids, weights=weights)[0], y.to(FP32).to(BF16)), names


@pytest.mark.parametrize("T,D,F,E,k", [(1, 2048, 1024, 64, 8), (5, 1000, 1304, 10, 3), (64, 1024, 512, 8, 2), (40, 1001, 333, 4, 3)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_moe_errors_are_the_result_s_rounding(T, D, F, E, k, dtype):
    """Of random operands, relative to the result's norm: h in two parts, the activation (2e-6) and the sums are all some
    hundred times more exact than the result's rounding in bf16 and some ten times in fp16, and add a tenth at most."""
    m = Moe(T, D, F, E, k, dtype)
    out, ids, weights = m.run()
    m.check_routes(ids, weights)
    x, y = m.x.double(), torch.zeros((T, D), device="cuda", dtype=torch.float64)
    for e in range(E):
        w = (weights.double() * (ids == e)).sum(1, keepdim=True)
        g = x @ m.wg[e].double().T
        y += w * ((g * torch.sigmoid(g) * (x @ m.wu[e].double().T)) @ m.wd[e].double().T)
    assert (out.double() - y).norm() <= 1.1 * (y.to(dtype).double() - y).norm()


# ---- norms in 8 bits: a case for each kernel that many rows choose ------------------------------------------

# (rows for each block of 64, 128, 192, 256, 384 and 512 threads, of 8, 12 and 16 elements a thread)
NARROW = [(9600, 65), (9600, 333), (9500, 511), (4800, 1001), (3000, 1501), (2400, 2047), (1200, 2501), (1300, 4001), (1250, 4095), (700, 5001),
          (650, 7001)]
# every operand there, rows that do not fill a block; 1 and 2 accesses a thread (fp32: up to 4)
RAGGED = [(4802, 1016), (1000, 2056), (1204, 5376), (1207, 5376)]


@pytest.mark.parametrize("T,D", NARROW + RAGGED)
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_norm_in_8_bits_of_many_rows(T, D, dtype):
    serve.test_norm_in_8_bits(T, D, dtype)


@pytest.mark.parametrize("T,D", NARROW[1:] + RAGGED)  # (its elements lie in the first two blocks of 128)
def test_norm_in_8_bits_of_many_rows_with_zeros_infinities_and_nan(T, D):
    serve.test_norm_in_8_bits_of_zeros_infinities_and_nan(T, D)


@pytest.mark.parametrize("T,D", NARROW)
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_norm_in_8_bits_of_many_rows_in_place_and_strided(T, D, dtype):
    serve.test_norm_in_8_bits_in_place_and_strided(T, D, dtype)


@pytest.mark.parametrize("T,D", NARROW + RAGGED)
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_norm_in_8_bits_values_are_the_nearest(T, D, dtype):
    """Against x / scale in 64 bits, with every operand there: the nearest e4m3 value, but where x / scale lies within its own
    error of the middle between two.

    That error: a sum of squares has at most 16 terms a thread and ten additions in a tree, 27 roundings of 2^-24, which the
    root halves; with the mean, eps and the root itself rho is within 2^-19 of itself.  n = y rho w_post gate is so within
    (2^-19 + 3 2^-24) |n|, r' = base + n within that and 2^-23 |base| + 2^-24 |r'|, however little of them is left in
    r'; x = r' rho w_pre adds (2^-19 + 2 2^-24) |x|, the quotient 2^-23: together less than 2^-18 |x| (1 + (|base| + |n|) / |r'|)."""
    n = serve.Norm(T, D, dtype, gate=max(1, T // 3))
    out, q, s = n.run()
    r, _, x, _ = n.exact()
    base = n.scale * n.resid.double()
    v = (x / s.double().repeat_interleave(128, 1)[:, :D].clamp(min=1e-300)).clamp(-448, 448)
    parts = (base.abs() + (r - base).abs()) / r.abs().clamp(min=1e-300)
    m, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (e - 4).clamp(min=-9))
    nearest = torch.round(v / step) * step
    middle = ((v / step).abs() % 1 - 0.5).abs() * step  # distance from there
    off = q.double() != nearest
    assert not (off & (middle > 2.0 ** -18 * v.abs() * (1 + parts))).any()
    assert ((q.double() - nearest).abs()[off] <= 1.01 * step[off]).all()


# ---- sizes beyond 32 bits ------------------------------------------------------------------------------------

def test_int4_products_beyond_32_bits():
    """Weights of more than 2^32 bytes for few tokens; expanded ones of more than 2^32 bytes for many."""
    g = gen(77)
    for M, N, K, dtype in ((1, 150001, 60000, BF16), (20, 150001, 60000, BF16), (66, 40001, 60000, FP16)):
        q = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
        x, scale = integers(g, -1, 1, (M, K), dtype), (2.0 ** -integers(g, 0, 1, (N, -(-K // 128)), FP32)).to(dtype)
        out = block.int4_product(x, q, scale, poisoned((M, N), dtype))
        at = torch.cat([torch.arange(40, device="cuda"), torch.randint(0, N, (100,), generator=g, device="cuda"), torch.arange(N - 40, N, device="cuda")])
        k = torch.arange(K, device="cuda")
        w = ((q[at][:, k // 2].int() >> (4 * (k % 2)) & 15) - 8).double() * scale[at].double()[:, k // 128]
        assert torch.equal(out[:, at], (x.double() @ w.T).to(FP32).to(dtype))
        assert torch.isfinite(out).all()


def test_norm_in_8_bits_beyond_32_bits():
    T, D = 1 << 20, 4104
    r = torch.empty((T, D), device="cuda", dtype=BF16)
    for i in range(0, T, 1 << 17):
        r[i:i + (1 << 17)].normal_(generator=gen(i))
    out, q, s = torch.empty_like(r), torch.empty((T, D), device="cuda", dtype=serve.E4M3), poisoned((T, 33), FP32)
    block.residual_norm_quantize(r, out, q, s)
    for rows in (slice(0, 50), slice(T // 2 - 25, T // 2 + 25), slice(T - 50, T)):
        assert torch.equal(out[rows], r[rows])
        x = r[rows].double()
        x = x / (x.square().mean(1, keepdim=True) + serve.EPS).sqrt()
        sc = s[rows].double().repeat_interleave(128, 1)[:, :D]
        close(s[rows], torch.nn.functional.pad(x, (0, 120)).reshape(50, 33, 128).abs().amax(2) / 448, 2.0 ** -17 * s[rows].double(), "scales")
        close(q[rows].double() * sc, x, x.abs() * (2.0 ** -4 + 2.0 ** -17) + 2.0 ** -10 * sc, "values")
    assert torch.isfinite(s).all()


def test_clipping_beyond_32_bits():
    n = (1 << 32) + 12347
    t = torch.full((n,), 0.5, device="cuda", dtype=BF16)
    t[-3:] = 64.0
    norm = poisoned((1,), FP32)
    exact = ((n - 3) * 0.25 + 3 * 4096.0) ** 0.5
    block.clip_gradients([t], exact / 4, norm)
    assert abs(norm.item() - exact) <= 24 * 2.0 ** -24 * exact
    # a quarter, but for eps and the norm's rounding: within a rounding to bf16
    for part, v in ((t[:1 << 20], 0.125), (t[1 << 31:(1 << 31) + 4096], 0.125), (t[(1 << 32) - 4096:-3], 0.125), (t[-3:], 16.0)):
        assert ((part.double() - v).abs() <= 2.0 ** -8 * v).all()
