"""The operators that serve the feed-forward sub-block against plain 64-bit forms: norms with 8-bit results,
products with 4-bit weights and their quantiser, clipping, mixtures of experts.

Tolerances.  u is a type's unit roundoff, eps / 2 (bf16 2^-8, fp16 2^-11, fp32 2^-24, e4m3 2^-4).  Sums of n products
in fp32 are off by at most (n + 16) 2^-23 of the sum of the products' sizes.  A result's own rounding adds u of its
size; below the type's normal range half of its smallest step.
"""
import pytest
import torch

from paper_1802_06905_b200 import block
from test_gpu_block import BF16, E4M3, FP16, FP32, TINY, U, close, gen, normal, poisoned, sum_err

pytestmark = pytest.mark.gpu

EPS = 1e-6


# ---- norms with 8-bit results ---------------------------------------------------------------------

class Norm:
    def __init__(self, T, D, dtype=BF16, gate=0, post=True, pre=True, seed=0):
        g = gen(seed + 5 * T + 11 * D)
        self.T, self.D, self.dtype = T, D, dtype
        self.scale = 0.875
        self.resid = normal(g, (T, D), dtype, 2.0)
        self.block = normal(g, (T, D), dtype, 0.7)
        self.w_post = (1 + 0.2 * normal(g, (D,), FP32)).to(dtype) if post else None
        self.w_pre = (1 + 0.2 * normal(g, (D,), FP32)).to(dtype) if pre else None
        self.rows = gate
        groups = -(-T // gate) if gate else 1
        self.gate = normal(g, (groups, D), dtype, 0.5) if gate is not None else None
        if gate is None:
            self.rows = 0

    def run(self, q=None, q_scale=None, resid_out=None, norm_out=None, resid=None, **kw):
        T, D = self.T, self.D
        q = torch.full((T, D), 3.0, device="cuda").to(E4M3) if q is None else q
        q_scale = poisoned((T, -(-D // 128)), FP32) if q_scale is None else q_scale
        resid_out = poisoned((T, D), self.dtype) if resid_out is None else resid_out
        block.residual_norm_quantize(self.resid if resid is None else resid, resid_out, q, q_scale, norm_out=norm_out,
                                     block=self.block, w_post=self.w_post, gate=self.gate, w_pre=self.w_pre,
                                     rows_per_gate=self.rows, scale=self.scale, eps=EPS, **kw)
        return resid_out, q, q_scale

    def exact(self):
        """r', x and how far 32 bits may be from them."""
        T, D = self.T, self.D
        n = self.block.double()
        en = torch.zeros_like(n)
        if self.w_post is not None:
            n = n / (n.square().mean(1, keepdim=True) + EPS).sqrt() * self.w_post.double()
            en = sum_err(D) * n.abs()
        if self.gate is not None:
            at = torch.arange(T, device="cuda") // self.rows if self.rows else torch.zeros(T, dtype=torch.long, device="cuda")
            n, en = n * self.gate.double()[at], en * self.gate.double()[at].abs()
        base = self.scale * self.resid.double()
        r = base + n
        er = en + 2.0 ** -21 * (base.abs() + n.abs())
        ms = r.square().mean(1, keepdim=True) + EPS
        w = 1.0 if self.w_pre is None else self.w_pre.double()
        x = r / ms.sqrt() * w
        ex = er / ms.sqrt() * abs(w) + x.abs() * (sum_err(D) + (er.square().mean(1, keepdim=True) / ms).sqrt() + 2.0 ** -21)
        return r, er, x, ex

    def check(self, resid_out, q, q_scale, what=""):
        r, er, x, ex = self.exact()
        close(resid_out, r, 1.01 * (er + U[self.dtype] * r.abs()) + TINY[self.dtype], what + " resid_out")
        T, D = self.T, self.D
        pad = (0, -D % 128)
        xb = torch.nn.functional.pad(x, pad).reshape(T, -1, 128)
        eb = torch.nn.functional.pad(ex, pad).reshape(T, -1, 128)
        amax, e = xb.abs().amax(2), eb.amax(2)
        close(q_scale, amax / 448, 1.01 * e / 448 + 2.0 ** -23 * amax / 448, what + " q_scale")
        s = q_scale.double().repeat_interleave(128, 1)[:, :D]
        # a scale that is off by a little, and the quotient's rounding: a step of 2^-4 of the value, at least 2^-10 of the scale
        close(q.double() * s, x, 1.01 * (ex + 2.0 ** -4 * x.abs() + 2.0 ** -10 * s) + 2.0 ** -22 * x.abs(), what + " q")


SHAPES = [(1, 4096), (1, 1), (2, 128), (3, 127), (5, 129), (4, 520), (9, 1000), (33, 2048), (17, 4100), (130, 264),
          (5, 8192), (3, 16384), (2, 16392), (3, 20001), (1300, 1024), (1200, 4096), (2500, 1000), (2400, 1001), (5000, 65),
          (700, 8192), (1300, 5001)]


@pytest.mark.parametrize("T,D", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_norm_in_8_bits(T, D, dtype):
    n = Norm(T, D, dtype, gate=(0, None, 1, max(1, T // 3))[(T + D) % 4], post=(T + D) % 3 != 0, pre=D % 5 != 0)
    n.check(*n.run(), f"{T}x{D}")
    # x itself, if asked for: the 8-bit values are those of x before its rounding, which in 32 bits is none
    x = poisoned((T, D), dtype)
    out, q, s = n.run(norm_out=x)
    n.check(out, q, s, f"{T}x{D} with x")
    if dtype is FP32:
        q2, s2 = torch.zeros_like(q), poisoned(s.shape, FP32)
        block.quantize_blocks(x, q2, s2)
        assert torch.equal(s, s2)
        assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8))
    r, er, xe, ex = n.exact()
    close(x, xe, 1.01 * (ex + U[dtype] * xe.abs()) + TINY[dtype], "norm_out")
    assert block.status() == (0, 0)


@pytest.mark.parametrize("T,D", [(3, 256), (1300, 512), (2400, 1001), (2, 16640)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_norm_in_8_bits_in_place_and_strided(T, D, dtype):
    n = Norm(T, D, dtype)
    exp = n.run()
    r = n.resid.clone()
    got = n.run(resid=r, resid_out=r)
    for a, b in zip(got, exp):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # rows apart, beginning anywhere; scales with the tokens next to one another; what lies between stays
    for at in (0, 4, 3):
        big = torch.full((T, D + 24), 5.0, device="cuda").to(E4M3)
        q = big[:, at:at + D]
        scales = torch.full((D // 128 + 3, T + 1), -1.0, device="cuda")
        q_scale = scales[1:1 + -(-D // 128), :T].t()
        out, _, _ = n.run(q=q, q_scale=q_scale)
        n.check(out, q, q_scale, f"offset {at}")
        mask = torch.ones_like(big, dtype=torch.bool)
        mask[:, at:at + D] = False
        assert (big.float()[mask] == 5.0).all()
        inside = torch.zeros_like(scales, dtype=torch.bool)
        inside[1:1 + -(-D // 128), :T] = True
        assert (scales[~inside] == -1.0).all()


@pytest.mark.parametrize("T,D", [(4, 512), (4, 333), (3, 17000), (1300, 512), (2400, 333)])
def test_norm_in_8_bits_of_zeros_infinities_and_nan(T, D):
    for dtype in (BF16, FP32):
        resid = torch.randn((T, D), device="cuda").to(dtype)
        resid[0] = 0
        resid[1, 5] = float("inf")
        resid[2, 200] = float("nan")
        out, q, s = torch.empty_like(resid), torch.empty((T, D), dtype=E4M3, device="cuda"), poisoned((T, -(-D // 128)), FP32)
        x = torch.empty_like(resid)
        block.residual_norm_quantize(resid, out, q, s, norm_out=x)
        assert (q[0].float() == 0).all() and (s[0] == 0).all()
        # an infinite row norm: the infinite element is NaN, the others 0
        f = q[1].float()
        assert torch.isnan(x[1, 5]) and torch.isnan(f[5]) and torch.isnan(s[1, 0])
        assert torch.isnan(f[:128]).all() and (f[128:] == 0).all() and (s[1, 1:] == 0).all()
        assert torch.isnan(q[2].float()).all() and torch.isnan(s[2]).all()
        assert not torch.isnan(s[3:]).any() and not torch.isnan(q[3:].float()).any()
    assert block.status() == (0, 0)


def test_norm_in_8_bits_without_block_or_weights():
    for T, D in ((6, 384), (1300, 384), (2, 100)):
        resid = torch.randn((T, D), device="cuda").to(FP32)
        out, q, s = torch.empty_like(resid), torch.empty((T, D), dtype=E4M3, device="cuda"), poisoned((T, -(-D // 128)), FP32)
        block.residual_norm_quantize(resid, out, q, s)
        assert torch.equal(out, resid)
        r = resid.double()
        x = r / (r.square().mean(1, keepdim=True) + EPS).sqrt()
        sc = s.double().repeat_interleave(128, 1)[:, :D]
        close(q.double() * sc, x, x.abs() * (2.0 ** -4 + 2 * sum_err(D)) + 2.0 ** -10 * sc, "q")


def test_norm_in_8_bits_of_nothing():
    for T, D in ((0, 256), (3, 0)):
        e = torch.empty((T, D), device="cuda", dtype=BF16)
        block.residual_norm_quantize(e, torch.empty_like(e), torch.empty((T, D), device="cuda", dtype=E4M3),
                                     torch.empty((T, -(-D // 128)), device="cuda"))
    torch.cuda.synchronize()


# ---- 4-bit weights --------------------------------------------------------------------------------

U8 = torch.uint8


class Int4:
    """Random codes, scales, zero points and tokens; exact values and tolerances."""

    def __init__(self, M, N, K, group=128, dtype=BF16, scale=None, zero=False, seed=0):
        g = gen(seed + 3 * M + 5 * N + 7 * K + group)
        self.M, self.N, self.K, self.group, self.dtype = M, N, K, group, dtype
        groups = -(-K // group)
        self.x = normal(g, (M, K), dtype)
        self.q = torch.randint(0, 256, (N, -(-K // 2)), generator=g, device="cuda", dtype=U8)
        self.scale = (torch.exp(0.3 * normal(g, (N, groups), FP32)) * (0.2 * max(K, 1) ** -0.5)).to(scale or dtype)
        # (the upper halves of the bytes do not count)
        self.zero = torch.randint(0, 256, (N, groups), generator=g, device="cuda", dtype=U8) if zero else None

    def run(self, out=None, **kw):
        out = poisoned((self.M, self.N), self.dtype) if out is None else out
        return block.int4_product(self.x, self.q, self.scale, out, zero=self.zero, group=self.group, **kw)

    def weights(self):
        """q, z and s of every element, in 64 bits."""
        at = torch.arange(self.K, device="cuda")
        q = (self.q[:, at // 2].int() >> (4 * (at % 2)) & 15).double()
        z = torch.full_like(q, 8.0) if self.zero is None else (self.zero.int() & 15).double()[:, at // self.group]
        return q, z, self.scale.double()[:, at // self.group]

    def check(self, out, what=""):
        q, z, s = self.weights()
        x, u = self.x.double(), U[self.dtype]
        w = s * (q - z)
        c = x @ w.T
        if self.M <= 64:  # sums of 16 + q and 16 + z
            e = sum_err(self.K) * (x.abs() @ (s.abs() * (32 + q + z)).T)
        else:             # weights rounded to the type
            e = (u + sum_err(self.K)) * (x.abs() @ w.abs().T) + 2.0 ** -25 * x.abs().sum(1, keepdim=True)
        close(out, c, 1.01 * (e + u * c.abs()) + TINY[self.dtype], what)


INT4_SHAPES = [(1, 64, 64), (1, 1, 1), (2, 16, 128), (3, 17, 33), (1, 4096, 1024), (4, 33, 256), (5, 130, 1000), (8, 4800, 384),
               (9, 100, 4200), (16, 5000, 520), (17, 48, 96), (23, 75, 2056), (33, 129, 130), (64, 200, 640), (65, 256, 256),
               (130, 72, 1001), (300, 513, 320), (1, 8192, 8192), (64, 31, 16416)]


@pytest.mark.parametrize("M,N,K", INT4_SHAPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_int4_product(M, N, K, group, dtype):
    scale = (dtype, FP32, BF16, FP16)[(M + N + K + group // 32) % 4]
    for zero in (False, True):
        c = Int4(M, N, K, group, dtype, scale, zero)
        c.check(c.run(), f"{M}x{N}x{K} group {group} zero {zero}")
    assert block.status() == (0, 0)


@pytest.mark.parametrize("M", [1, 3, 12, 40, 100])
@pytest.mark.parametrize("K", [256, 264, 300])
def test_int4_strided_operands(M, K):
    c = Int4(M, 72, K, 32, BF16, zero=True)

    def transposed(t):
        return t.t().contiguous().t()

    def shifted(by, pad):
        def f(t):
            big = torch.full((t.shape[0], t.shape[1] + pad), 9, device="cuda").to(t.dtype)
            big[:, by:by + t.shape[1]] = t
            return big[:, by:by + t.shape[1]]
        return f

    def every_other(t):
        big = torch.full((t.shape[0], 2 * t.shape[1]), 9, device="cuda").to(t.dtype)
        big[:, ::2] = t
        return big[:, ::2]
    exp = c.run()
    for store in (transposed, shifted(0, 16), shifted(4, 8), shifted(8, 24), shifted(1, 3), every_other):
        h = Int4(M, 72, K, 32, BF16, zero=True)
        for name in ("x", "q", "scale", "zero"):
            setattr(h, name, store(getattr(c, name)))
        big = torch.full((M + 2, 80), 7.0, device="cuda", dtype=BF16)
        out = big[1:M + 1, 3:75]
        h.run(out=out)
        assert torch.equal(out, exp)  # the same sums in the same order
        big[1:M + 1, 3:75] = 7.0
        assert (big == 7.0).all()
        wide = torch.full((72, M), 7.0, device="cuda", dtype=BF16)
        assert torch.equal(h.run(out=wide.t()), exp)


def test_int4_rows_with_a_shared_token_and_shared_weights():
    c = Int4(5, 40, 320, 64, FP16)
    c.x = c.x[:1].expand(5, 320)
    c.q, c.scale = c.q[:1].expand(40, 160), c.scale[:1].expand(40, 5)
    c.check(c.run(), "broadcast")


@pytest.mark.parametrize("M", [9, 40])
@pytest.mark.parametrize("N,K", [(34, 8), (34, 24), (18, 136), (50, 264), (129, 40)])
def test_int4_short_rows(M, N, K):
    """Rows of less than the bytes that are read of one at once, side by side, overlapping and all the same."""
    c = Int4(M, N, K, 32, BF16, zero=True)
    c.check(c.run(), "side by side")
    bytes_ = K // 2
    flat = c.q.reshape(-1)
    for pitch in (4, 0):
        c.q = flat[4:].as_strided((N, bytes_), (pitch, 1), 4) if (N - 1) * pitch + bytes_ + 4 <= flat.numel() else c.q
        c.check(c.run(), f"{pitch} bytes apart")


def test_int4_of_nothing():
    for M, N, K in ((0, 8, 64), (3, 0, 64), (3, 8, 0)):
        c = Int4(M, N, K)
        assert (c.run() == 0).all()


def test_int4_infinities_and_nan():
    for M in (4, 100):
        c = Int4(M, 64, 512)
        c.x[1, 7] = float("inf")
        c.x[2, 300] = float("nan")
        c.scale[9, 2] = float("nan")
        out = c.run()
        bad = ~torch.isfinite(out)
        assert bad[2].all() and bad[:, 9].all()
        bad[1:3], bad[:, 9] = False, False
        assert not bad.any()


def test_int4_offsets_beyond_32_bits():
    """Rows so far apart that their offsets pass 2^32 bytes."""
    N, K = 3, 256
    c = Int4(2, N, K)
    big = torch.empty(3 * (1 << 31) + 256, device="cuda", dtype=U8)
    q = big.as_strided((N, K // 2), (1 << 31, 1))
    q.copy_(c.q)
    exp = c.run()
    c.q = q
    assert torch.equal(c.run(), exp)
    c.x = c.x.repeat(40, 1)
    c.M = 80
    c.check(c.run(), "many tokens")


def quantized(w, group, zero, stype):
    """The definition, operation by operation in fp32."""
    N, K = w.shape
    groups = -(-K // group)
    f = torch.nn.functional.pad(w.float(), (0, groups * group - K)).reshape(N, groups, group)
    if zero:
        lo, hi = f.amin(2, keepdim=True).clamp(max=0), f.amax(2, keepdim=True).clamp(min=0)
        s = (hi - lo) / torch.full_like(lo, 15.0)
    else:
        s = f.abs().amax(2, keepdim=True) / torch.full((N, groups, 1), 7.0, device="cuda")
    s = torch.where(torch.isfinite(f).all(2, keepdim=True), s, float("nan"))
    st = s.to(stype)
    sf = st.float()
    ok = torch.isfinite(sf) & (sf > 0)
    by = torch.where(ok, sf, 1.0)
    z = (-lo / by).round().clamp(0, 15) if zero else torch.full_like(sf, 8.0)
    q = ((f / by).round() + z).clamp(0, 15)
    z = torch.where(ok, z, 8.0)
    q = torch.where(ok, q, 8.0).reshape(N, -1)[:, :K].to(torch.int32)
    q = torch.nn.functional.pad(q, (0, K % 2))
    return (q[:, ::2] | q[:, 1::2] << 4).to(U8), st[:, :, 0], z[:, :, 0].to(U8)


@pytest.mark.parametrize("N,K", [(1, 1), (3, 32), (5, 33), (17, 256), (64, 1000), (9, 2048), (2, 5001), (70000, 40)])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("zero", [False, True])
def test_quantize_groups(N, K, dtype, zero):
    g = gen(N + K)
    w = normal(g, (N, K), dtype, 0.02) + (0.01 if zero else 0)
    if N > 3:
        w[1] = 0
        w[2, : min(K, 40)] = 0.5
        w[3, K // 2] = float("inf")
        w[3, 0] = float("nan")
    for group in (32, 64, 128):
        for stype in (BF16, FP16, FP32):
            groups = -(-K // group)
            q = torch.full((N, -(-K // 2)), 77, device="cuda", dtype=U8)
            s = poisoned((N, groups), stype)
            z = torch.full((N, groups), 99, device="cuda", dtype=U8) if zero else None
            block.quantize_groups(w, q, s, zero=z, group=group)
            eq, es, ez = quantized(w, group, zero, stype)
            assert torch.equal(torch.nan_to_num(s, nan=-1), torch.nan_to_num(es, nan=-1))
            assert torch.equal(q, eq)
            assert z is None or torch.equal(z, ez)


def test_quantize_groups_strided_and_back():
    w = normal(gen(4), (100, 330), FP32, 0.1)
    q0, s0, z0 = quantized(w, 32, True, BF16)
    store = torch.zeros((330, 100), device="cuda").t()
    store.copy_(w)
    q, s, z = (torch.zeros((c, 100), device="cuda", dtype=t).t() for c, t in ((165, U8), (11, BF16), (11, U8)))
    block.quantize_groups(store, q, s, zero=z, group=32)
    assert torch.equal(q, q0) and torch.equal(s, s0) and torch.equal(z, z0)
    # what the product makes of them is within half a step of w, and the scale's and zero point's rounding
    out = poisoned((330, 100), BF16)
    block.int4_product(torch.eye(330, device="cuda", dtype=BF16), q, s, out, zero=z, group=32)
    step = s.double().repeat_interleave(32, 1)[:, :330]
    close(out.t(), w.double(), 1.1 * step + 2.0 ** -7 * w.double().abs(), "back")


def test_quantize_groups_of_nothing():
    for N, K in ((0, 64), (4, 0)):
        block.quantize_groups(torch.empty((N, K), device="cuda"), torch.empty((N, K // 2), device="cuda", dtype=U8),
                              torch.empty((N, -(-K // 128)), device="cuda"))


# ---- the norm of a list of gradients, and clipping --------------------------------------------------

def gradients(shapes, seed=0, scale=0.02):
    g = gen(seed)
    return [normal(g, shape, dtype, scale) for shape, dtype in shapes]


def norm64(ts):
    return sum(t.double().square().sum().item() for t in ts) ** 0.5


def check_clipped(outs, grads, norm, max_norm, eps=1e-6, what=""):
    """Squares in fp32 over at most 34 elements, then 64 bits: 40 2^-24 of the sum, half of that of its root."""
    exact = norm64(grads)
    assert abs(norm.item() - exact) <= 24 * 2.0 ** -24 * exact, (what, norm.item(), exact)
    factor = min(1.0, max_norm / (exact + eps))
    for o, g in zip(outs, grads):
        assert o.dtype == g.dtype and o.shape == g.shape
        v = g.double() * factor
        close(o, v, v.abs() * (U[g.dtype] * 1.01 + 30 * 2.0 ** -24) + 2.0 ** -25 * (g.dtype == FP16) + 1e-45, what)


LISTS = [[((1,), FP32)], [((7,), BF16), ((0,), FP32), ((3, 5), FP16)], [((1000, 1000), BF16)], [((300, 700), FP32), ((700,), FP32)],
         [((256, 700), BF16), ((700, 256), FP16), ((256,), FP32)] * 17, [((33,), FP32)] * 700, [((4096, 4097), FP16), ((5, 3, 7, 11), BF16)],
         [((2, 8191), BF16), ((1, 8193), BF16), ((1, 4095), FP32), ((1, 4097), FP32)]]


@pytest.mark.parametrize("shapes", LISTS, ids=range(len(LISTS)))
@pytest.mark.parametrize("part", [0.25, 4.0])
def test_clip_gradients(shapes, part):
    grads = gradients(shapes)
    exact = norm64(grads)
    norm = poisoned((1,), FP32)
    outs = [poisoned(g.shape, g.dtype) for g in grads]
    block.clip_gradients(grads, part * exact, norm, outs=outs)
    check_clipped(outs, grads, norm, part * exact, what="outs")
    alone = poisoned((1,), FP32)
    block.gradient_norm(grads, alone)
    assert torch.equal(alone, norm)
    # in place, the list made once; and with the norm given
    mine = [g.clone() for g in grads]
    lst = block.TensorList(mine)
    norm2 = poisoned((1,), FP32)
    block.clip_gradients(lst, part * exact, norm2)
    assert torch.equal(norm2, norm)
    for a, b in zip(mine, outs):
        assert torch.equal(a, b)
    more = [poisoned(g.shape, g.dtype) for g in grads]
    block.clip_gradients(grads, part * exact, norm, outs=more, norm_given=True)
    for a, b in zip(more, outs):
        assert torch.equal(a, b)


def test_clip_views_of_a_buffer_that_begin_anywhere():
    flat = normal(gen(5), (200001,), BF16)
    cuts = [0, 1, 4, 17, 1000, 9192, 9193, 30000, 131072, 200001]
    out = torch.full_like(flat, 7.0)
    # results two elements further on than the gradients: no common alignment
    target = torch.full((200005,), 7.0, device="cuda", dtype=BF16)
    grads = [flat[a:b] for a, b in zip(cuts, cuts[1:])]
    norm = poisoned((1,), FP32)
    block.clip_gradients(grads, 1.0, norm, outs=[target[a + 3:b + 3] for a, b in zip(cuts, cuts[1:])])
    check_clipped([target[3:200004]], [flat], norm, 1.0)
    assert (target[:3] == 7).all() and target[200004] == 7
    block.clip_gradients(grads[1:-1], 1.0, norm, outs=[out[a:b] for a, b in zip(cuts, cuts[1:])][1:-1])
    assert out[0] == 7 and (out[131072:] == 7).all() and not (out[1:131072] == 7).any()


def test_clip_strided_tensors():
    g = gen(6)
    whole = [normal(g, s, t) for s, t in (((64, 3000), BF16), ((500, 40), FP32), ((6, 4, 10, 8), FP16), ((90, 70), BF16))]
    views = [whole[0][:, 7:2900], whole[1][::2, ::3], whole[2].permute(0, 3, 1, 2), whole[3].t()]
    before = [w.clone() for w in whole]
    copies = [v.clone() for v in views]
    norm = poisoned((1,), FP32)
    m = 0.5 * norm64(copies)
    block.clip_gradients(views, m, norm)
    check_clipped(views, copies, norm, m)
    for w, b, v in zip(whole, before, ((slice(None), slice(7, 2900)), (slice(None, None, 2), slice(None, None, 3)))):
        w, b = w.clone(), b.clone()
        w[v], b[v] = 0, 0
        assert torch.equal(w, b)  # what lies between stays


def test_clip_extreme_values():
    for value, dtype in ((1e30, FP32), (3e38, BF16), (1e-30, FP32), (1e-38, BF16), (6e-8, FP16), (6e4, FP16)):
        x = torch.full((70001,), value, device="cuda").to(dtype)
        v = x[0].item()
        norm = poisoned((1,), FP32)
        block.gradient_norm([x], norm)
        exact = abs(v) * 70001 ** 0.5
        if exact > 3.4e38:
            assert norm.item() == float("inf")
        else:
            assert abs(norm.item() - exact) <= 2.0 ** -19 * exact + 1e-45, (value, dtype)
    zeros = [torch.zeros(5000, device="cuda"), torch.zeros(3, device="cuda", dtype=BF16)]
    block.clip_gradients(zeros, 1.0, norm)
    assert norm.item() == 0 and all((z == 0).all() for z in zeros)
    # one element of 1e-20 among zeros
    zeros[0][4321] = 1e-25
    block.gradient_norm(zeros, norm)
    assert abs(norm.item() - 1e-25) < 1e-31


def test_clip_infinities_and_nan():
    a, b = torch.ones(9000, device="cuda", dtype=BF16), torch.ones(100, device="cuda")
    a[5] = float("inf")
    norm = poisoned((1,), FP32)
    block.clip_gradients([a, b], 1.0, norm)
    assert norm.item() == float("inf")
    assert torch.isnan(a[5]) and (a[6:] == 0).all() and (b == 0).all()
    a, b = torch.ones(9000, device="cuda", dtype=BF16), torch.ones(100, device="cuda")
    a[5] = float("nan")
    block.clip_gradients([a, b], 1.0, norm)
    assert torch.isnan(norm).all() and torch.isnan(a).all() and torch.isnan(b).all()


def test_clip_without_a_limit():
    a = torch.full((5000,), 3.0, device="cuda", dtype=BF16)
    norm = poisoned((1,), FP32)
    block.clip_gradients([a], float("inf"), norm)
    assert abs(norm.item() - 3.0 * 5000 ** 0.5) < 1e-3 and (a == 3.0).all()
    a[7] = float("inf")
    block.clip_gradients([a], float("inf"), norm)  # the formula's quotient is none
    assert norm.item() == float("inf") and torch.isnan(a).all()


def test_clip_of_nothing():
    norm = poisoned((1,), FP32)
    block.clip_gradients([torch.empty(0, device="cuda"), torch.empty((3, 0), device="cuda")], 1.0, norm)
    assert norm.item() == 0
    block.gradient_norm([torch.empty(0, device="cuda")], norm.fill_(3))
    assert norm.item() == 0


def test_clip_refuses_results_that_meet_others():
    a = torch.ones(100, device="cuda")
    norm = poisoned((1,), FP32)
    for grads, outs in (([a, a], None), ([a[:60], a[50:]], None), ([a[:50]], [a[10:60]]), ([a[:1]], [norm])):
        with pytest.raises(block.CconvError):
            block.clip_gradients(grads, 1.0, norm, outs=outs)
    block.clip_gradients([a, a], 1.0, norm, outs=[torch.empty_like(a), torch.empty_like(a)])  # read twice: counted twice
    assert abs(norm.item() - 200 ** 0.5) < 1e-5
    with pytest.raises(ValueError):
        block.clip_gradients([a], 1.0, norm, outs=[a[:50]])
    with pytest.raises(ValueError):
        block.TensorList([a, torch.ones(3)])
    with pytest.raises(ValueError):
        block.TensorList([torch.ones((4, 4, 4), device="cuda")[::2, ::2, ::2]])
    for bad in (-1.0, float("nan")):
        with pytest.raises(block.CconvError):
            block.clip_gradients([a], bad, norm)


# ---- mixture of experts -----------------------------------------------------------------------------

class Moe:
    """A layer's operands, exact values and tolerances."""

    def __init__(self, T, D, F, E, k, dtype=BF16, act="silu", normalize=True, seed=0):
        g = gen(seed + T + 3 * D + 5 * F + 7 * E + 11 * k)
        self.T, self.D, self.F, self.E, self.k, self.dtype, self.act, self.normalize = T, D, F, E, k, dtype, act, normalize
        self.x = normal(g, (T, D), dtype)
        self.router = normal(g, (E, D), dtype, max(D, 1) ** -0.5)
        self.wg, self.wu = (normal(g, (E, F, D), dtype, max(D, 1) ** -0.5) for _ in range(2))
        self.wd = normal(g, (E, D, F), dtype, max(F, 1) ** -0.5)

    def run(self, ids=None, weights=None, out=None, **kw):
        routed = ids is None
        out = poisoned((self.T, self.D), self.dtype) if out is None else out
        ids = torch.full((self.T, self.k), -7, device="cuda", dtype=torch.int32) if routed else ids
        weights = poisoned((self.T, self.k), FP32) if weights is None else weights
        return block.moe_forward(self.x, self.router if routed else None, self.wg, self.wu, self.wd, out, ids, weights,
                                 act=block.ACTS[self.act], normalize=self.normalize, **kw)

    def check_routes(self, ids, weights, what=""):
        x, r = self.x.double(), self.router.double()
        logits = x @ r.T
        e = sum_err(self.D) * (x.abs() @ r.abs().T).amax(1, keepdim=True)
        assert (ids >= 0).all() and (ids < self.E).all(), what
        assert all(len(set(row)) == self.k for row in ids.tolist()), what
        got = logits.gather(1, ids.long())
        best = logits.sort(1, descending=True)[0][:, :self.k]
        assert ((got - best).abs() <= 2 * e).all(), what  # the right ones, in order, but for ties within the sums' rounding
        p = torch.softmax(got if self.normalize else logits, 1)
        p = p if self.normalize else p.gather(1, ids.long())
        # a shift of e in every logit changes p by 2 e of itself; the exponential, the sum and the quotient
        close(weights, p, p * (2 * e * 1.01 + (self.E + 40) * 2.0 ** -23), what + " weights")

    def check_out(self, out, ids, weights, what=""):
        from test_gpu_block import act64
        u = U[self.dtype]
        y = torch.zeros((self.T, self.D), device="cuda", dtype=torch.float64)
        ey = torch.zeros_like(y)
        x = self.x.double()
        for e in range(self.E):
            w = (weights.double() * (ids == e)).sum(1)
            rows = (ids == e).any(1).nonzero()[:, 0]
            if not len(rows):
                continue
            xs, wg, wu, wd = x[rows], self.wg[e].double(), self.wu[e].double(), self.wd[e].double()
            g, v = xs @ wg.T, xs @ wu.T
            eg, ev = sum_err(self.D) * (xs.abs() @ wg.abs().T), sum_err(self.D) * (xs.abs() @ wu.abs().T)
            a, _ = act64(self.act, g)
            h = a * v
            # as the feed-forward block's; h in two parts is rounded to u^2
            eh = 1.13 * eg * (v.abs() + ev) + (a.abs() + 1e-6) * ev + 2.0 ** -20 * (h.abs() + g.abs() * v.abs()) + u * u * h.abs() + TINY[self.dtype]
            p = w[rows, None]
            y[rows] += p * (h @ wd.T)
            ey[rows] += p.abs() * (eh @ wd.abs().T + sum_err(2 * self.F + 2 * self.k) * (h.abs() @ wd.abs().T))
        close(out, y, 1.01 * (ey + u * y.abs()) + TINY[self.dtype], what + " out")


MOE_SHAPES = [(1, 64, 64, 4, 2), (1, 2048, 1024, 64, 8), (2, 8, 8, 1, 1), (3, 72, 40, 5, 5), (5, 1000, 1304, 10, 3), (7, 65, 33, 6, 2),
              (8, 512, 136, 16, 4), (9, 130, 264, 3, 1), (16, 256, 96, 40, 6), (17, 1, 1, 9, 3), (31, 384, 200, 128, 8),
              (33, 96, 120, 7, 7), (64, 512, 256, 20, 4), (65, 128, 72, 12, 3), (130, 64, 136, 4, 2), (4, 4800, 64, 8, 2),
              (6, 40, 16, 1000, 32), (40, 66, 34, 300, 5)]


@pytest.mark.parametrize("T,D,F,E,k", MOE_SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_moe_forward(T, D, F, E, k, dtype):
    act = ["silu", "gelu", "gelu_tanh", "relu"][(T + D) % 4]
    m = Moe(T, D, F, E, k, dtype, act, normalize=(T + F) % 2 == 0)
    out, ids, weights = m.run()
    what = f"{T}x{D}x{F} {k} of {E}"
    m.check_routes(ids, weights, what)
    m.check_out(out, ids, weights, what)
    # the same choice given: the same result
    again, _, _ = m.run(ids=ids, weights=weights)
    assert torch.equal(again, out)


def test_moe_ties_and_order():
    """Whole numbers, so that scores are exact and many are equal: the lower number goes first."""
    g = gen(9)
    m = Moe(40, 64, 32, 24, 6)
    m.x = torch.randint(-2, 3, (40, 64), generator=g, device="cuda").to(BF16)
    m.router = torch.randint(-1, 2, (24, 64), generator=g, device="cuda").to(BF16)
    m.x[3] = 0
    m.router[5] = m.router[4]
    out, ids, weights = m.run()
    logits = m.x.double() @ m.router.double().T
    assert torch.equal(ids.long(), torch.sort(logits, dim=1, descending=True, stable=True)[1][:, :6])
    assert ids[3].tolist() == list(range(6)) and torch.allclose(weights[3], torch.full((6,), 1 / 6, device="cuda"))
    m.check_out(out, ids, weights)


def test_moe_given_choices():
    """Numbers that are no expert's, experts named twice, negative and zero weights, one expert for all, none for some."""
    g = gen(10)
    for T in (1, 6, 40, 70):
        m = Moe(T, 128, 72, 8, 5)
        ids = torch.randint(-3, 11, (T, 5), generator=g, device="cuda", dtype=torch.int32)
        weights = normal(g, (T, 5), FP32)
        weights[0, 1] = 0
        ids[T // 2] = 3
        if T > 1:
            ids[1] = -1
        out, _, _ = m.run(ids=ids, weights=weights)
        m.check_out(out, ids, weights, f"T {T}")
        assert T == 1 or (out[1] == 0).all()
        ids.fill_(7)
        m.check_out(m.run(ids=ids, weights=weights)[0], ids, weights, "one expert")
        ids.fill_(1 << 30)
        assert (m.run(ids=ids, weights=weights)[0] == 0).all()


@pytest.mark.parametrize("T", [1, 5, 70])
@pytest.mark.parametrize("D,F", [(128, 96), (100, 60), (51, 33)])
def test_moe_strided_operands(T, D, F):
    m = Moe(T, D, F, 6, 3, FP16)
    exp = m.run()

    def transposed(t):
        return t.transpose(-1, -2).contiguous().transpose(-1, -2)

    def padded(by, pad):
        def f(t):
            big = torch.full((*t.shape[:-1], t.shape[-1] + pad), 9.0, device="cuda", dtype=t.dtype)
            big[..., by:by + t.shape[-1]] = t
            return big[..., by:by + t.shape[-1]]
        return f

    def experts_inside(t):  # experts next to one another for each row
        return t.transpose(0, 1).contiguous().transpose(0, 1) if t.dim() == 3 else t
    for store in (transposed, padded(8, 16), padded(2, 4), padded(1, 3), experts_inside):
        h = Moe(T, D, F, 6, 3, FP16)
        for name in ("x", "router", "wg", "wu", "wd"):
            setattr(h, name, store(getattr(m, name)))
        big = torch.full((T + 1, D + 3), 7.0, device="cuda", dtype=FP16)
        ids = torch.full((3, T), -1, device="cuda", dtype=torch.int32).t()
        got = block.moe_forward(h.x, h.router, h.wg, h.wu, h.wd, big[1:, 2:D + 2], ids, torch.empty((3, T), device="cuda").t())
        for a, b in zip(got, exp):
            assert torch.equal(a, b)
        big[1:, 2:D + 2] = 7.0
        assert (big == 7).all()
    # gate and up as halves of one array, which may lie in different orders
    both = torch.cat([m.wg, m.wu], 1)
    m.wg, m.wu = both[:, :F], both[:, F:]
    assert torch.equal(m.run()[0], exp[0])
    m.wu = transposed(m.wu)
    assert torch.equal(m.run()[0], exp[0])


def test_moe_of_nothing():
    m = Moe(4, 32, 0, 6, 2)
    out, ids, weights = m.run()
    assert (out == 0).all()
    m.check_routes(ids, weights)
    for T, D, F, E in ((0, 32, 16, 6), (3, 0, 16, 6), (3, 32, 16, 0), (3, 32, 0, 4)):
        m = Moe(T, D, F, E, 2)
        out, _, _ = m.run(ids=torch.zeros((T, 2), device="cuda", dtype=torch.int32), weights=torch.ones((T, 2), device="cuda"))
        assert (out == 0).all()


def test_moe_infinities_and_nan():
    m = Moe(6, 64, 48, 5, 2)
    exp, _, _ = m.run()
    m.x[2, 5] = float("nan")
    out, ids, weights = m.run()
    assert torch.isnan(out[2]).all() and torch.isnan(weights[2]).all() and ids[2].tolist() == [0, 1]
    keep = [0, 1, 3, 4, 5]
    assert torch.equal(out[keep], exp[keep])  # (a token's neighbours do not notice)


def test_moe_offsets_beyond_32_bits():
    """Experts so far apart that their offsets pass 2^32 bytes."""
    m = Moe(3, 64, 16, 4, 4)
    exp = m.run()[0]
    big = torch.empty(3 * (1 << 31) + 64 * 16, device="cuda", dtype=BF16)
    for name in ("wg", "wu", "wd"):
        t = getattr(m, name)
        far = big.as_strided(t.shape, (1 << 31, t.shape[2], 1))
        far.copy_(t)
        old, _ = t, setattr(m, name, far)
        assert torch.equal(m.run()[0], exp), name
        setattr(m, name, old)


@pytest.mark.parametrize("T", [1, 4, 20])
@pytest.mark.parametrize("D,F", [(64, 64), (63, 65), (33, 127), (40, 66), (129, 191), (70, 1)])
def test_moe_rows_keep_their_neighbours_out(T, D, F):
    """An infinity in one row of the last matrix reaches its channel alone: nothing of a row's neighbours, which lie
    right in front of it and behind it, enters its sums, wherever rows begin."""
    for at in (0, 1, 2):
        m = Moe(T, D, F, 3, 2)
        store = torch.zeros(at + 3 * D * F, device="cuda", dtype=BF16)
        wd = store[at:].view(3, D, F)
        wd.copy_(m.wd)
        m.wd = wd
        exp, ids, weights = m.run()
        m.check_out(exp, ids, weights, "plain")
        for d in (0, D // 2, D - 1):
            for f in (0, F - 1):
                old = wd[:, d, f].clone()
                wd[:, d, f] = float("inf")
                out = m.run()[0]
                others = [c for c in range(D) if c != d]
                assert torch.equal(out[:, others], exp[:, others]) and not torch.isfinite(out[:, d]).any()
                wd[:, d, f] = old
