"""The operators that serve the feed-forward sub-block against plain 64-bit forms: norms with 8-bit results.

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
