"""The feed-forward sub-block's operators through the C ABI against plain 64-bit forms.

Tolerances.  u is the type's unit roundoff (bf16 2^-8, fp16 2^-11, fp32 2^-24).  Sums of n products in
fp32 are off by at most (n + 16) 2^-23 of the sum of the products' sizes (truncating additions, a few
operations around them); an operand that was rounded to the type in between adds u of the same sum; the
result's own rounding adds u of its size.  Tiny absolute terms cover the types' underflow.
"""
import math

import pytest
import torch

from paper_1802_06905_b200 import binding, block

pytestmark = pytest.mark.gpu

BF16, FP16, FP32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
U = {BF16: 2.0 ** -8, FP16: 2.0 ** -11, FP32: 2.0 ** -24}
TINY = {BF16: 1e-30, FP16: 2.0 ** -24, FP32: 1e-30}
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def poisoned(shape, dtype):
    return torch.full(shape, float("nan"), dtype=torch.float32, device="cuda").to(dtype)


def act64(name, g):
    """Value and derivative in 64 bits."""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        cdf = torch.special.ndtr(g)
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (g + 0.044715 * g ** 3))
        return g * (1 + t) / 2, (1 + t) / 2 + g / 2 * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)
    return torch.clamp(g, min=0), (g > 0).double()


def close(got, exp, tol, what):
    got = got.double()
    bad = ~((got - exp).abs() <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off; worst {(got - exp).abs().max().item():.3e}, "
                           f"first {bad.nonzero()[0].tolist()}: {got[tuple(bad.nonzero()[0])].item()} for "
                           f"{exp[tuple(bad.nonzero()[0])].item()}")


def sum_err(n):
    return (n + 16) * 2.0 ** -23


class Ffn:
    """Operands of one shape, exact values and tolerances."""

    def __init__(self, T, D, F, dtype=BF16, act="silu", seed=0):
        g = gen(seed + 7 * T + 13 * D + 29 * F)
        self.T, self.D, self.F, self.dtype, self.act = T, D, F, dtype, act
        self.x = normal(g, (T, D), dtype)
        self.wg = normal(g, (F, D), dtype, max(D, 1) ** -0.5)
        self.wu = normal(g, (F, D), dtype, max(D, 1) ** -0.5)
        self.wd = normal(g, (D, F), dtype, max(F, 1) ** -0.5)
        self.dy = normal(g, (T, D), dtype)
        self.g = normal(g, (T, F), dtype)
        self.u = normal(g, (T, F), dtype)

    def forward(self, save, **kw):
        out = poisoned((self.T, self.D), self.dtype)
        gp, up = (poisoned((self.T, self.F), self.dtype) for _ in range(2)) if save else (None, None)
        block.ffn_forward(self.x, self.wg, self.wu, self.wd, out, act=block.ACTS[self.act], gate_pre=gp, up_pre=up, **kw)
        return out, gp, up

    def check_forward(self, out, gp, up, what=""):
        u = U[self.dtype]
        x, wg, wu, wd = (t.double() for t in (self.x, self.wg, self.wu, self.wd))
        g, v = x @ wg.T, x @ wu.T
        ag, av = x.abs() @ wg.abs().T, x.abs() @ wu.abs().T
        eg, ev = sum_err(self.D) * ag, sum_err(self.D) * av
        a, da = act64(self.act, g)
        h = a * v
        # |a'| <= 1.13 for all four; the fast exponential and quotient: 16 units of fp32
        eh = 1.13 * eg * (v.abs() + ev) + (a.abs() + 1e-6) * ev + 2.0 ** -20 * (h.abs() + g.abs() * v.abs()) + u * h.abs() + TINY[self.dtype]
        y = h @ wd.T
        ey = eh @ wd.abs().T + sum_err(self.F) * (h.abs() @ wd.abs().T)
        close(out, y, 1.01 * (ey + u * y.abs()) + TINY[self.dtype], what + " out")
        if gp is not None:
            close(gp, g, 1.01 * (eg + u * g.abs()) + TINY[self.dtype], what + " gate_pre")
            close(up, v, 1.01 * (ev + u * v.abs()) + TINY[self.dtype], what + " up_pre")

    def backward(self, **kw):
        outs = [poisoned(s, self.dtype) for s in ((self.T, self.D), (self.F, self.D), (self.F, self.D), (self.D, self.F))]
        block.ffn_backward(self.dy, self.x, self.wg, self.wu, self.wd, self.g, self.u, *outs, act=block.ACTS[self.act], **kw)
        return outs

    def check_backward(self, dx, dwg, dwu, dwd, what=""):
        u, tiny = U[self.dtype], TINY[self.dtype]
        x, wg, wu, wd, dy, g, v = (t.double() for t in (self.x, self.wg, self.wu, self.wd, self.dy, self.g, self.u))
        a, da = act64(self.act, g)
        dh = dy @ wd
        edh = sum_err(self.D) * (dy.abs() @ wd.abs())
        fast = 2.0 ** -20 * (1 + g.abs())
        dg, du, h = dh * v * da, dh * a, a * v
        edg = edh * (v * da).abs() + fast * (dh * v).abs() + u * dg.abs() + tiny
        edu = edh * a.abs() + fast * dh.abs() * (1 + a.abs()) + u * du.abs() + tiny
        eh = fast * v.abs() * (1 + a.abs()) + u * h.abs() + tiny

        def prod(p, ep, q, n):  # p^T-style products are passed as matrices already in place
            return p @ q, ep @ q.abs() + sum_err(n) * (p.abs() @ q.abs())
        y1, e1 = prod(dg, edg, wg, 2 * self.F)
        y2, e2 = prod(du, edu, wu, 2 * self.F)
        for got, (y, e), name in ((dx, (y1 + y2, e1 + e2), "dx"), (dwg, prod(dg.T, edg.T, x, self.T), "dw_gate"),
                                  (dwu, prod(du.T, edu.T, x, self.T), "dw_up")):
            close(got, y, 1.01 * (e + u * y.abs()) + tiny, f"{what} {name}")
        y = dy.T @ h
        e = dy.abs().T @ eh + sum_err(self.T) * (dy.abs().T @ h.abs())
        close(dwd, y, 1.01 * (e + u * y.abs()) + tiny, what + " dw_down")


SHAPES = [(1, 64, 128), (1, 1, 1), (1, 520, 1032), (2, 2048, 512), (3, 65, 131), (7, 130, 66), (8, 256, 1000), (9, 72, 200),
          (16, 512, 512), (17, 24, 136), (33, 264, 520), (64, 128, 704), (65, 1024, 96), (127, 63, 129), (128, 128, 128),
          (129, 136, 264), (255, 384, 257), (256, 256, 256), (300, 1000, 333), (513, 320, 640), (1030, 192, 448)]


@pytest.mark.parametrize("T,D,F", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_ffn_forward(T, D, F, dtype):
    f = Ffn(T, D, F, dtype, ACTS[(T + D + F) % 4])
    f.check_forward(*f.forward(True), f"{T}x{D}x{F}")
    f.check_forward(*f.forward(False), f"{T}x{D}x{F} no save")
    assert block.status() == (0, 0)


@pytest.mark.parametrize("T,D,F", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_ffn_backward(T, D, F, dtype):
    f = Ffn(T, D, F, dtype, ACTS[(T + D + F + 1) % 4])
    f.check_backward(*f.backward(), f"{T}x{D}x{F}")
    assert block.status() == (0, 0)


@pytest.mark.parametrize("act", ACTS)
def test_ffn_activations(act):
    for T in (2, 40, 300):
        f = Ffn(T, 96, 160, BF16, act)
        f.check_forward(*f.forward(True), act)
        f.check_backward(*f.backward(), act)


def test_ffn_large_pre_activations():
    """Both saturated ends of every activation: finite, and right."""
    for act in ACTS:
        f = Ffn(20, 64, 128, BF16, act)
        f.g = (f.g * 60).contiguous()
        f.check_backward(*f.backward(), act)
        f.x = f.x * 40
        f.check_forward(*f.forward(True), act)


def strided_variants(f):
    """The same values in other storage: (what, function that re-stores one operand)."""
    def transposed(t):
        return t.t().contiguous().t()

    def pitched(t):
        big = torch.full((t.shape[0], t.shape[1] + 8), 9.0, device="cuda").to(t.dtype)
        big[:, :t.shape[1]] = t
        return big[:, :t.shape[1]]

    def shifted(t):  # rows that start 2 bytes off a 16-byte boundary
        big = torch.full((t.shape[0], t.shape[1] + 8), 9.0, device="cuda").to(t.dtype)
        big[:, 1:t.shape[1] + 1] = t
        return big[:, 1:t.shape[1] + 1]

    def every_other(t):
        big = torch.full((t.shape[0], 2 * t.shape[1]), 9.0, device="cuda").to(t.dtype)
        big[:, ::2] = t
        return big[:, ::2]
    return [("transposed", transposed), ("pitched", pitched), ("shifted", shifted), ("every_other", every_other)]


@pytest.mark.parametrize("T", [1, 5, 40, 200])
def test_ffn_strided_operands(T):
    f = Ffn(T, 136, 272, BF16)
    exp_f, exp_b = f.forward(True), f.backward()
    for what, store in strided_variants(f):
        h = Ffn(T, 136, 272, BF16)
        for name in ("x", "wg", "wu", "wd", "dy", "g", "u"):
            setattr(h, name, store(getattr(f, name)))
        h.check_forward(*h.forward(True), what)
        h.check_backward(*h.backward(), what)
        # strided results
        out, gp, up = store(exp_f[0].clone()), store(exp_f[1].clone()), store(exp_f[2].clone())
        for t in (out, gp, up):
            t.fill_(float("nan"))
        block.ffn_forward(f.x, f.wg, f.wu, f.wd, out, gate_pre=gp, up_pre=up)
        f.check_forward(out, gp, up, what + " results")
        outs = [store(t.clone()) for t in exp_b]
        for t in outs:
            t.fill_(float("nan"))
        block.ffn_backward(f.dy, f.x, f.wg, f.wu, f.wd, f.g, f.u, *outs)
        f.check_backward(*outs, what + " results")
    assert block.status() == (0, 0)


def test_ffn_results_leave_their_surroundings():
    """Nothing outside the T x D and T x F elements is written, whatever the pitch."""
    for T in (1, 6, 70, 260):
        f = Ffn(T, 72, 136, BF16)
        bufs = [torch.full((T + 2, n + 24), 5.0, device="cuda", dtype=BF16) for n in (72, 136, 136)]
        views = [b[1:T + 1, 8:8 + n] for b, n in zip(bufs, (72, 136, 136))]
        block.ffn_forward(f.x, f.wg, f.wu, f.wd, views[0], gate_pre=views[1], up_pre=views[2])
        f.check_forward(*views)
        for b, n in zip(bufs, (72, 136, 136)):
            b[1:T + 1, 8:8 + n] = 5.0
            assert (b == 5.0).all()
        sizes = ((T, 72), (136, 72), (136, 72), (72, 136))
        bufs = [torch.full((r + 2, c + 24), 5.0, device="cuda", dtype=BF16) for r, c in sizes]
        views = [b[1:r + 1, 8:8 + c] for b, (r, c) in zip(bufs, sizes)]
        block.ffn_backward(f.dy, f.x, f.wg, f.wu, f.wd, f.g, f.u, *views)
        f.check_backward(*views)
        for b, (r, c) in zip(bufs, sizes):
            b[1:r + 1, 8:8 + c] = 5.0
            assert (b == 5.0).all()


def test_ffn_column_slices_and_broadcast_inputs():
    T, D, F = 50, 64, 96
    f = Ffn(T, D, F)
    both = poisoned((T, 2 * F), BF16)
    out = poisoned((T, D), BF16)
    block.ffn_forward(f.x, f.wg, f.wu, f.wd, out, gate_pre=both[:, :F], up_pre=both[:, F:])
    f.check_forward(out, both[:, :F], both[:, F:])
    # dL/dy of a sum: one element repeated; one row of x for every token
    f.dy = torch.ones((), device="cuda", dtype=BF16).expand(T, D)
    f.x = f.x[:1].expand(T, D)
    f.check_backward(*f.backward())
    f.check_forward(*f.forward(True))


def test_ffn_nan_and_inf_stay_in_their_token():
    for T in (3, 30, 300):
        f = Ffn(T, 72, 136, BF16)
        clean = f.forward(True)
        f.x[1, 3] = float("nan")
        f.x[2, 5] = float("inf")
        out = f.forward(True)
        keep = [t for t in range(T) if t not in (1, 2)]
        for a, b in zip(clean, out):
            assert torch.equal(a[keep], b[keep])
            assert b[1].isnan().all()
            assert not b[2].isfinite().any()


def test_ffn_zero_lengths():
    for T, D, F in ((0, 64, 96), (5, 0, 96), (5, 64, 0)):
        f = Ffn(T, D, F)
        out, gp, up = f.forward(True)
        assert (out == 0).all() and (gp == 0).all() and (up == 0).all()
        for t in f.backward():
            assert (t == 0).all()


def test_ffn_repeats_bit_for_bit_on_any_stream():
    for T in (1, 20, 90, 500):
        f = Ffn(T, 256, 520)
        a, b = f.forward(True), f.backward()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            c = f.forward(True)
        d = f.backward(stream=side)
        torch.cuda.synchronize()
        for p, q in zip(list(a) + list(b), list(c) + list(d)):
            assert torch.equal(p, q)


def test_ffn_in_a_cuda_graph():
    f = Ffn(48, 128, 256)
    out = poisoned((48, 128), BF16)
    f.forward(False)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.ffn_forward(f.x, f.wg, f.wu, f.wd, out)
    for seed in (1, 2):
        f2 = Ffn(48, 128, 256, seed=seed)
        for name in ("x", "wg", "wu", "wd"):
            getattr(f, name).copy_(getattr(f2, name))
        graph.replay()
        f2.check_forward(out, None, None)


def test_ffn_own_workspace_is_enough_and_not_exceeded():
    f = Ffn(77, 200, 312)
    outs = [poisoned(s, BF16) for s in ((77, 200), (312, 200), (312, 200), (200, 312))]
    args = (f.dy, f.x, f.wg, f.wu, f.wd, f.g, f.u, *outs)
    n = block.ffn_backward_workspace(*args)
    ws = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
    block.ffn_backward(*args, workspace=ws[:n])
    f.check_backward(*outs)
    assert (ws[n:] == 77).all()
    if n:
        with pytest.raises(binding.CconvError):
            block.ffn_backward(*args, workspace=ws[:n - 1])


def test_ffn_gradients_against_differences():
    """(L(p + e v) - L(p - e v)) / 2e in 64 bits, L = sum(dy * y), against the gradients times v.  The
    operator works on the given g and u, so L's inner point is the operands' own forward result."""
    f = Ffn(24, 80, 112, FP16, "gelu")
    _, f.g, f.u = f.forward(True)
    grads = f.backward()

    def loss(x, wg, wu, wd):
        return (f.dy.double() * ((act64("gelu", x @ wg.T)[0] * (x @ wu.T)) @ wd.T)).sum()
    ps = [t.double() for t in (f.x, f.wg, f.wu, f.wd)]
    g = gen(5)
    for i, grad in enumerate(grads):
        v = torch.randn(ps[i].shape, generator=g, device="cuda", dtype=torch.float64)
        e = 1e-5
        up, dn = list(ps), list(ps)
        up[i], dn[i] = ps[i] + e * v, ps[i] - e * v
        diff = ((loss(*up) - loss(*dn)) / (2 * e)).item()
        got = (grad.double() * v).sum().item()
        # roundings of g, u, h, dg, du and the gradient itself, each at most u = 2^-11 of a factor: their
        # sum over the elements is bounded by 8 u sum |grad v| plus what cancels inside the products
        bound = 8 * U[FP16] * (grad.double().abs() * v.abs()).sum().item() * 4
        assert abs(got - diff) <= bound, (i, got, diff, bound)


def test_ffn_refusals():
    f = Ffn(4, 16, 24)
    out = poisoned((4, 16), BF16)
    ok = dict(x=f.x, w_gate=f.wg, w_up=f.wu, w_down=f.wd, out=out)
    for name, bad in (("x", f.x.float()), ("x", f.x.cpu()), ("x", f.x[0]), ("w_gate", f.wg.half()), ("w_up", f.wu[:-1]),
                      ("w_down", f.wd.t()), ("out", out[:, :-1]), ("out", out.float())):
        with pytest.raises(ValueError):
            block.ffn_forward(**{**ok, name: bad})
    with pytest.raises(ValueError):
        block.ffn_forward(**ok, gate_pre=f.g)
    for bad in (dict(out=f.x), dict(out=out[:1].expand(4, 16)), dict(act=7), dict(gate_pre=f.g, up_pre=f.g)):
        with pytest.raises(binding.CconvError) as e:
            block.ffn_forward(**{**ok, **bad})
        assert e.value.code == binding.EINVAL
    assert out.isnan().all()


# ---- residual norm ---------------------------------------------------------------------------------

class Norm:
    def __init__(self, T, D, dtype=BF16, gate="none", rows=0, post=True, pre=True, blk=True, scale=1.0, eps=1e-6, seed=0):
        g = gen(seed + 3 * T + 11 * D)
        self.T, self.D, self.dtype, self.rows, self.scale, self.eps = T, D, dtype, rows, scale, eps
        self.r = normal(g, (T, D), dtype, 3.0)
        self.y = normal(g, (T, D), dtype, 0.6) if blk else None
        self.wpost = (1 + normal(g, (D,), FP32, 0.2)).to(dtype) if post and blk else None
        self.wpre = (1 + normal(g, (D,), FP32, 0.2)).to(dtype) if pre else None
        groups = -(-T // rows) if rows else 1
        self.gate = normal(g, (groups, D), dtype, 0.5) if gate and gate != "none" and blk else None
        self.dr, self.dx = normal(g, (T, D), dtype), normal(g, (T, D), dtype)

    def gate_rows64(self):
        if self.gate is None:
            return 1.0
        at = torch.arange(self.T, device="cuda") // (self.rows or max(self.T, 1))
        return self.gate.double()[at]

    def forward64(self, r, y, wpost, gate, wpre):
        n = 0.0
        if y is not None:
            n = y
            if wpost is not None:
                n = y * torch.rsqrt((y * y).mean(1, keepdim=True) + self.eps) * wpost
            if gate is not None:
                at = torch.arange(self.T, device="cuda") // (self.rows or max(self.T, 1))
                n = gate[at] * n
        o = self.scale * r + n
        x = o * torch.rsqrt((o * o).mean(1, keepdim=True) + self.eps)
        return o, x if wpre is None else x * wpre

    def run(self, norm=True, out=None, xout=None):
        out = poisoned((self.T, self.D), self.dtype) if out is None else out
        xout = poisoned((self.T, self.D), self.dtype) if norm and xout is None else xout
        block.residual_norm_forward(self.r, out, xout, block=self.y, w_post=self.wpost, gate=self.gate,
                                    w_pre=self.wpre if norm else None, rows_per_gate=self.rows, scale=self.scale, eps=self.eps)
        return out, xout

    def check(self, out, xout, what=""):
        d = lambda t: None if t is None else t.double()  # noqa: E731
        u, tiny = U[self.dtype], TINY[self.dtype]
        o, x = self.forward64(d(self.r), d(self.y), d(self.wpost), d(self.gate), d(self.wpre))
        # a term of r' passes through at most 8 fp32 operations, the mean of squares adds (D + 16) 2^-24
        # of itself (all terms positive), which rsqrt halves
        e = (self.D + 64) * 2.0 ** -24
        size = (self.scale * self.r.double()).abs() + (o - self.scale * self.r.double()).abs()
        close(out, o, u * o.abs() + 1.01 * e * size + tiny, what + " resid_out")
        if xout is not None:
            rho = torch.rsqrt((o * o).mean(1, keepdim=True) + self.eps)
            w = 1.0 if self.wpre is None else self.wpre.double().abs()
            spread = (size * size).mean(1, keepdim=True).sqrt() * rho  # error of the norm itself
            close(xout, x, u * x.abs() + 1.01 * e * (size * rho * w + x.abs() * (1 + 2 * spread)) + tiny, what + " norm_out")

    def run_backward(self, use_dr=True, use_dx=True, **kw):
        self.o = self.forward64(self.r.double(), *(None if t is None else t.double() for t in (self.y, self.wpost, self.gate, self.wpre)))[0].to(self.dtype)
        new = lambda t: None if t is None else poisoned(t.shape, self.dtype)  # noqa: E731
        dres, dblk, dwpost, dgate = poisoned((self.T, self.D), self.dtype), new(self.y), new(self.wpost), new(self.gate)
        dwpre = new(self.wpre) if use_dx else None
        block.residual_norm_backward(self.dr if use_dr else None, self.dx if use_dx else None, self.o, dres, block=self.y, dblock=dblk,
                                     w_post=self.wpost, dw_post=dwpost, gate=self.gate, dgate=dgate,
                                     w_pre=self.wpre if use_dx else None, dw_pre=dwpre, rows_per_gate=self.rows,
                                     scale=self.scale, eps=self.eps, **kw)
        return dres, dblk, dwpost, dgate, dwpre

    def check_backward(self, got, use_dr=True, use_dx=True, what=""):
        u, tiny, T, D = U[self.dtype], TINY[self.dtype], self.T, self.D
        dres, dblk, dwpost, dgate, dwpre = got
        e = (D + 64) * 2.0 ** -23
        S, aS = 0.0, 0.0
        if use_dr:
            S, aS = S + self.dr.double(), aS + self.dr.double().abs()
        if use_dx:
            o, dx = self.o.double(), self.dx.double()
            w = 1.0 if self.wpre is None else self.wpre.double()
            rho = torch.rsqrt((o * o).mean(1, keepdim=True) + self.eps)
            ee, rhat = dx * w, o * rho
            S = S + rho * (ee - rhat * (ee * rhat).mean(1, keepdim=True))
            aS = aS + rho * (ee.abs() + rhat.abs() * (ee * rhat).abs().mean(1, keepdim=True))
            if dwpre is not None:
                y, a = (dx * rhat).sum(0), (dx * rhat).abs().sum(0)
                close(dwpre, y, u * y.abs() + (e + (T + 16) * 2.0 ** -24) * a + tiny, what + " dw_pre")
        close(dres, self.scale * S, u * (self.scale * S).abs() + e * abs(self.scale) * aS + tiny, what + " dresid")
        if self.y is None:
            return
        y = self.y.double()
        wp = 1.0 if self.wpost is None else self.wpost.double()
        rho = torch.rsqrt((y * y).mean(1, keepdim=True) + self.eps) if self.wpost is not None else 1.0
        yhat, gt = y * rho, self.gate_rows64()
        dn, adn = gt * S, abs(gt) * aS
        sums = e + (T + 16) * 2.0 ** -24
        if self.gate is not None:
            per = self.rows or T
            groups = self.gate.shape[0]
            at = torch.arange(T, device="cuda") // per
            z = lambda: torch.zeros((groups, D), dtype=torch.float64, device="cuda")  # noqa: E731
            ex, ab = z().index_add_(0, at, S * yhat * wp), z().index_add_(0, at, aS * (yhat * wp).abs())
            close(dgate, ex, u * ex.abs() + sums * ab + tiny, what + " dgate")
        f, af = dn * wp, adn * abs(wp)
        if self.wpost is not None:
            ex, ab = (dn * yhat).sum(0), (adn * yhat.abs()).sum(0)
            close(dwpost, ex, u * ex.abs() + sums * ab + tiny, what + " dw_post")
            ab = rho * (af + yhat.abs() * (af * yhat.abs()).mean(1, keepdim=True))
            f = rho * (f - yhat * (f * yhat).mean(1, keepdim=True))
        else:
            ab = af
        close(dblk, f, u * f.abs() + e * ab + tiny, what + " dblock")


NORM_SHAPES = [(1, 64), (1, 4096), (1, 1), (2, 7), (3, 1000), (5, 1001), (33, 256), (64, 2048), (130, 520), (700, 96),
               (300, 4096), (9, 8192), (5, 8200), (3, 16384), (2, 16392), (3, 20001), (4, 9001), (1500, 64)]


@pytest.mark.parametrize("T,D", NORM_SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_residual_norm(T, D, dtype):
    for gate, rows in (("none", 0), ("all", 0), ("tokens", 1), ("groups", max(1, T // 3))):
        n = Norm(T, D, dtype, gate, rows, scale=0.75 if D % 2 else 1.0)
        n.check(*n.run(), f"{gate}")
        n.check_backward(n.run_backward(), what=gate)


def test_residual_norm_parts_that_are_absent():
    for T, D in ((5, 200), (3, 301), (2, 17000)):
        for kw in (dict(post=False), dict(pre=False), dict(post=False, gate="all"), dict(blk=False), dict(blk=False, pre=False)):
            n = Norm(T, D, BF16, **kw)
            n.check(*n.run(), str(kw))
            n.check(*n.run(norm=False), str(kw))
            for use_dr, use_dx in ((True, True), (True, False), (False, True)):
                n.check_backward(n.run_backward(use_dr, use_dx), use_dr, use_dx, f"{kw} {use_dr} {use_dx}")


@pytest.mark.parametrize("T,rows", [(1000, 1), (1000, 2), (1000, 7), (1000, 333), (1000, 999), (1000, 1000), (1000, 5000), (148, 3),
                                    (2368, 16), (5000, 8), (5000, 100)])
def test_residual_norm_gate_groups(T, rows):
    """Groups inside one block's rows, across two and across many; more groups than blocks and fewer."""
    for D in (64, 72, 1024):
        n = Norm(T, D, BF16, "groups", rows)
        n.check(*n.run())
        n.check_backward(n.run_backward(), what=f"D={D}")


def test_residual_norm_in_place_and_strided():
    for D in (256, 251):
        n = Norm(40, D, BF16, "all")
        out, x = n.run()
        r = n.r
        n.r = r.clone()
        got = n.run(out=n.r)
        assert torch.equal(got[0], out) and torch.equal(got[1], x)
        n.r = r
        for pad, off in ((8, 0), (8, 8), (3, 1)):
            def store(t, rows=0):
                big = torch.full((t.shape[0], t.shape[1] + pad + off), 5.0, device="cuda").to(BF16)
                v = big[:, off:off + t.shape[1]]
                v.copy_(t)
                return big, v
            m = Norm(40, D, BF16, "all")
            for name in ("r", "y", "dr", "dx"):
                setattr(m, name, store(getattr(m, name))[1])
            big, v = store(out)
            big2, v2 = store(x)
            m.run(out=v, xout=v2)
            assert torch.equal(v, out) and torch.equal(v2, x)
            for b in (big, big2):
                b[:, off:off + D] = 5.0
                assert (b == 5.0).all()
            m.check_backward(m.run_backward())
        # dresid in the place of dresid_out; one row of resid and block for every token
        exp = n.run_backward()
        dr = n.dr.clone()
        new = [None if t is None else torch.empty_like(t) for t in exp]
        block.residual_norm_backward(dr, n.dx, n.o, dr, block=n.y, dblock=new[1], w_post=n.wpost, dw_post=new[2], gate=n.gate,
                                     dgate=new[3], w_pre=n.wpre, dw_pre=new[4], scale=n.scale, eps=n.eps)
        for a, b in zip((dr, *new[1:]), exp):
            assert torch.equal(a, b)
        n.r, n.y = n.r[:1].expand(40, D), n.y[:1].expand(40, D)
        n.check(*n.run())


def test_residual_norm_zero_rows_and_special_values():
    n = Norm(4, 128, BF16, "all")
    n.r[1] = 0
    n.y[1] = 0
    n.y[2, 5] = float("nan")
    out, x = n.run()
    assert (out[1] == 0).all() and (x[1] == 0).all()
    assert out[2].isnan().all() and x[2].isnan().all()
    assert out[[0, 3]].isfinite().all() and x[[0, 3]].isfinite().all()
    e = Norm(0, 128, BF16, "all")
    e.run()
    _, _, dwpost, dgate, dwpre = e.run_backward()
    assert (dwpost == 0).all() and (dgate == 0).all() and (dwpre == 0).all()


def test_residual_norm_gradients_against_differences():
    n = Norm(12, 48, FP32, "groups", 5, scale=0.9)
    got = dict(zip(("r", "y", "wpost", "gate", "wpre"), n.run_backward()))
    ps = dict(r=n.r.double(), y=n.y.double(), wpost=n.wpost.double(), gate=n.gate.double(), wpre=n.wpre.double())

    def loss(p):
        o, x = n.forward64(p["r"], p["y"], p["wpost"], p["gate"], p["wpre"])
        return (n.dr.double() * o).sum() + (n.dx.double() * x).sum()
    g = gen(3)
    for name, grad in got.items():
        v = torch.randn(ps[name].shape, generator=g, device="cuda", dtype=torch.float64)
        e = 1e-6
        diff = ((loss({**ps, name: ps[name] + e * v}) - loss({**ps, name: ps[name] - e * v})) / (2 * e)).item()
        # fp32 gradients and r' rounded to fp32: 2^-18 of the sizes covers them; the differences: 1e-8 of the loss / e
        bound = 2.0 ** -18 * (grad.double().abs() * v.abs()).sum().item() * 8 + 1e-5
        assert abs((grad.double() * v).sum().item() - diff) <= bound, name


def test_residual_norm_refusals():
    n = Norm(4, 64, BF16, "all")
    out, x = poisoned((4, 64), BF16), poisoned((4, 64), BF16)
    ok = dict(resid=n.r, resid_out=out, norm_out=x, block=n.y, w_post=n.wpost, gate=n.gate, w_pre=n.wpre)
    for bad in (dict(resid=n.r.to(torch.float64)), dict(block=n.y[:3]), dict(w_post=n.wpost.float()), dict(gate=n.gate[0]),
                dict(rows_per_gate=2), dict(resid_out=out.t().contiguous().t()), dict(w_pre=n.wpre[:-1])):
        with pytest.raises(ValueError):
            block.residual_norm_forward(**{**ok, **bad})
    for bad in (dict(eps=0.0), dict(eps=float("nan")), dict(norm_out=out), dict(norm_out=n.y), dict(scale=float("inf")),
                dict(block=None), dict(norm_out=None), dict(rows_per_gate=-1), dict(resid_out=n.y)):
        with pytest.raises((binding.CconvError, ValueError)):
            block.residual_norm_forward(**{**ok, **bad})
    assert out.isnan().all() and x.isnan().all()
    with pytest.raises(binding.CconvError):   # dblock is missing
        block.residual_norm_backward(n.dr, n.dx, n.r, out, block=n.y, w_pre=n.wpre, dw_pre=poisoned((64,), BF16))


# ---- 8-bit product and quantisation ----------------------------------------------------------------

def fp8_operands(M, N, K, seed=0):
    g = gen(seed + M + 5 * N + 17 * K)
    kb, nb = -(-K // 128), -(-N // 128)
    a = normal(g, (M, K), FP32, 120).clamp(-448, 448).to(E4M3)
    b = normal(g, (N, K), FP32, 120).clamp(-448, 448).to(E4M3)
    sa = torch.exp(normal(g, (M, kb), FP32, 0.5)) / 120
    sb = torch.exp(normal(g, (nb, kb), FP32, 0.5)) / (120 * max(K, 1) ** 0.5)
    return a, sa, b, sb


def fp8_check(a, sa, b, sb, out, what=""):
    (M, K), N = a.shape, b.shape[0]
    ks, ns = torch.arange(K, device="cuda") // 128, torch.arange(N, device="cuda") // 128
    fa, fb = a.double() * sa.double()[:, ks], b.double() * sb.double()[ns][:, ks]
    y, ab = fa @ fb.T, fa.abs() @ fb.abs().T
    close(out, y, U[out.dtype] * y.abs() + sum_err(K) * ab + TINY[out.dtype], what)


FP8_SHAPES = [(1, 128, 128), (1, 1, 1), (2, 8192, 256), (1, 64, 4096), (3, 130, 129), (4, 200, 1000), (7, 1000, 512), (8, 24, 2000),
              (9, 512, 640), (16, 300, 384), (17, 129, 272), (33, 640, 200), (64, 256, 1024), (100, 1000, 127), (128, 128, 128),
              (129, 257, 144), (250, 384, 1536), (256, 256, 512), (300, 777, 1111), (1025, 640, 640)]


@pytest.mark.parametrize("M,N,K", FP8_SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_fp8_product(M, N, K, dtype):
    a, sa, b, sb = fp8_operands(M, N, K)
    out = poisoned((M, N), dtype)
    block.fp8_product(a, sa, b, sb, out)
    fp8_check(a, sa, b, sb, out, f"{M}x{N}x{K}")
    assert block.status() == (0, 0)


@pytest.mark.parametrize("M", [1, 6, 40, 200])
def test_fp8_strided_operands(M):
    N, K = 200, 400
    a, sa, b, sb = fp8_operands(M, N, K)

    def as_bytes(f, t):
        return f(t.view(torch.uint8)).view(E4M3)
    for what, f in (("transposed", lambda t: t.t().contiguous().t()),
                    ("shifted", lambda t: torch.cat([t[:, :1], t, t[:, :4]], 1)[:, 1:t.shape[1] + 1]),
                    ("every_other", lambda t: t.repeat_interleave(2, 1)[:, ::2])):
        out = torch.full((M, N + 3), 5.0, device="cuda", dtype=BF16)
        block.fp8_product(as_bytes(f, a), f(sa), as_bytes(f, b), f(sb), out[:, 1:N + 1])
        fp8_check(a, sa, b, sb, out[:, 1:N + 1], what)
        assert (out[:, 0] == 5).all() and (out[:, N + 1:] == 5).all()
        out = poisoned((N, M), FP32).t()
        block.fp8_product(as_bytes(f, a), f(sa), as_bytes(f, b), f(sb), out)
        fp8_check(a, sa, b, sb, out, what + " transposed result")
    sa1 = sa[:, :1].expand(M, 4)   # one scale for each token
    out = poisoned((M, N), BF16)
    block.fp8_product(a, sa1, b, sb, out)
    fp8_check(a, sa1, b, sb, out, "broadcast scale")


def test_fp8_special_values():
    for M in (2, 20, 200):
        a, sa, b, sb = fp8_operands(M, 256, 300)
        out, clean = poisoned((M, 256), FP32), poisoned((M, 256), FP32)
        block.fp8_product(a, sa, b, sb, clean)
        bits = a.view(torch.uint8)
        bits[1, 290] = 0x7F          # NaN
        block.fp8_product(a, sa, b, sb, out)
        assert out[1].isnan().all()
        keep = [m for m in range(M) if m != 1]
        assert torch.equal(out[keep], clean[keep])
        bits[1, 290] = 0
        sa[0, 1] = float("inf")
        sb[1, 2] = float("nan")
        block.fp8_product(a, sa, b, sb, out)
        assert out[:, 128:].isnan().all() and not out[0].isfinite().any()
        keep = [m for m in range(M) if m not in (0, 1)]
        assert torch.equal(out[keep, :128], clean[keep, :128])


def test_fp8_zero_lengths():
    for M, N, K in ((0, 5, 6), (5, 0, 6), (5, 6, 0)):
        a, sa, b, sb = fp8_operands(M, N, K)
        out = poisoned((M, N), BF16)
        block.fp8_product(a, sa, b, sb, out)
        assert (out == 0).all()


def test_fp8_refusals():
    a, sa, b, sb = fp8_operands(4, 16, 200)
    out = poisoned((4, 16), BF16)
    for bad in (dict(a=a.float()), dict(a=a[:, :-1]), dict(a_scale=sa[:, :1]), dict(b_scale=sb.double()), dict(b=b[:3]),
                dict(out=out.double()), dict(out=out[0])):
        with pytest.raises((ValueError, IndexError)):
            block.fp8_product(**{**dict(a=a, a_scale=sa, b=b, b_scale=sb, out=out), **bad})
    with pytest.raises(binding.CconvError):
        block.fp8_product(a, sa, b, sb, out[:1].expand(4, 16))


@pytest.mark.parametrize("T,D", [(1, 1), (1, 128), (3, 130), (16, 4096), (17, 1000), (128, 128), (129, 255), (300, 777), (513, 1024)])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_quantize(T, D, dtype):
    for rows in (1, 128):
        x = normal(gen(T + D), (T, D), dtype, 3.0)
        x[0, 0] = 0
        x[-1] = 0                                     # a token of zeros
        for store in (lambda t: t, lambda t: t.t().contiguous().t(), lambda t: torch.cat([t[:, :1], t], 1)[:, 1:]):
            rb, cb = -(-T // rows), -(-D // 128)
            q, s = torch.full((T, D + 8), 0.5, device="cuda").to(E4M3), poisoned((rb, cb), FP32)
            block.quantize_blocks(store(x), q[:, :D], s, block_rows=rows)
            pad = torch.nn.functional.pad(x.float(), (0, cb * 128 - D, 0, rb * rows - T)).reshape(rb, rows, cb, 128)
            amax = pad.abs().amax((1, 3), keepdim=True)
            scale = amax / torch.full_like(amax, 448.0)
            exp = (pad / torch.where(scale == 0, torch.ones_like(scale), scale)).reshape(rb * rows, cb * 128)[:T, :D]
            assert torch.equal(s, scale.reshape(rb, cb))
            assert torch.equal(q[:, :D].float(), exp.contiguous().to(E4M3).float())
            assert (q[:, D:].float() == 0.5).all()


def test_quantize_special_values():
    x = normal(gen(1), (4, 256), BF16)
    x[1, 3] = float("nan")
    x[2, 200] = float("inf")
    q, s = torch.empty((4, 256), device="cuda", dtype=E4M3), poisoned((4, 2), FP32)
    block.quantize_blocks(x, q, s)
    assert s[1, 0].isnan() and q[1, :128].float().isnan().all() and s[1, 1].isfinite()
    assert s[2, 1].isinf() and q[2, 200].float().isnan() and (q[2, 128:200].float() == 0).all()
    assert s[[0, 3]].isfinite().all() and q[[0, 3]].float().isfinite().all()
    e = x[:0]
    block.quantize_blocks(e, q[:0], s[:0])
    tiny = torch.full((1, 128), 1e-38, device="cuda", dtype=BF16)
    block.quantize_blocks(tiny, q[:1, :128], s[:1, :1])
    assert (q[:1, :128].float() == 448).all()


def test_quantize_refusals():
    x = normal(gen(1), (4, 256), BF16)
    q, s = torch.empty((4, 256), device="cuda", dtype=E4M3), poisoned((4, 2), FP32)
    for bad in (dict(x=x.double()), dict(q=q[:, :-1]), dict(scale=s[:1]), dict(block_rows=64), dict(q=x), dict(x=x[0])):
        with pytest.raises((ValueError, IndexError)):
            block.quantize_blocks(**{**dict(x=x, q=q, scale=s), **bad})


def test_quantised_operands_give_the_product():
    """quantize_blocks and fp8_product together against the unquantised product: each factor is off by at
    most 2^-4 of itself (3 mantissa bits) or 2^-10 of its block's scale (below the smallest normal)."""
    g = gen(9)
    x, w = normal(g, (200, 640), BF16), normal(g, (384, 640), BF16, 640 ** -0.5)
    qx, sx = torch.empty((200, 640), device="cuda", dtype=E4M3), poisoned((200, 5), FP32)
    qw, sw = torch.empty((384, 640), device="cuda", dtype=E4M3), poisoned((3, 5), FP32)
    out = poisoned((200, 384), FP32)
    block.quantize_blocks(x, qx, sx)
    block.quantize_blocks(w, qw, sw, block_rows=128)
    block.fp8_product(qx, sx, qw, sw, out)
    fp8_check(qx, sx, qw, sw, out)
    ex, ew = (2.0 ** -4 * t.double().abs() for t in (x, w))
    ex += 2.0 ** -10 * sx.double().repeat_interleave(128, 1)
    ew += 2.0 ** -10 * sw.double().repeat_interleave(128, 0).repeat_interleave(128, 1)
    X, W = x.double(), w.double()
    tol = ex @ W.abs().T + X.abs() @ ew.T + ex @ ew.T + sum_err(640) * (X.abs() @ W.abs().T) * 1.2
    close(out, X @ W.T, tol, "quantised product")
