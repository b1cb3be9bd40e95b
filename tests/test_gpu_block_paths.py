"""The feed-forward sub-block where its pieces meet: every cut of a product, offsets past 32 bits, the order of
a stream that convolutions share, other devices' streams, and the command that runs all of it together."""
import ctypes
import random

import pytest
import torch

from paper_1802_06905_b200 import binding, block
from test_block_host import struct_of
from test_gpu_block import BF16, E4M3, FP16, FP32, Ffn, Norm, act64, close, fp8_check, fp8_operands, gen, normal, poisoned

pytestmark = pytest.mark.gpu


# T, D, F that take: cuts of a tile over 2 and 4 pairs (few tiles, long k), 64-column tiles, several rounds of
# tiles, the gradients together and apart, tokens of one CTA only and of two
@pytest.mark.parametrize("T,D,F", [(16, 2048, 4096), (48, 512, 8192), (100, 4096, 256), (130, 264, 8200), (200, 128, 6000),
                                   (260, 8192, 128), (700, 1000, 2600), (1500, 72, 4000), (2000, 2048, 136), (4100, 512, 520),
                                   (4096, 64, 64)])
def test_ffn_cuts(T, D, F):
    f = Ffn(T, D, F, BF16 if T % 3 else FP16, "silu")
    f.check_forward(*f.forward(True), "forward")
    f.check_backward(*f.backward(), "backward")
    assert block.status() == (0, 0)


@pytest.mark.parametrize("M,N,K", [(12, 128, 16384), (50, 300, 8192), (150, 1000, 4096), (300, 128, 10000), (600, 4096, 256),
                                   (2000, 2100, 520), (1100, 136, 130), (20, 8192, 144)])
def test_fp8_cuts(M, N, K):
    a, sa, b, sb = fp8_operands(M, N, K)
    for dtype in (BF16, FP32):
        out = poisoned((M, N), dtype)
        block.fp8_product(a, sa, b, sb, out)
        fp8_check(a, sa, b, sb, out)
    assert block.status() == (0, 0)


@pytest.mark.parametrize("T", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype,most", [(BF16, 0.0020), (FP16, 0.00025)])
def test_few_tokens_round_the_result_alone(T, dtype, most):
    """One rounding of normal values to 8 bits is 0.00166 of their norm (11 bits: 0.00021), two in a row 0.0024."""
    for act in block.ACTS:
        f = Ffn(T, 1024, 512, dtype, act)
        out, _, _ = f.forward(False)
        x, wg, wu, wd = (t.double() for t in (f.x, f.wg, f.wu, f.wd))
        want = (act64(act, x @ wg.T)[0] * (x @ wu.T)) @ wd.T
        assert (out.double() - want).norm() <= most * want.norm()


@pytest.mark.parametrize("T", [5, 8, 9, 11, 15, 16, 17])
@pytest.mark.parametrize("D,F", [(512, 1408), (2400, 520), (72, 2400), (8, 16)])
def test_few_tokens_either_side_of_their_limits(T, D, F):
    for dtype, save in ((BF16, True), (FP16, False)):
        f = Ffn(T, D, F, dtype, "gelu_tanh")
        f.check_forward(*f.forward(save), "forward")
        wide = Ffn(T, D, F, dtype, "gelu_tanh")
        for n in ("x", "wg", "wu", "wd"):
            v = getattr(f, n)
            setattr(wide, n, shifted(v, v.shape[1] + 16, 8))
        wide.check_forward(*wide.forward(save), "rows with a pitch")


@pytest.mark.parametrize("M", [5, 8, 9, 13, 16, 17])
@pytest.mark.parametrize("N,K", [(1408, 512), (4800, 144), (24, 4096), (130, 16)])
def test_few_tokens_in_8_bits_either_side_of_their_limits(M, N, K):
    a, sa, b, sb = fp8_operands(M, N, K)
    for dtype in (BF16, FP16, FP32):
        out = poisoned((M, N), dtype)
        block.fp8_product(a, sa, b, sb, out)
        fp8_check(a, sa, b, sb, out)
    assert block.status() == (0, 0)


def test_few_tokens_whose_hidden_values_overflow():
    f = Ffn(2, 128, 256, FP16)
    f.x[1] *= 3000.0  # h passes 65504 for this token only
    out = f.forward(False)[0]
    alone = Ffn(2, 128, 256, FP16).forward(False)[0]
    assert torch.equal(out[0], alone[0]) and not torch.isfinite(out[1]).all()


def far_rows(t, pitch):
    """The same values in rows `pitch` elements apart, so that offsets pass 2^31 elements."""
    buf = torch.empty(pitch * (t.shape[0] - 1) + t.shape[1], dtype=t.dtype, device="cuda")
    v = buf.as_strided(t.shape, (pitch, 1))
    v.copy_(t)
    return v


def test_offsets_past_32_bits():
    pitch = (1 << 30) + 64
    f = Ffn(4, 256, 384)
    f.x = far_rows(f.x, pitch)
    f.check_forward(*f.forward(True))
    f.check_backward(*f.backward())
    del f
    torch.cuda.empty_cache()
    n = Norm(4, 256, BF16, "all")
    n.r, n.y = far_rows(n.r, pitch), n.y
    n.check(*n.run())
    out = far_rows(torch.zeros(4, 256, device="cuda", dtype=BF16), pitch)
    n.check(*n.run(out=out))
    del n, out
    torch.cuda.empty_cache()
    x = far_rows(normal(gen(1), (4, 256), BF16), pitch)
    q, s = torch.empty((4, 256), device="cuda", dtype=E4M3), poisoned((4, 2), FP32)
    block.quantize_blocks(x, q, s)
    q2, s2 = torch.empty_like(q), poisoned((4, 2), FP32)
    block.quantize_blocks(x.contiguous(), q2, s2)
    assert torch.equal(q.float(), q2.float()) and torch.equal(s, s2)


def conv_chain(T, steps, sync):
    """A convolution whose Image a residual norm writes and whose Out a quantisation and the next norm read,
    over and over in the same buffers; with a synchronisation after each call, or none."""
    B, C, K = 64, 64, 128
    g = gen(4)
    rows = normal(g, (9 * C, B), BF16)            # the Image [3][3][C][B] as rows of B
    w = normal(g, (B,), BF16)
    filt = normal(g, (K, 3, 3, C), BF16, (9 * C) ** -0.5)
    image = torch.empty((9 * C, B), dtype=BF16, device="cuda")
    out = torch.empty((K, 1, 1, B), dtype=BF16, device="cuda")
    q, s = torch.empty((K, B), dtype=E4M3, device="cuda"), torch.empty((K, 1), device="cuda")
    got = []

    def done():
        if sync:
            torch.cuda.synchronize()
    for i in range(steps):
        block.residual_norm_forward(rows, rows, image, w_pre=w, scale=0.9)
        done()
        binding.conv_forward(image.view(3, 3, C, B), filt, out, B, C, K, 1, 1, 3, 3)
        done()
        block.quantize_blocks(out.view(K, B), q, s)
        done()
        block.residual_norm_forward(out.view(K, B), rows[:K], w_pre=None, scale=1.25)
        done()
        if i % 8 == 7:
            got.append((image.clone(), out.clone(), q.float(), s.clone(), rows.clone()))
            done()
    torch.cuda.synchronize()
    return got


def test_stream_order_with_convolutions():
    want = conv_chain(0, 40, True)
    for _ in range(5):
        for a, b in zip(want, conv_chain(0, 40, False)):
            for x, y in zip(a, b):
                assert torch.equal(x, y)


def test_a_call_between_two_convolutions_keeps_them_in_order():
    """A convolution reads what one two calls in front wrote; the call between them touches neither array."""
    B, C, K, H = 64, 64, 128, 14
    g = gen(11)
    image = normal(g, (H + 2, H + 2, C, B), BF16)
    f1, f2 = normal(g, (C, 3, 3, C), BF16, (9 * C) ** -0.5), normal(g, (K, 1, 1, C), BF16, C ** -0.5)
    x, q, s = normal(g, (1, 128), BF16), torch.empty((1, 128), dtype=E4M3, device="cuda"), torch.empty((1, 1), device="cuda")
    w, h = normal(g, (128,), BF16), torch.empty((1, 128), dtype=BF16, device="cuda")
    ffn = Ffn(4, 128, 256)
    between = (lambda: block.quantize_blocks(x, q, s), lambda: block.residual_norm_forward(x, x.clone(), h, w_pre=w),
               lambda: ffn.forward(False))
    middles = [torch.empty((C, H, H, B), dtype=BF16, device="cuda") for _ in range(12)]

    def chain(sync):
        outs = []
        for i, mid in enumerate(middles):
            mid.zero_()
        torch.cuda.synchronize()
        for i, mid in enumerate(middles):
            out = torch.zeros((K, H, H, B), dtype=BF16, device="cuda")
            for call in (lambda: binding.conv_forward(image, f1, mid, B, C, C, H, H, 3, 3), between[i % 3],
                         lambda: binding.conv_forward(mid.view(H, H, C, B), f2, out, B, C, K, H, H, 1, 1)):
                call()
                if sync:
                    torch.cuda.synchronize()
            outs.append(out)
        torch.cuda.synchronize()
        return outs
    want = chain(True)
    for _ in range(3):
        for a, b in zip(want, chain(False)):
            assert torch.equal(a, b)


def test_a_chain_of_calls_without_waiting_equals_one_with():
    """Quantise, product, norm, feed-forward in shared buffers: every call reads what the one in front wrote."""
    g = gen(8)
    T, D, F = 24, 256, 512
    w8, s8 = torch.empty((D, D), device="cuda", dtype=E4M3), poisoned((2, 2), FP32)
    wq = normal(g, (D, D), BF16, D ** -0.5)
    wg, wu, wd = normal(g, (F, D), BF16, D ** -0.5), normal(g, (F, D), BF16, D ** -0.5), normal(g, (D, F), BF16, F ** -0.5)
    w = normal(g, (D,), BF16)

    def chain(tokens, sync):
        x = normal(gen(9), (tokens, D), BF16)
        res, q, s = x.clone(), torch.empty((tokens, D), device="cuda", dtype=E4M3), poisoned((tokens, 2), FP32)
        y = torch.empty_like(x)
        for _ in range(25):
            for call in (lambda: block.quantize_blocks(wq, w8, s8, block_rows=128), lambda: block.quantize_blocks(x, q, s),
                         lambda: block.fp8_product(q, s, w8, s8, y), lambda: block.ffn_forward(y, wg, wu, wd, x),
                         lambda: block.residual_norm_forward(res, res, y, block=x, w_post=w, w_pre=w, scale=0.5),
                         lambda: block.ffn_forward(y, wg, wu, wd, x)):
                call()
                if sync:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        return x, y, res, q.float(), s
    for tokens in (1, 5, T, 300):
        want = chain(tokens, True)
        for _ in range(3):
            for a, b in zip(want, chain(tokens, False)):
                assert torch.equal(a, b)


def test_two_streams_at_once():
    f, h = Ffn(300, 512, 1408), Ffn(40, 1024, 2048, seed=3)
    want = f.forward(True) + h.forward(True)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):
        with torch.cuda.stream(a):
            p = f.forward(True)
        with torch.cuda.stream(b):
            q = h.forward(True)
        torch.cuda.synchronize()
        for x, y in zip(want, p + q):
            assert torch.equal(x, y)
    assert block.status() == (0, 0)


def test_the_command_runs_a_block():
    from paper_1802_06905_b200 import ffn_block
    r = ffn_block.run(tokens=96, channels=256, hidden=512, steps=6, serve=3)
    assert r["loss"][-1] < 0.9 * r["loss"][0]
    assert r["serve_error"] < 0.1                   # 8-bit operands: 2^-4 of a factor at worst, less on average


@pytest.mark.parametrize("cut", ["256,1", "256,2", "256,4", "128,1", "128,2", "128,4", "64,1", "64,2"])
def test_every_cut_in_every_storage_order(cut, monkeypatch):
    """The diagnostic switch makes every product take the cut where it can; operands in both orders."""
    monkeypatch.setenv("CCONV_BLOCK_CUT", cut)
    flip = lambda t: t.t().contiguous().t()  # noqa: E731
    for T, D, F, dtype in ((24, 512, 640, BF16), (300, 520, 1032, FP16)):
        f = Ffn(T, D, F, dtype, "gelu")
        for names in ((), ("x", "dy"), ("wg", "wu", "wd"), ("x", "wg", "wu", "wd", "dy")):
            h = Ffn(T, D, F, dtype, "gelu")
            for n in names:
                setattr(h, n, flip(getattr(f, n)))
            h.check_forward(*h.forward(True), f"{cut} {names}")
            h.check_backward(*h.backward(), f"{cut} {names}")
    for M, N, K in ((20, 300, 1100), (300, 520, 2048)):
        a, sa, b, sb = fp8_operands(M, N, K)
        for dtype in (BF16, FP32):
            out = poisoned((M, N), dtype)
            block.fp8_product(a, sa, b, sb, out)
            fp8_check(a, sa, b, sb, out, cut)
    assert block.status() == (0, 0)


def shifted(t, pitch, by):
    """The same values in rows `pitch` apart, `by` elements behind an allocation's start."""
    buf = torch.full((by + pitch * t.shape[0] + 8,), float("nan"), dtype=t.dtype, device="cuda")
    v = buf.as_strided(t.shape, (pitch, 1), by)
    v.copy_(t)
    return v


# rows that begin anywhere, enough of them for the ring: T >= 4 rows a block of up to 16 blocks on 148 SMs
@pytest.mark.parametrize("T,D,dtype,gate,rows", [
    (2400, 4095, BF16, "groups", 300), (2500, 2049, FP16, "all", 0), (9600, 1001, BF16, "groups", 1), (9600, 67, FP16, "groups", 777),
    (9500, 700, BF16, "none", 0), (4800, 1999, BF16, "groups", 5000), (1200, 5001, FP32, "none", 0), (4800, 1026, FP32, "all", 0),
    (1250, 8190, BF16, "groups", 1250), (4800, 1500, BF16, "groups", 7), (9600, 33, FP32, "groups", 1)])
@pytest.mark.parametrize("by,pad", [(0, 0), (3, 0), (1, 5)])
def test_norms_of_many_rows_that_begin_anywhere(T, D, dtype, gate, rows, by, pad):
    n = Norm(T, D, dtype, gate, rows, scale=0.75)
    for name in ("r", "y", "dr", "dx"):
        setattr(n, name, shifted(getattr(n, name), D + pad, by))
    n.check(*n.run(), "forward")
    inplace = shifted(n.r, D + pad, by)
    want = n.run()
    block.residual_norm_forward(inplace, inplace, torch.empty_like(want[1]), block=n.y, w_post=n.wpost, gate=n.gate,
                                w_pre=n.wpre, rows_per_gate=n.rows, scale=n.scale, eps=n.eps)
    assert torch.equal(inplace, want[0])
    got = n.run_backward()
    n.check_backward(got)
    inplace = shifted(n.dr, D + pad, by)
    like = lambda t: None if t is None else torch.empty_like(t)  # noqa: E731
    block.residual_norm_backward(inplace, n.dx, n.o, inplace, block=n.y, dblock=like(got[1]), w_post=n.wpost,
                                 dw_post=like(got[2]), gate=n.gate, dgate=like(got[3]), w_pre=n.wpre, dw_pre=like(got[4]),
                                 rows_per_gate=n.rows, scale=n.scale, eps=n.eps)
    assert torch.equal(inplace, got[0])
    assert block.status() == (0, 0)


def test_norms_of_many_rows_with_parts_left_out():
    for kw in (dict(blk=False), dict(post=False), dict(pre=False), dict(gate="all", post=False)):
        n = Norm(2600, 1001, BF16, **kw)
        n.check(*n.run(), f"{kw}")
        n.check(*n.run(norm=False), f"{kw} without the second norm")
        n.check_backward(n.run_backward())
        n.check_backward(n.run_backward(use_dr=False), use_dr=False)
        n.check_backward(n.run_backward(use_dx=False), use_dx=False)
    assert block.status() == (0, 0)


# rows shared by the 2, 4 and 8 blocks of a cluster, the shortest and longest of each; rows that no cluster takes
@pytest.mark.parametrize("T,D,dtype,gate,rows", [
    (300, 8193, BF16, "groups", 33), (40, 16384, BF16, "all", 0), (37, 16385, FP16, "groups", 1), (150, 32768, BF16, "none", 0),
    (5, 32769, BF16, "groups", 2), (160, 65536, FP16, "groups", 160), (3, 65537, BF16, "all", 0), (200, 9999, FP32, "groups", 7),
    (6, 14000, FP32, "all", 0), (33, 20000, FP32, "groups", 33), (2, 12288, BF16, "groups", 1), (1, 16384, BF16, "all", 0)])
@pytest.mark.parametrize("by,pad", [(0, 0), (1, 3)])
def test_norm_gradients_of_long_rows(T, D, dtype, gate, rows, by, pad):
    n = Norm(T, D, dtype, gate, rows, scale=0.75)
    for name in ("r", "y", "dr", "dx"):
        setattr(n, name, shifted(getattr(n, name), D + pad, by))
    got = n.run_backward()
    n.check_backward(got)
    for again in range(3):  # sums in a fixed order
        for a, b in zip(got, n.run_backward()):
            assert a is b or torch.equal(a, b)
    n.check_backward(n.run_backward(use_dr=False), use_dr=False)
    n.check_backward(n.run_backward(use_dx=False), use_dx=False)
    assert block.status() == (0, 0)


def test_an_empty_call_between_two_convolutions_keeps_them_in_order():
    """The same with calls of zero length, which launch nothing: the second convolution follows the first."""
    B, C, K, H = 64, 64, 128, 14
    g = gen(12)
    image = normal(g, (H + 2, H + 2, C, B), BF16)
    f1, f2 = normal(g, (C, 3, 3, C), BF16, (9 * C) ** -0.5), normal(g, (K, 1, 1, C), BF16, C ** -0.5)
    e = Ffn(0, 128, 256)
    a, sa, b, sb = fp8_operands(2, 128, 128)
    no, row = torch.empty((0, 128), dtype=BF16, device="cuda"), torch.empty((0, 1), device="cuda")
    between = (lambda: e.forward(True), lambda: block.fp8_product(a[:0], sa[:0], b, sb, no),
               lambda: block.residual_norm_backward(None, no, no, torch.empty_like(no)),
               lambda: block.quantize_blocks(no, torch.empty((0, 128), dtype=E4M3, device="cuda"), row))
    middles = [torch.empty((C, H, H, B), dtype=BF16, device="cuda") for _ in range(12)]

    def chain(sync):
        outs = []
        for mid in middles:
            mid.zero_()
        torch.cuda.synchronize()
        for i, mid in enumerate(middles):
            out = torch.zeros((K, H, H, B), dtype=BF16, device="cuda")
            for one in (lambda: binding.conv_forward(image, f1, mid, B, C, C, H, H, 3, 3), between[i % 4],
                        lambda: binding.conv_forward(mid.view(H, H, C, B), f2, out, B, C, K, H, H, 1, 1)):
                one()
                if sync:
                    torch.cuda.synchronize()
            outs.append(out)
        torch.cuda.synchronize()
        return outs
    want = chain(True)
    for _ in range(3):
        for x, y in zip(want, chain(False)):
            assert torch.equal(x, y)


def test_pre_activations_in_the_columns_of_one_array_in_turn():
    for T, D, F in ((3, 72, 136), (40, 72, 136), (300, 72, 136)):
        f = Ffn(T, D, F)
        both, out = poisoned((T, 2 * F), BF16), poisoned((T, D), BF16)
        block.ffn_forward(f.x, f.wg, f.wu, f.wd, out, gate_pre=both[:, ::2], up_pre=both[:, 1::2])
        f.check_forward(out, both[:, ::2], both[:, 1::2], "in turn")
        f.g, f.u = both[:, ::2], both[:, 1::2]
        f.check_backward(*f.backward(), "in turn")


def workspace(name, struct, addresses, matrices, **sizes):
    s = struct_of(struct)()
    for k, v in sizes.items():
        setattr(s, k, v)
    for i, (k, (rs, cs)) in enumerate(matrices.items()):
        m = getattr(s, k)
        m.data, m.row_stride, m.col_stride = addresses(i), rs, cs
    f = getattr(binding.load_library(), name)
    f.restype, f.argtypes = ctypes.c_int64, [ctypes.c_void_p]
    return f(ctypes.addressof(s))


@pytest.mark.parametrize("T", [2, 40, 333, 3000])
@pytest.mark.parametrize("step", [1, 2])
def test_the_workspace_does_not_depend_on_which_addresses_are_equal(T, step):
    """A query with one placeholder for every matrix, or with none, gives what the call needs: odd sizes, so that
    every operand is copied, and results that go through the workspace too."""
    far, same, none = (lambda i: (i + 1) << 30), (lambda i: 1 << 30), (lambda i: None)
    # T = D and D = F too: then matrices of different arguments have equal shapes and strides
    for D, F in ((T if T % 2 else T + 1, 263), (263, 263)):
        fd, td, tf, df = (D * step, step), (D * step, step), (F * step, step), (F * step, step)
        for name, m in (
                ("cconv_ffn_forward_workspace", dict(x=td, w_gate=fd, w_up=fd, w_down=df, out=td)),
                ("cconv_ffn_backward_workspace", dict(x=td, dout=td, w_gate=fd, w_up=fd, w_down=df, gate_pre=tf, up_pre=tf, dx=td,
                                                      dw_gate=fd, dw_up=fd, dw_down=df))):
            sizes = [workspace(name, "cconv_ffn_args", a, m, T=T, D=D, F=F, dtype=block.TYPE_BF16) for a in (far, same, none)]
            assert sizes[0] > 0 and sizes[0] == sizes[1] == sizes[2], (name, sizes)
    m = dict(a=(D * step, step), b=(D * step, step), a_scale=(99, 1), b_scale=(99, 1), c=(F * step, step))
    sizes = [workspace("cconv_fp8_product_workspace", "cconv_fp8_product_args", a, m, M=T, N=F, K=D, dtype=block.TYPE_BF16)
             for a in (far, same, none)]
    assert sizes[0] > 0 and sizes[0] == sizes[1] == sizes[2], sizes


def tail_inputs(act, dtype, T, F):
    """T x F pre-activations over both tails, to where the exponential's argument reaches 85, and that argument."""
    far = {"silu": 85.0, "gelu": 13.0, "gelu_tanh": 9.8, "relu": 9.0}[act]
    far = min(far, 9.0) if dtype is FP16 else far
    g = ((torch.rand((T, F), generator=gen(T + F), device="cuda") * 2 - 1) * far).to(dtype)
    v = g.double()
    z = {"silu": v, "gelu": v * v / 2, "gelu_tanh": 2 * (2 / torch.pi) ** 0.5 * (v + 0.044715 * v ** 3), "relu": 0 * v}[act]
    return g, z.abs()


def act64_in_the_tails(name, g):
    """a(g), a'(g) and the first of the two terms that a' adds, in 64 bits without a difference from 1 (as 1 + tanh
    and 1 + erf are, which leave nothing of values below 1e-16)."""
    if name == "silu":
        s, rest = torch.sigmoid(g), torch.sigmoid(-g)
        return g * s, s + g * s * rest, s
    if name == "gelu":
        cdf = torch.special.erfc(-g * 0.5 ** 0.5) / 2
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5, cdf
    if name == "gelu_tanh":
        k = 2 * (2 / torch.pi) ** 0.5
        s, rest = (torch.sigmoid(sign * k * (g + 0.044715 * g ** 3)) for sign in (1, -1))
        return g * s, s + g * s * rest * k * (1 + 3 * 0.044715 * g * g), s
    on = (g > 0).double()
    return g * on, on, on


# The hidden values reach the result one by one: w_gate and w_down are identities, u is 512 everywhere.  The fast
# exponential is off by 2 + 1.2 |z| units, its argument's roundings by up to 2.5 |z|, the rest by fewer than 14.
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("T", [2, 16, 100, 300])
def test_hidden_values_are_right_relative_to_themselves(act, dtype, T):
    F, D, u = 64, 128, {BF16: 2.0 ** -8, FP16: 2.0 ** -11}[dtype]
    g, z = tail_inputs(act, dtype, T, F)
    x = torch.zeros((T, D), device="cuda", dtype=dtype)
    x[:, :F], x[:, F] = g, 512.0
    wg, wu, wd = (torch.zeros(s, device="cuda", dtype=dtype) for s in ((F, D), (F, D), (D, F)))
    wg[:, :F], wd[:F], wu[:, F] = torch.eye(F, device="cuda"), torch.eye(F, device="cuda"), 1.0
    out = poisoned((T, D), dtype)
    block.ffn_forward(x, wg, wu, wd, out, act=block.ACTS[act])
    h = 512 * act64_in_the_tails(act, g.double())[0]
    tiny = 2.0 ** -24 if dtype is FP16 else 1e-36
    close(out[:, :F], h, 1.01 * (u + 2.0 ** -23 * (16 + 4 * z)) * h.abs() + tiny, f"{act} of {T}")
    assert (out[:, F:] == 0).all()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("T", [16, 128, 320])
def test_hidden_gradients_are_right_relative_to_themselves(act, dtype, T):
    """As many tokens as channels, dout and x identities: dw_down = h, dw_up = (dL/du)^T, dw_gate = (dL/dg)^T, where
    dL/dh = w_down = 512.  dL/dg adds two terms, relative to whose sizes it is right."""
    F, D, u = 64, T, {BF16: 2.0 ** -8, FP16: 2.0 ** -11}[dtype]
    g, z = tail_inputs(act, dtype, T, F)
    eye, up = torch.eye(T, device="cuda").to(dtype), torch.full((T, F), 2.0, device="cuda").to(dtype)
    wg, wu = torch.zeros((F, D), device="cuda", dtype=dtype), torch.zeros((F, D), device="cuda", dtype=dtype)
    wd = torch.full((D, F), 512.0, device="cuda").to(dtype)
    dx, dwg, dwu, dwd = poisoned((T, D), dtype), poisoned((F, D), dtype), poisoned((F, D), dtype), poisoned((D, F), dtype)
    block.ffn_backward(eye, eye, wg, wu, wd, g, up, dx, dwg, dwu, dwd, act=block.ACTS[act])
    v = g.double()
    a, da, share = act64_in_the_tails(act, v)
    size = share.abs() + (da - share).abs()
    tiny = 2.0 ** -24 if dtype is FP16 else 1e-35
    off = 2.0 ** -23 * (16 + 4 * z)
    close(dwd, 2 * a, 1.01 * (u + off) * 2 * a.abs() + tiny, act + " h")
    close(dwu.t(), 512 * a, 1.01 * (u + off) * 512 * a.abs() + tiny, act + " dL/du")
    close(dwg.t(), 1024 * da, 1.01 * 1024 * (u * da.abs() + off * size) + tiny, act + " dL/dg")
    assert (dx == 0).all()


# every backward kernel: wide rows, rows that begin anywhere (few, many), rows that clusters share, longer ones
EVERY_NORM_KERNEL = [(5, 256), (700, 1024), (3, 251), (2400, 1001), (6, 9999), (1, 12001)]


@pytest.mark.parametrize("T,D", EVERY_NORM_KERNEL)
def test_norm_gradients_of_rows_of_any_size(T, D):
    """Values of 1e15 (rho^3 is below the least fp32 number), of 1e-14 and 0 under an eps of 1e-30 (it is above
    the largest): the bound is relative, as for rows near 1."""
    for dtype in (FP32, BF16):
        n = Norm(T, D, dtype, "all")
        n.r, n.y = n.r * 1e15, n.y * 1e15
        n.check_backward(n.run_backward(use_dr=False), use_dr=False, what="large")
        n = Norm(T, D, dtype, blk=False, eps=1e-30)
        n.r = n.r * 1e-14
        n.r[T - 1] = 0
        n.check_backward(n.run_backward(use_dr=False), use_dr=False, what="small")
        n = Norm(T, D, dtype, "all", eps=1e-30)
        n.y = n.y * 1e-14
        n.y[T - 1] = 0
        n.check_backward(n.run_backward(), what="small block")
    assert block.status() == (0, 0)


@pytest.mark.parametrize("T,D", EVERY_NORM_KERNEL)
def test_without_a_norm_the_block_s_gradient_does_not_depend_on_the_block(T, D):
    n = Norm(T, D, BF16, "all", post=False)
    want = n.run_backward(use_dx=False)
    n.y[0, 1], n.y[0, 2], n.y[T - 1, 3] = float("inf"), float("nan"), float("-inf")
    got = n.run_backward(use_dx=False)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_pre_activations_of_any_finite_size(act):
    """Up to the ends of bf16's range every activation is g or 0, and its derivative 1 or 0."""
    T, F = 64, 64
    g = torch.cat([s * 10.0 ** torch.arange(3.0, 35.0, device="cuda") for s in (1, -1)]).to(BF16).expand(T, F).contiguous()
    eye = torch.eye(T, device="cuda").to(BF16)
    up = torch.full((T, F), 2.0, device="cuda").to(BF16)
    wd, none = torch.ones((T, F), device="cuda").to(BF16), torch.zeros((F, T), device="cuda").to(BF16)
    dx, dwg, dwu, dwd = poisoned((T, T), BF16), poisoned((F, T), BF16), poisoned((F, T), BF16), poisoned((T, F), BF16)
    block.ffn_backward(eye, eye, none, none, wd, g, up, dx, dwg, dwu, dwd, act=block.ACTS[act])
    on = (g > 0).double()
    # (products with the identity add zeros: values are exact but for their own rounding, 1 of them 2^-8)
    close(dwd, 2 * g.double() * on, 2.0 ** -8 * 2 * g.double().abs() * on, act + " h")
    close(dwu.t(), g.double() * on, 2.0 ** -8 * g.double().abs() * on, act + " dL/du")
    close(dwg.t(), 2 * on, 2.0 ** -7 * on, act + " dL/dg")


def embedded(shape, dtype, pad, above=1, left=0):
    """A result inside a larger array, from a 16-byte boundary on and at a pitch of 16 bytes where `pad` allows."""
    big = torch.full((shape[0] + above + 1, left + shape[1] + pad), 5.0, device="cuda").to(dtype)
    return big, big[above:above + shape[0], left:left + shape[1]]


def pitch_to(n, unit):
    return -n % unit + unit


# rows that end within 16 bytes, with the next row or another array right behind them
@pytest.mark.parametrize("T,D,F", [(1, 69, 133), (6, 1, 5), (20, 69, 133), (70, 129, 63), (260, 257, 131), (700, 65, 1021)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_ffn_results_of_any_length_leave_their_surroundings(T, D, F, dtype):
    f = Ffn(T, D, F, dtype)
    for left in (0, 8):
        bufs = [embedded(s, dtype, pitch_to(s[1], 8), left=left) for s in ((T, D), (T, F), (T, F))]
        for save in (True, False):
            block.ffn_forward(f.x, f.wg, f.wu, f.wd, bufs[0][1], gate_pre=bufs[1][1] if save else None,
                              up_pre=bufs[2][1] if save else None)
            f.check_forward(bufs[0][1], *((bufs[1][1], bufs[2][1]) if save else (None, None)))
            for big, v in bufs:
                v.fill_(5.0)
                assert (big == 5.0).all()
        bufs = [embedded(s, dtype, pitch_to(s[1], 8), left=left) for s in ((T, D), (F, D), (F, D), (D, F))]
        block.ffn_backward(f.dy, f.x, f.wg, f.wu, f.wd, f.g, f.u, *[v for _, v in bufs])
        f.check_backward(*[v for _, v in bufs])
        for big, v in bufs:
            v.fill_(5.0)
            assert (big == 5.0).all()


@pytest.mark.parametrize("M,N,K", [(1, 345, 897), (3, 5, 128), (40, 133, 256), (232, 1, 1), (600, 1021, 384)])
@pytest.mark.parametrize("dtype,unit", [(BF16, 8), (FP16, 8), (FP32, 4)])
def test_fp8_results_of_any_length_leave_their_surroundings(M, N, K, dtype, unit):
    a, sa, b, sb = fp8_operands(M, N, K)
    for left in (0, unit):
        big, v = embedded((M, N), dtype, pitch_to(N, unit), left=left)
        block.fp8_product(a, sa, b, sb, v)
        fp8_check(a, sa, b, sb, v)
        v.fill_(5.0)
        assert (big == 5.0).all()


def test_norms_and_values_in_8_bits_of_any_length_leave_their_surroundings():
    for T, D in ((3, 69), (40, 1001), (2500, 1001), (6, 8201), (2, 20001), (2500, 260)):
        for dtype in (BF16, FP32):
            n = Norm(T, D, dtype, "groups", max(1, T // 3))
            (big, v), (big2, v2) = embedded((T, D), dtype, pitch_to(D, 8)), embedded((T, D), dtype, pitch_to(D, 8))
            n.check(*n.run(out=v, xout=v2))
            want = n.run_backward()
            (big3, v3), (big4, v4), (big5, v5) = (embedded(t.shape, dtype, pitch_to(D, 8)) for t in (want[0], want[1], want[3]))
            vectors = [torch.full((D + 16,), 5.0, device="cuda").to(dtype) for _ in range(2)]
            block.residual_norm_backward(n.dr, n.dx, n.o, v3, block=n.y, dblock=v4, w_post=n.wpost, dw_post=vectors[0][8:8 + D],
                                         gate=n.gate, dgate=v5, w_pre=n.wpre, dw_pre=vectors[1][8:8 + D], rows_per_gate=n.rows,
                                         scale=n.scale, eps=n.eps)
            n.check_backward((v3, v4, vectors[0][8:8 + D], v5, vectors[1][8:8 + D]))
            for whole, part in ((big, v), (big2, v2), (big3, v3), (big4, v4), (big5, v5), *((t, t[8:8 + D]) for t in vectors)):
                part.fill_(5.0)
                assert (whole == 5.0).all()
        x = normal(gen(T), (T, D), BF16)
        for rows in (1, 128):
            bytes_, q = embedded((T, D), torch.int8, pitch_to(D, 8))
            big, s = embedded((-(-T // rows), -(-D // 128)), FP32, 4)
            block.quantize_blocks(x, q.view(E4M3), s, block_rows=rows)
            q.fill_(5)
            s.fill_(5.0)
            assert (bytes_ == 5).all() and (big == 5.0).all()


def test_random_sequences_with_convolutions_run_in_order(monkeypatch):
    """Calls of every kind, empty ones among them, over five buffers that they read and write in turn: without
    synchronisation bit for bit what they give with a synchronisation after each.  (Convolutions that have to wait
    would take another kernel, which rounds otherwise; the switch keeps them on one.)"""
    monkeypatch.setenv("CCONV_WAIT_TWIN", "0")
    rng = random.Random(4)
    B, C, H, D = 64, 64, 13, 208
    n, g = H * H * C * B, gen(21)
    f3, f1 = normal(g, (C, 3, 3, C), BF16, (9 * C) ** -0.5), normal(g, (C, 1, 1, C), BF16, C ** -0.5)
    wg, wu, wd, w = normal(g, (320, D), BF16, D ** -0.5), normal(g, (320, D), BF16, D ** -0.5), normal(g, (D, 320), BF16, 0.06), normal(g, (D,), BF16)
    w8, s8 = torch.empty((D, D), dtype=E4M3, device="cuda"), torch.empty((2, 2), device="cuda")
    block.quantize_blocks(normal(g, (D, D), BF16, D ** -0.5), w8, s8, block_rows=128)
    start = [normal(g, (n,), BF16) for _ in range(5)]
    kinds = ("conv3", "conv1", "conv1", "ffn", "ffn", "norm", "in place", "backward", "fp8", "quantize", "empty", "torch")

    def run(calls, sync):
        bufs = [t.clone() for t in start]
        q, s, dw = torch.zeros((n // D, D), dtype=E4M3, device="cuda"), torch.zeros((n // D, 2), device="cuda"), torch.zeros_like(w)
        torch.cuda.synchronize()
        for kind, i, j, k, T, at in calls:
            a, b, c = (bufs[m][at:at + T * D].view(T, D) for m in (i, j, k))
            x, y = bufs[i].view(H, H, C, B), bufs[j]
            if kind == "conv3":
                binding.conv_forward(x, f3, y[:11 * 11 * C * B].view(C, 11, 11, B), B, C, C, 11, 11, 3, 3)
            elif kind == "conv1":
                binding.conv_forward(x, f1, y.view(C, H, H, B), B, C, C, H, H, 1, 1)
            elif kind == "ffn":
                block.ffn_forward(a, wg, wu, wd, b)
            elif kind == "norm":
                block.residual_norm_forward(a, b, c, w_pre=w, scale=0.5)
            elif kind == "in place":
                block.residual_norm_forward(a, a, b, block=c, w_post=w, w_pre=w, scale=0.5)
            elif kind == "backward":
                block.residual_norm_backward(a, b, c, a, w_pre=w, dw_pre=dw, scale=0.25)
            elif kind == "quantize":
                block.quantize_blocks(a, q[:T], s[:T])
            elif kind == "fp8":
                block.fp8_product(q[:T], s[:T], w8, s8, b)
            elif kind == "empty":
                block.ffn_forward(a[:0], wg, wu, wd, b[:0])
            else:
                b.copy_(a * 0.5)
            if sync:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return [*bufs, q.view(torch.uint8), s, dw]
    for _ in range(100):
        calls = [(rng.choice(kinds), *rng.sample(range(5), 3), rng.choice([1, 3, 16, 40, 300, 1500, n // D - 40]), rng.choice([0, 8, 8192]))
                 for _ in range(rng.randint(5, 30))]
        want = run(calls, True)
        for _ in range(2):
            for x, y in zip(want, run(calls, False)):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), calls
    assert block.status() == (0, 0)
