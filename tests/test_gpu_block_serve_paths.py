"""How the operators that serve the sub-block and clip its gradients are called: streams, captured graphs, workspaces,
convolutions between them, results' surroundings, and all of them together."""
import pytest
import torch

from paper_1802_06905_b200 import binding, block
from test_gpu_block import BF16, E4M3, FP16, FP32, close, gen, normal, poisoned
from test_gpu_block_paths import embedded, pitch_to
from test_gpu_block_serve import U8, Int4, Moe, Norm, check_clipped, gradients, norm64

pytestmark = pytest.mark.gpu


class Call:
    """One call with operands of its own: run() gives the results, inputs are `inputs`."""

    def __init__(self, run, *inputs):
        self.run, self.inputs = run, inputs


def calls():
    """A call of every kind: every kernel that a size chooses."""
    out = {}
    for T, D in ((1, 4096), (40, 1000), (1300, 512), (2400, 333), (2, 17000)):
        n = Norm(T, D)
        out[f"norm {T}x{D}"] = Call(n.run, n.resid, n.block)
    for M, N, K, group in ((1, 4800, 512, 128), (2, 300, 1000, 32), (7, 4096, 4096, 64), (23, 500, 1030, 64), (64, 700, 512, 32), (200, 256, 640, 128)):
        c = Int4(M, N, K, group, zero=group != 128)
        out[f"int4 {M}x{N}x{K}"] = Call(lambda c=c, **kw: (c.run(**kw),), c.x)
    for T, D, F, E, k in ((1, 1024, 256, 16, 4), (5, 200, 136, 10, 3), (40, 333, 60, 6, 2), (70, 128, 128, 4, 2)):
        m = Moe(T, D, F, E, k)
        out[f"moe {T}x{D}x{F}"] = Call(m.run, m.x)
    for shapes in ([((300, 700), BF16), ((700,), FP32)] * 3, [((33,), FP32)] * 400):
        g = gradients(shapes)
        lst = block.TensorList(g)

        def run(g=g, lst=lst, **kw):
            outs, norm = [poisoned(t.shape, t.dtype) for t in g], poisoned((1,), FP32)
            block.clip_gradients(lst, 0.1, norm, outs=outs, **kw)
            return (norm, *outs)
        out[f"clip {len(g)}"] = Call(run, *g)
    w = normal(gen(3), (70, 520), BF16)

    def quantize(**kw):
        q, s, z = torch.zeros((70, 260), device="cuda", dtype=U8), poisoned((70, 9), FP16), torch.zeros((70, 9), device="cuda", dtype=U8)
        return block.quantize_groups(w, q, s, zero=z, group=64, **kw)
    out["quantize"] = Call(quantize, w)
    return out


def same(a, b):
    for x, y in zip(a, b):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


@pytest.fixture(scope="module")
def every():
    return calls()


def test_they_repeat_bit_for_bit_on_any_stream(every):
    side = torch.cuda.Stream()
    for name, c in every.items():
        want = c.run()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            a = c.run()
        torch.cuda.synchronize()
        b = c.run(stream=side)
        torch.cuda.synchronize()
        same(want, a), same(want, b)
    assert block.status() == (0, 0)


def test_in_cuda_graphs(every):
    """Captured, replayed with other inputs: what an eager call gives for those; two graphs in turn and one after
    the other."""
    graphs = {}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for name, c in every.items():
        with torch.cuda.stream(side):
            c.run()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                results = c.run()
        graphs[name] = (g, results)
    torch.cuda.synchronize()
    for step in range(2):
        for c in every.values():
            for t in c.inputs:
                t.copy_(normal(gen(step + 40), t.shape, t.dtype, 0.5))
        torch.cuda.synchronize()
        want = {name: c.run() for name, c in every.items()}
        for g, results in graphs.values():
            for t in results:
                t.zero_()
        torch.cuda.synchronize()
        for g, _ in graphs.values():
            g.replay()
            g.replay()
        torch.cuda.synchronize()
        for name, (_, results) in graphs.items():
            same(want[name], results)


def test_two_streams_at_once(every):
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    want = {name: c.run() for name, c in every.items()}
    names = list(every)
    torch.cuda.synchronize()
    got = []
    for i in range(3 * len(names)):
        for s, name in ((a, names[i % len(names)]), (b, names[(i * 5 + 2) % len(names)])):
            with torch.cuda.stream(s):
                got.append((name, every[name].run()))
    torch.cuda.synchronize()
    for name, results in got:
        same(want[name], results)


def test_calls_between_convolutions_keep_them_in_order(every):
    """A convolution reads what one two calls in front wrote; the calls between them touch neither array."""
    B, C, K, H = 64, 64, 128, 14
    g = gen(11)
    image = normal(g, (H + 2, H + 2, C, B), BF16)
    f1, f2 = normal(g, (C, 3, 3, C), BF16, (9 * C) ** -0.5), normal(g, (K, 1, 1, C), BF16, C ** -0.5)
    between = list(every.values())
    middles = [torch.empty((C, H, H, B), dtype=BF16, device="cuda") for _ in between]

    def chain(sync):
        outs = []
        for mid in middles:
            mid.zero_()
        torch.cuda.synchronize()
        for c, mid in zip(between, middles):
            out = torch.zeros((K, H, H, B), dtype=BF16, device="cuda")
            for call in (lambda: binding.conv_forward(image, f1, mid, B, C, C, H, H, 3, 3), c.run,
                         lambda: binding.conv_forward(mid.view(H, H, C, B), f2, out, B, C, K, H, H, 1, 1)):
                call()
                if sync:
                    torch.cuda.synchronize()
            outs.append(out)
        torch.cuda.synchronize()
        return outs
    want = chain(True)
    for _ in range(3):
        for x, y in zip(want, chain(False)):
            assert torch.equal(x, y)


def test_convolutions_that_read_results_and_write_operands_wait():
    """out = operator(conv(image)), conv again on the result: without waiting as with a synchronisation after each."""
    B, C, H = 64, 64, 13
    g = gen(12)
    n = H * H * C * B
    f = normal(g, (C, 1, 1, C), BF16, C ** -0.5)
    start = normal(g, (n,), BF16)
    D, T = 64, 60
    four = Int4(T, D, D)
    m = Moe(T, D, 96, 4, 2)
    w = torch.ones(D, device="cuda", dtype=BF16)

    def run(kind, sync):
        a, b = start.clone(), torch.zeros_like(start)
        q, s = torch.zeros((T, D), dtype=E4M3, device="cuda"), torch.zeros((T, 1), device="cuda")
        norm, ids, weights = torch.zeros(1, device="cuda"), torch.zeros((T, 2), device="cuda", dtype=torch.int32), torch.zeros((T, 2), device="cuda")
        torch.cuda.synchronize()
        for _ in range(6):
            binding.conv_forward(a.view(H, H, C, B), f, b.view(C, H, H, B), B, C, C, H, H, 1, 1)
            if sync:
                torch.cuda.synchronize()
            x, y = b[:T * D].view(T, D), a[64:64 + T * D].view(T, D)
            if kind == "int4":
                block.int4_product(x, four.q, four.scale, y)
            elif kind == "moe":
                block.moe_forward(x, m.router, m.wg, m.wu, m.wd, y, ids, weights)
            elif kind == "norm":
                block.residual_norm_quantize(x, y, q, s, w_pre=w)
            else:
                block.clip_gradients([b, x.t()], 3.0, norm, outs=[a, torch.empty_like(x).t()])
            if sync:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return a, b, q, s, norm, ids
    for kind in ("int4", "moe", "norm", "clip"):
        want = run(kind, True)
        for _ in range(3):
            same(want, run(kind, False))


def test_results_leave_their_surroundings():
    for M, N, K in ((1, 345, 256), (5, 133, 1000), (40, 77, 130), (90, 201, 264)):
        for group in (32, 128):
            c = Int4(M, N, K, group, zero=True)
            big, v = embedded((M, N), BF16, pitch_to(N, 8))
            c.check(c.run(out=v))
            v.fill_(5.0)
            assert (big == 5.0).all()
    for T, D, F in ((1, 77, 40), (9, 1001, 33), (70, 130, 64)):
        m = Moe(T, D, F, 5, 2)
        (big, v), (big2, ids), (big3, weights) = embedded((T, D), BF16, pitch_to(D, 8)), embedded((T, 2), torch.int32, 4), embedded((T, 2), FP32, 4)
        block.moe_forward(m.x, m.router, m.wg, m.wu, m.wd, v, ids, weights)
        m.check_routes(ids, weights)
        m.check_out(v, ids, weights)
        for whole, part in ((big, v), (big2, ids), (big3, weights)):
            part.fill_(5)
            assert (whole == 5).all()
    for N, K in ((5, 33), (70, 257), (3, 1001)):
        (big, q), (big2, s), (big3, z) = (embedded((N, -(-K // 2)), U8, pitch_to(-(-K // 2), 4)), embedded((N, -(-K // 64)), FP32, 4),
                                          embedded((N, -(-K // 64)), U8, 4))
        block.quantize_groups(normal(gen(N), (N, K), BF16), q, s, zero=z, group=64)
        for whole, part in ((big, q), (big2, s), (big3, z)):
            part.fill_(5)
            assert (whole == 5).all()


def test_workspaces():
    """The caller's own, of the size that the library gives, whatever it holds; a smaller or a shifted one is refused."""
    four, m = Int4(5, 70, 301, 64), Moe(6, 77, 33, 5, 2)
    g = gradients([((300, 700), BF16), ((9,), FP32)])
    norm = poisoned((1,), FP32)
    out, mo = poisoned((5, 70), BF16), poisoned((6, 77), BF16)
    ids, weights = torch.zeros((6, 2), device="cuda", dtype=torch.int32), torch.zeros((6, 2), device="cuda")
    cases = (
        (block.int4_product_workspace(four.x, four.q, four.scale, out, group=64),
         lambda w: four.run(out=out, workspace=w), lambda: four.check(out)),
        (block.moe_workspace(m.x, m.router, m.wg, m.wu, m.wd, mo, ids, weights), lambda w: m.run(out=mo, workspace=w),
         lambda: m.check_out(mo, *m.run()[1:])),
        (block.clip_workspace(g), lambda w: block.gradient_norm(g, norm, workspace=w),
         lambda: close(norm, torch.tensor([norm64(g)], device="cuda", dtype=torch.float64), 1e-6 * norm64(g), "norm")))
    for n, call, check in cases:
        assert n > 0
        for byte in (0, 255):
            call(torch.full((n,), byte, device="cuda", dtype=U8))
            check()
        big = torch.zeros((n + 512,), device="cuda", dtype=U8)
        for bad in (big[:n - 1], big[16:n + 16]):
            with pytest.raises(block.CconvError):
                call(bad)


def test_a_caller_without_a_router_and_ranks_of_experts():
    """Two halves of the experts, each with the choices numbered from its first: the halves add up to the layer."""
    m = Moe(9, 256, 128, 8, 3)
    whole, ids, weights = m.run()
    parts = []
    for first in (0, 4):
        h = Moe(9, 256, 128, 8, 3)
        h.wg, h.wu, h.wd = h.wg[first:first + 4], h.wu[first:first + 4], h.wd[first:first + 4]
        parts.append(h.run(ids=ids - first, weights=weights)[0].double())
    # each half is rounded to 16 bits, and so is the whole
    close(whole, parts[0] + parts[1], 2.0 ** -8 * (whole.double().abs() + parts[0].abs() + parts[1].abs()) + 1e-6, "halves")


def test_clipping_across_lists():
    """The norm of two lists, each on its own, put together by the caller, clips both."""
    a, b = gradients([((100, 33), FP32)], 1), gradients([((64, 700), BF16)], 2)
    na, nb = poisoned((1,), FP32), poisoned((1,), FP32)
    block.gradient_norm(a, na)
    block.gradient_norm(b, nb)
    both = (na * na + nb * nb).sqrt()
    before = [t.clone() for t in a + b]
    m = 0.5 * norm64(a + b)
    block.clip_gradients(a, m, both, norm_given=True)
    block.clip_gradients(b, m, both, norm_given=True)
    check_clipped(a + b, before, both, m)


def test_trained_with_clipping_and_served_in_every_way():
    from paper_1802_06905_b200 import ffn_block
    r = ffn_block.run(tokens=96, channels=256, hidden=512, steps=6, serve=3, max_norm=0.5, experts=4, chosen=2)
    assert len(r["norm"]) == 6 and all(v > 0 for v in r["norm"])
    # 8-bit operands: 2^-4 of a factor at worst; 4 bits: steps of a seventh of the group's range; copies with 1 % of noise
    assert r["serve_error"] < 0.1 and r["serve_in_norm_error"] < 0.1
    assert r["serve_4_bit_error"] < 0.3 and r["mixture_error"] < 0.1
    free = ffn_block.run(tokens=96, channels=256, hidden=512, steps=6, serve=3)
    assert free["norm"] == []
    loose = ffn_block.run(tokens=96, channels=256, hidden=512, steps=6, serve=3, max_norm=1e6)
    assert loose["loss"] == free["loss"]  # a limit that is never reached changes nothing


def test_a_step_of_all_of_them_against_plain_forms():
    """norm in 8 bits -> 8-bit product; 4-bit product; mixture; from the same tokens, each against its definition."""
    T, D, N = 6, 512, 384
    n = Norm(T, D)
    x = poisoned((T, D), BF16)
    r, q, s = n.run(norm_out=x)
    w = normal(gen(5), (N, D), BF16, D ** -0.5)
    qw, sw = torch.empty((N, D), dtype=E4M3, device="cuda"), torch.empty((N // 128, D // 128), device="cuda")
    block.quantize_blocks(w, qw, sw, block_rows=128)
    y8 = poisoned((T, N), BF16)
    block.fp8_product(q, s, qw, sw, y8)
    exact = (q.double() * s.double().repeat_interleave(128, 1)) @ (qw.double() * sw.double().repeat_interleave(128, 0).repeat_interleave(128, 1)).T
    close(y8, exact, 2.0 ** -8 * exact.abs() + (D + 16) * 2.0 ** -23 * (q.double().abs() * s.double().repeat_interleave(128, 1))
          @ (qw.double().abs() * sw.double().repeat_interleave(128, 0).repeat_interleave(128, 1)).T * 1.01, "8-bit product")
    four = Int4(T, N, D, 64, zero=True)
    four.x = x
    block.quantize_groups(w, four.q, four.scale, zero=four.zero, group=64)
    four.check(four.run(), "4-bit product")
    m = Moe(T, D, 128, 8, 2)
    m.x = x
    out, ids, weights = m.run()
    m.check_routes(ids, weights)
    m.check_out(out, ids, weights)
    assert block.status() == (0, 0)
