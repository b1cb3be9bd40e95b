"""Calls of the sub-block whose kernels were once slowed down by a change that left their results as they were: times
against a neighbour's in the same process.  The limits lie in the middle between the two measured ratios (B200)."""
import pytest
import torch

from paper_1802_06905_b200 import block
from test_gpu_block import BF16, FP32, gen, normal, poisoned

pytestmark = pytest.mark.gpu


def pace(calls, n=20, rounds=7):
    """The least time of n calls of each, measured in turn."""
    best = [float("inf")] * len(calls)
    for _ in range(rounds):
        for i, call in enumerate(calls):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            torch.cuda.synchronize()
            a.record()
            for _ in range(n):
                call()
            b.record()
            b.synchronize()
            best[i] = min(best[i], a.elapsed_time(b))
    return best


def forward_norm(T, D):
    g = gen(T + D)
    resid, y, w = normal(g, (T, D), BF16), normal(g, (T, D), BF16), normal(g, (D,), BF16)
    gate = normal(g, (-(-T // 2048), D), BF16)
    out, x = torch.empty_like(resid), torch.empty_like(resid)
    return lambda: block.residual_norm_forward(resid, out, x, block=y, w_post=w, gate=gate, w_pre=w, rows_per_gate=2048)


# ratios before and after the mend: with too few blocks an SM 2.04 and 1.41, 1.50 and 1.22;
# of a block a row 2.62 and 1.87 (against 1000 channels)
@pytest.mark.parametrize("T,D,limit", [(16384, 4095, 1.72), (16384, 2047, 1.36), (2400, 1001, 2.22)])
def test_rows_that_begin_anywhere_keep_their_pace(T, D, limit):
    odd, even = pace([graph_of(forward_norm(T, d), 20).replay for d in (D, D + 1 if T > 10000 else 1000)], n=3)
    assert odd < limit * even, (odd, even)


def graph_of(call, n=1):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            for _ in range(n):
                call()
    torch.cuda.synchronize()
    return g


def test_clipping_adds_the_sums_of_many_tensors_up_once():
    """Of tensors of so many that they take 200 launches: the norm alone and the clipping with a given norm take as long
    together as both at once (which took 2.4 times as long where every launch added up the sums of all)."""
    flat = normal(gen(1), (64000,), FP32)
    grads, outs = (block.TensorList([v for v in t.split(1)]) for t in (flat, torch.empty_like(flat)))
    norm, alone = poisoned((1,), FP32), poisoned((1,), FP32)
    both = graph_of(lambda: block.clip_gradients(grads, 1.0, norm, outs=outs))
    first = graph_of(lambda: block.gradient_norm(grads, alone))
    second = graph_of(lambda: block.clip_gradients(grads, 1.0, norm, outs=outs, norm_given=True))
    t = pace([both.replay, first.replay, second.replay], n=2)
    assert torch.equal(norm, alone)
    assert t[0] < 1.5 * (t[1] + t[2]), t
