"""A gated feed-forward sub-block of a network, trained for a few steps and then served in 8 bits.

    python -m paper_1802_06905_b200.ffn_block [--tokens T] [--channels D] [--hidden F] [--steps N] [--serve N]

Training (bf16): x = norm(r) w_in;  y = ffn(x);  r' = r + gate * norm(y) w_post;  z = norm(r') w_out;  squared
distance of z to a target; the backward pass of every step through the library, plain gradient descent on the
weights.  Serving: the trained weights in blocks of 128 x 128, one token a call through quantize_blocks and
fp8_product, compared with the same tokens in bf16.
"""
from __future__ import annotations

import argparse
import sys

import torch

from . import block


class FfnBlock:
    """Parameters of the sub-block and its two ways of running."""

    def __init__(self, channels, hidden, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def rand(*shape, scale):
            return (torch.randn(shape, generator=g, device=device) * scale).to(torch.bfloat16)
        D, F = channels, hidden
        self.D, self.F = D, F
        self.w_gate, self.w_up = rand(F, D, scale=D ** -0.5), rand(F, D, scale=D ** -0.5)
        self.w_down = rand(D, F, scale=F ** -0.5)
        ones = torch.ones(D, device=device, dtype=torch.bfloat16)
        self.w_in, self.w_post, self.w_out = ones.clone(), ones.clone(), ones.clone()
        self.gate = torch.full((1, D), 0.5, device=device, dtype=torch.bfloat16)

    def parameters(self):
        return {n: getattr(self, n) for n in ("w_gate", "w_up", "w_down", "w_in", "w_post", "w_out", "gate")}

    def forward(self, r):
        """z and what the backward pass needs."""
        T, D, F = r.shape[0], self.D, self.F
        new = lambda *s: torch.empty(s, dtype=r.dtype, device=r.device)  # noqa: E731
        r0, x, g, u, y, r1, z = new(T, D), new(T, D), new(T, F), new(T, F), new(T, D), new(T, D), new(T, D)
        block.residual_norm_forward(r, r0, x, w_pre=self.w_in)
        block.ffn_forward(x, self.w_gate, self.w_up, self.w_down, y, gate_pre=g, up_pre=u)
        block.residual_norm_forward(r0, r1, z, block=y, w_post=self.w_post, gate=self.gate, w_pre=self.w_out)
        return z, (r0, x, g, u, y, r1)

    def backward(self, saved, dz):
        """Gradients of all parameters, and of r."""
        r0, x, g, u, y, r1 = saved
        like = torch.empty_like
        grads = {n: like(p) for n, p in self.parameters().items()}
        dr, dy, dx = like(r0), like(y), like(x)
        block.residual_norm_backward(None, dz, r1, dr, block=y, dblock=dy, w_post=self.w_post, dw_post=grads["w_post"],
                                     gate=self.gate, dgate=grads["gate"], w_pre=self.w_out, dw_pre=grads["w_out"])
        block.ffn_backward(dy, x, self.w_gate, self.w_up, self.w_down, g, u, dx, grads["w_gate"], grads["w_up"],
                           grads["w_down"])
        block.residual_norm_backward(dr, dx, r0, dr, w_pre=self.w_in, dw_pre=grads["w_in"])
        return grads, dr


class Served:
    """The sub-block with its projections in 8 bits."""

    def __init__(self, b: FfnBlock):
        self.b = b
        both = torch.cat([b.w_gate, b.w_up])         # one product for both (F a multiple of 128)
        self.up, self.down = self._blocks(both), self._blocks(b.w_down)

    @staticmethod
    def _blocks(w):
        N, K = w.shape
        q = torch.empty((N, K), dtype=torch.float8_e4m3fn, device=w.device)
        s = torch.empty((-(-N // 128), -(-K // 128)), device=w.device)
        block.quantize_blocks(w, q, s, block_rows=128)
        return q, s

    @staticmethod
    def _tokens(x):
        T, K = x.shape
        q = torch.empty((T, K), dtype=torch.float8_e4m3fn, device=x.device)
        s = torch.empty((T, -(-K // 128)), device=x.device)
        block.quantize_blocks(x, q, s)
        return q, s

    def forward(self, r):
        b, T = self.b, r.shape[0]
        new = lambda n: torch.empty((T, n), dtype=r.dtype, device=r.device)  # noqa: E731
        r0, x, gu, y, r1, z = new(b.D), new(b.D), new(2 * b.F), new(b.D), new(b.D), new(b.D)
        block.residual_norm_forward(r, r0, x, w_pre=b.w_in)
        block.fp8_product(*self._tokens(x), *self.up, gu)
        h = torch.nn.functional.silu(gu[:, :b.F].float()) * gu[:, b.F:].float()
        block.fp8_product(*self._tokens(h.to(r.dtype)), *self.down, y)
        block.residual_norm_forward(r0, r1, z, block=y, w_post=b.w_post, gate=b.gate, w_pre=b.w_out)
        return z


def run(tokens=2048, channels=1024, hidden=4096, steps=10, serve=8, lr=None):
    """Trains and serves; the losses, and how far 8-bit serving is from 16 bits (of the result's norm)."""
    if hidden % 128:
        raise ValueError("hidden must be a multiple of 128")
    b = FfnBlock(channels, hidden)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    r = torch.randn((tokens, channels), generator=g, device="cuda").to(torch.bfloat16)
    target = torch.randn((tokens, channels), generator=g, device="cuda")
    lr = 0.3 if lr is None else lr
    losses = []
    for _ in range(steps):
        z, saved = b.forward(r)
        diff = z.float() - target
        losses.append((diff * diff).mean().item())
        grads, _ = b.backward(saved, (diff * (2.0 / tokens)).to(torch.bfloat16))
        for n, p in b.parameters().items():
            p.copy_(p.float() - lr * grads[n].float())
    s = Served(b)
    full = b.forward(r[:serve])[0].float()
    served = torch.cat([s.forward(r[i:i + 1]) for i in range(serve)]).float()
    error = ((served - full).norm() / full.norm()).item()
    code, detail = block.status()
    if code != block.OK:
        raise block.CconvError(code, f"cconv_block_status (detail={detail:#x})")
    return {"loss": losses, "serve_error": error}


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--channels", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--serve", type=int, default=8)
    a = ap.parse_args(argv)
    r = run(a.tokens, a.channels, a.hidden, a.steps, a.serve)
    print("loss " + " ".join(f"{v:.4f}" for v in r["loss"]))
    print(f"8-bit serving differs from bf16 by {r['serve_error']:.4f} of the result's norm")
    return 0


if __name__ == "__main__":
    sys.exit(main())
