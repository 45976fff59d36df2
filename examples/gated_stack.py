"""A stack of gated layers, served: prompts in one pass, then token by token.

Every layer is a mixer between two 4-bit projections, with the norms around it:

    p      = W_in n                       (Q4: gate, channels, B, C and steps in one product)
    y      = mixer(p)                     (Ssm; or the relaxed long convolution, Lcsm, every ``conv_every``-th layer)
    r, n   = norm(W_out y, r)             (Q4, then Norm: norm after the block, scale, sum, norm before the next one)

and the next token's input is the last layer's n plus noise (the sampler of the synthetic models here).  Run

    python examples/gated_stack.py [--layers 8 --dim 768 --batch 4 --prompt 1024 --tokens 64 --conv-every 4]

for the time of a prompt and of a token, and a check that a prompt leaves what its tokens one by one leave.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_12982_amd.lcsm as lcsm  # noqa: E402


class GatedStack:
    """``layers`` layers of width ``dim`` for ``batch`` sequences of at most ``length`` tokens.  Heads of 64 channels (of
    ``dim / 12`` where that is less), inner width twice the width, ``states`` states, one group."""

    def __init__(self, layers, dim, batch, length, prompt, states=64, conv_every=0, dtype=torch.bfloat16, seed=0, device="cuda:0"):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=gen, device=device)  # noqa: E731
        P = min(64, dim // 12)
        H, G, N, W = 2 * dim // P, 1, states, 4
        D, C = H * P, H * P + 2 * G * N
        self.dim, self.batch, self.dtype, self.device, self.inner = dim, batch, dtype, torch.device(device), D
        self.D, self.C, self.H = D, C, H
        self.is_conv = [bool(conv_every) and m % conv_every == conv_every - 1 for m in range(layers)]

        def q4(n, k, gain=1.0):
            codes, scales = lcsm.Q4.quantize(rand(1, n, k) * (gain / math.sqrt(k)), 64, torch.float32 if dtype is torch.float32 else dtype)
            return lcsm.Q4(codes, scales, k, 64)

        self.w_in, self.w_out, self.conv, kinds = [], [], {}, []
        for m, conv in enumerate(self.is_conv):
            self.w_in.append(q4(dim if conv else D + C + H, dim))
            self.w_out.append(q4(dim, dim if conv else D, 0.5))
            if conv:  # one context a layer: a prompt's layers follow each other
                h = rand(1, dim, length) * torch.exp(-torch.arange(length, device=device) / (length / 8)) / math.sqrt(length / 16)
                self.conv[m] = lcsm.Lcsm(h, batch)
            else:
                kinds.append(m)
        self.ssm_layer = {m: i for i, m in enumerate(kinds)}
        M = max(len(kinds), 1)
        step = torch.exp(torch.rand((M, H), generator=gen, device=device) * math.log(100.0) + math.log(1e-3))
        self.ssm = lcsm.Ssm((torch.rand((M, C, W), generator=gen, device=device) * 2 - 1) / math.sqrt(W),
                            -(1 + 15 * torch.rand((M, H), generator=gen, device=device)), slots=batch, groups=G, states=N,
                            skip=torch.ones((M, H), device=device), dt_bias=step + torch.log(-torch.expm1(-step)), dtype=dtype,
                            max_tokens=batch * prompt)
        ones = torch.ones((layers, dim), device=device)
        self.norm = lcsm.Norm(dim, post="rms", pre="rms", post_weight=ones, pre_weight=ones, scale=0.5 * ones, dtype=dtype,
                              res_dtype=torch.float32)
        self.fresh = torch.full((batch,), -1, dtype=torch.int32, device=device)
        self.slots = torch.arange(batch, dtype=torch.int32, device=device)

    def reset(self):
        self.ssm.reset()
        for c in self.conv.values():
            c.reset()

    def _layers(self, x, mix):
        """The stack over rows x [rows, dim]; mix(m, p): layer m's mixer over its projected rows."""
        r = x.float()
        _, n = self.norm.block(0, None, r, res_out=False)
        for m in range(len(self.is_conv)):
            o = self.w_out[m].matvec(0, mix(m, self.w_in[m].matvec(0, n)))
            r, n = self.norm.block(m, o, r)
        return n

    def _split(self, p):
        return p[:, self.D:self.D + self.C], p[:, self.D + self.C:], p[:, :self.D]

    def prompt(self, x):
        """Rows of every sequence's prompt, x [batch, T, dim] (T a power of two where there are convolutions), from the
        beginning; the outputs, the same shape."""
        B, T, _ = x.shape
        offsets = torch.arange(0, (B + 1) * T, T, dtype=torch.int32, device=self.device)

        def mix(m, p):
            if m in self.conv:  # [T, 1, B, dim] fp32, a position after the other
                y = p.view(B, T, self.dim).transpose(0, 1).float().contiguous().unsqueeze(1)
                z = self.conv[m].prefill(y, torch.empty_like(y))
                return z.squeeze(1).transpose(0, 1).reshape(B * T, self.dim).to(self.dtype)
            xbc, dt, z = self._split(p)
            return self.ssm.prompt(self.ssm_layer[m], xbc, dt, z=z, offsets=offsets, src=self.fresh, dst=self.slots)

        return self._layers(x.reshape(B * T, self.dim), mix).view(B, T, self.dim)

    def step(self, x):
        """One token of every sequence, x [batch, dim]."""
        def mix(m, p):
            if m in self.conv:
                return self.conv[m].step(p.float().view(1, self.batch, self.dim))[0].to(self.dtype)
            xbc, dt, z = self._split(p)
            return self.ssm.step(self.ssm_layer[m], xbc, dt, z=z)

        return self._layers(x, mix)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("layers", 8), ("dim", 768), ("batch", 4), ("prompt", 1024), ("tokens", 64), ("conv-every", 4)):
        ap.add_argument(f"--{name}", type=int, default=default)
    a = ap.parse_args()
    stack = GatedStack(a.layers, a.dim, a.batch, 2 * a.prompt + a.tokens, a.prompt, conv_every=a.conv_every)
    x = torch.randn((a.batch, a.prompt, a.dim), device="cuda:0").to(stack.dtype)
    stack.prompt(x)
    stack.reset()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    y = stack.prompt(x)[:, -1]
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    for _ in range(a.tokens):
        y = stack.step(y + 0.1 * torch.randn_like(y))
    torch.cuda.synchronize()
    t2 = time.perf_counter()
    print(f"{a.layers} layers of {a.dim}, batch {a.batch}: prompt of {a.prompt} {1e3 * (t1 - t0):.2f} ms, "
          f"a token {1e6 * (t2 - t1) / max(a.tokens, 1):.0f} us")
    short = min(a.prompt, 64)
    stack.reset()
    whole = stack.prompt(x[:, :short].contiguous())
    stack.reset()
    single = torch.stack([stack.step(x[:, t].contiguous()) for t in range(short)], 1)
    err = ((whole - single).float().norm() / single.float().norm()).item()
    print(f"a prompt of {short} against its tokens one by one: {err:.1e}")
    return 0 if err < 0.05 else 1


if __name__ == "__main__":
    sys.exit(main())
