"""Linear attention layers as they are served (needs an MI355X): an 8-bit product
for queries, keys, values and gate, norms and rotation in place in its rows,
attention, the gated norm of each head, and an 8-bit product; prompts, tokens, and
tokens recorded into a graph.

Every operator is checked on what it was in fact given, by the bounds of its own
tests: an 8-bit product by five roundings of 2^-24 of its sum and half an ulp; the
rotation by 2e-6 of its row's largest value and half an ulp; attention by 2e-5 (and
2^-15 where outputs have 16 bits) of the magnitudes it sums and half an ulp."""
import os
import sys

import numpy as np
import pytest
import torch

from gpu_harness import dev, lcsm_mod, say
from oracle import lin as oracle

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 1e-38, "bf16": 1e-38, "f16": 2.0 ** -25}


def near(got, want, room, what):
    off = np.abs(got.double().cpu().numpy() - want) - room
    assert off.max(initial=-1.0) <= 0, (what, float(off.max()))


class Served:
    """One layer of width D: H heads of queries on G states of K keys and V values."""

    def __init__(self, D, H, G, K, V, dtype, slots, max_tokens, seed=0):
        lcsm, r = lcsm_mod(), np.random.default_rng(seed)
        self.D, self.H, self.G, self.K, self.V, self.dtype, self.rng = D, H, G, K, V, dtype, r
        self.widths = [H * V, H * K, G * K, G * V]
        up = lambda a, t=np.float32: torch.from_numpy(np.ascontiguousarray(a, t)).to(dev())  # noqa: E731
        self.weights = []
        for n, k in ((sum(self.widths), D), (D, H * V)):
            codes, scales = lcsm.Q8.quantize(up(r.standard_normal((1, n, k)) / np.sqrt(k)))
            self.weights.append((lcsm.Q8(codes, scales, max(max_tokens, slots)), codes[0].cpu().numpy(), scales[0].cpu().numpy()))
        self.decay = -np.exp2(-1 - 6 * r.random((1, G))).astype(np.float32)
        self.lin = lcsm.Lin(up(self.decay), slots=slots, heads=H, keys=K, values=V, scale=K ** -0.5, dtype=TYPES[dtype],
                            max_tokens=max_tokens)
        self.w = (1 + 0.1 * r.standard_normal((2, 1, K))).astype(np.float32)
        self.rot = lcsm.Rot(K, H, G, q_weight=up(self.w[0]), k_weight=up(self.w[1]), dtype=TYPES[dtype])
        self.freqs = np.array([10000.0 ** (-2.0 * j / (K // 2 * 2)) for j in range(K // 2)])
        self.norm = lcsm.Norm(H * V, post="rms", pre="none", act="silu", groups=H, alpha=0.0, dtype=TYPES[dtype], device=dev())

    def __call__(self, x, positions, attend):
        """The layer's rows; what the operators were given and gave is kept."""
        p = self.weights[0][0].matmul(0, x)
        self.projected = p.clone()
        z, q, k, v = p.split(self.widths, 1)
        self.rot.apply(0, q, k, positions, q_out=q, k_out=k)
        y = attend(0, q, k, v)
        n = self.norm.block(0, y, y, gate=z, res_out=False)[1]
        self.turned, self.y, self.n = p, y, n
        return self.weights[1][0].matmul(0, n)

    def check(self, x, out, positions, offsets, states, after):
        """states: the sequences' states before the call, after: those after it, both [n, G, K, V] on the host."""
        e, tiny = ULP[self.dtype], TINY[self.dtype]
        for (_, codes, scales), a, b in zip(self.weights, (x, self.n), (self.projected, out)):
            want, size = oracle.q8(a.double().cpu().numpy(), codes, scales, None)
            near(b, want, e * np.abs(want) + 5 * 2.0 ** -24 * size + tiny, "8-bit product")
        q0, k0 = self.projected.split(self.widths, 1)[1:3]
        z, q, k, v = self.turned.split(self.widths, 1)
        for a, b, w in ((q0, q, self.w[0]), (k0, k, self.w[1])):
            want = oracle.heads(a.double().cpu().numpy(), self.K, "rms", w[0], np.float32(1e-5), positions, self.freqs, "half")
            near(b, want, (2e-6 + e) * np.abs(want).max(1, keepdims=True) + tiny, "rotation")
        heads = [a.double().cpu().numpy().reshape(len(a), n, -1) for a, n in ((q, self.H), (k, self.G), (v, self.G))]
        lost, scale = 2e-5 + (0.0 if self.dtype == "f32" else 2.0 ** -15), np.float32(self.K ** -0.5)
        y = self.y.view(len(x), self.H, self.V)
        for i, (a, b) in enumerate(zip(offsets, offsets[1:])):
            want, S = oracle.attend(*(t[a:b] for t in heads), self.decay[0], scale, states[i])
            big, Z = oracle.attend(*(np.abs(t[a:b]) for t in heads), self.decay[0], scale, np.abs(states[i]))
            near(y[a:b], want, e * np.abs(want) + lost * big + tiny, "attention")
            near(after[i], S, 2e-5 * Z, "state")
        g, o = z.double().cpu().numpy(), self.y.double().cpu().numpy()
        t = (o * g / (1 + np.exp(-g))).reshape(len(o), self.H, self.V)
        want = (t / np.sqrt((t * t).mean(-1, keepdims=True) + 1e-5)).reshape(o.shape)
        # (the norm: two dozen roundings of 2^-24 of each value, the gate's exponential among them)
        near(self.n, want, (e + 2e-6) * np.abs(want) + tiny, "gated norm")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,H,G,K,V", [(96, 3, 3, 32, 64), (130, 6, 2, 24, 40), (256, 4, 1, 128, 136), (64, 2, 2, 7, 9)])
def test_layer(D, H, G, K, V, dtype):
    """Ragged prompts, an empty one among them, and tokens after them, four sequences in slots of their own."""
    offs, slots = [0, 70, 70, 71, 300], 5
    s = Served(D, H, G, K, V, dtype, slots, offs[-1], seed=D)
    make = lambda n: torch.from_numpy(s.rng.standard_normal((n, D)).astype(np.float32)).to(TYPES[dtype]).to(dev())  # noqa: E731
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device=dev())  # noqa: E731
    at = [3, 0, 4, 1]
    src, dst, offsets = ints([-1] * 4), ints(at), ints(offs)
    pos = np.concatenate([np.arange(b - a) for a, b in zip(offs, offs[1:])]).astype(np.int32)
    say(f"[layer] prompts {D} {H} {G} {K} {V} {dtype}")
    x = make(offs[-1])
    out = s(x, ints(pos.tolist()), lambda m, q, k, v: s.lin.prompt(m, q, k, v, offsets=offsets, src=src, dst=dst))
    after = s.lin.state(0)[at].cpu()
    s.check(x, out, pos, offs, np.zeros((4, G, K, V)), after)
    for step in range(2):
        say(f"[layer] token {step}")
        before, x = after.double().numpy(), make(4)
        pos = np.array([b - a + step for a, b in zip(offs, offs[1:])], np.int32)
        out = s(x, ints(pos.tolist()), lambda m, q, k, v: s.lin.step(m, q, k, v, src=dst, dst=dst))
        after = s.lin.state(0)[at].cpu()
        s.check(x, out, pos, [0, 1, 2, 3, 4], before, after)


def test_tokens_in_a_graph():
    """A token recorded once and replayed, with eager tokens of the same layer between the replays: the same bits."""
    s = Served(192, 6, 3, 32, 48, "bf16", 3, 64, seed=7)
    xs = [torch.from_numpy(s.rng.standard_normal((3, 192)).astype(np.float32)).bfloat16().to(dev()) for _ in range(8)]
    x, positions = torch.zeros_like(xs[0]), torch.zeros(3, dtype=torch.int32, device=dev())

    def token():
        y = s(x, positions, s.lin.step)
        positions.add_(1)
        return y

    def eager():
        s.lin.reset()
        positions.zero_()
        out = []
        for t in xs:
            x.copy_(t)
            out.append(token().clone())
        return out, s.lin.state(0).clone()

    want, state = eager()
    say("[layer] capture")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # contexts belong to a stream: another set of them on this one
        s = Served(192, 6, 3, 32, 48, "bf16", 3, 64, seed=7)
        token()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y = token()
        s.lin.reset()
        positions.zero_()
        for i, t in enumerate(xs):
            x.copy_(t)
            if i % 3 == 2:
                got = token()
            else:
                graph.replay()
                got = y
            side.synchronize()
            assert torch.equal(got, want[i]), i
        assert torch.equal(s.lin.state(0), state)


@pytest.mark.parametrize("layers,dim,batch,T,conv_every,lin_every,dtype", [(4, 96, 3, 64, 4, 2, "f32"), (3, 192, 2, 100, 0, 1, "bf16"),
                                                                           (5, 768, 1, 256, 2, 3, "bf16")])
def test_stack(layers, dim, batch, T, conv_every, lin_every, dtype):
    """The example's stack with such layers runs: a prompt in one pass and its tokens one by one.  Both round their rows to
    8 bits, a step of a 127th of the largest of them, some four times a row's root mean square: 0.9 % of a row's norm each
    time.  Were all roundings of the two ways independent, two of a layer's would make 1.8 % of what the layer adds, half a
    norm: less than 5 % of the outputs after the few layers here."""
    from gated_stack import GatedStack
    stack = GatedStack(layers, dim, batch, 2 * T + 8, T, states=16, conv_every=conv_every, dtype=TYPES[dtype], seed=layers,
                       lin_every=lin_every)
    g = torch.Generator(device=dev())
    g.manual_seed(1)
    x = torch.randn((batch, T + 3, dim), generator=g, device=dev()).to(TYPES[dtype])
    say("[stack] prompt")
    whole = [stack.prompt(x[:, :T].contiguous())] + [stack.step(x[:, T + k].contiguous()).unsqueeze(1) for k in range(3)]
    stack.reset()
    single = torch.stack([stack.step(x[:, t].contiguous()) for t in range(T + 3)], 1).double()
    whole = torch.cat(whole, 1).double()
    assert torch.isfinite(single).all()
    assert ((whole - single).norm() / single.norm()).item() < 0.05


def test_no_rows():
    """Calls without rows give outputs without rows and leave the states as they are; a sequence of none moves its state."""
    s = Served(64, 4, 2, 16, 24, "bf16", 3, 32, seed=3)
    s.lin.state(0).copy_(torch.randn(s.lin.state(0).shape, device=dev()))
    state = s.lin.state(0).clone()
    x, none = torch.empty((0, 64), dtype=torch.bfloat16, device=dev()), torch.empty(0, dtype=torch.int32, device=dev())
    assert s(x, none, s.lin.step).shape == (0, 64)
    assert s(x, none, lambda m, q, k, v: s.lin.prompt(m, q, k, v, src=torch.tensor([2], dtype=torch.int32, device=dev()),
                                                      dst=torch.tensor([0], dtype=torch.int32, device=dev()))).shape == (0, 64)
    assert torch.equal(s.lin.state(0)[1:], state[1:]) and torch.equal(s.lin.state(0)[0], state[2])
