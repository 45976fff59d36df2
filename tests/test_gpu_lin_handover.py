"""The example's stack with linear attention layers: what a prompt hands on to the
tokens after it (needs an MI355X).

A prompt and its tokens one by one round the same rows to 8 bits, 0.9 % of a row's
norm each time, but not the same way where they differ by their sums' order.  Were
all roundings independent, the rows' 1.3 % on the way into a layer would reach gate,
queries, keys and values, and 1.3 % more come on the way out: 3 % of what the layer
adds, half a norm.  Two layers of that are 2.1 % of a token's outputs, and what the
second makes of the first one's less than one more: below 5 % for every token.  A
state is a sum over tokens of keys and values that are off by 1.3 % each: 5 % too."""
import os
import sys

import pytest
import torch

from gpu_harness import dev, say

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def off(got, want, keep):
    """The largest share of its norm that a part of `want` (along its first `keep` dimensions) is off by."""
    got, want = got.double().flatten(keep), want.double().flatten(keep)
    return ((got - want).norm(dim=-1) / want.norm(dim=-1)).max().item()


@pytest.mark.parametrize("layers,dim,T,conv_every,lin_every,dtype", [
    (2, 192, 100, 0, 1, torch.float32), (2, 192, 256, 0, 1, torch.bfloat16), (4, 96, 64, 4, 2, torch.float32)])
def test_tokens_after_a_prompt(layers, dim, T, conv_every, lin_every, dtype):
    from gated_stack import GatedStack
    batch, more = 3, 5
    stack = GatedStack(layers, dim, batch, 2 * T + more, T, states=16, conv_every=conv_every, dtype=dtype, seed=layers,
                       lin_every=lin_every)
    g = torch.Generator(device=dev())
    g.manual_seed(2)
    x = torch.randn((batch, T + more, dim), generator=g, device=dev()).to(dtype)
    lins = range(len(stack.lin_layer))

    def seen():
        return stack.positions.tolist(), [stack.lin.state(i)[:batch].clone() for i in lins]

    def tokens(a, b):
        return torch.stack([stack.step(x[:, t].contiguous()) for t in range(a, b)], 1)

    say("[stack] prompt, then tokens")
    prompt = stack.prompt(x[:, :T].contiguous())
    handed = seen()
    after = tokens(T, T + more)
    end = seen()
    stack.reset()
    say("[stack] tokens")
    single = tokens(0, T)
    single_handed = seen()
    single_after = tokens(T, T + more)
    single_end = seen()
    torch.cuda.synchronize()
    assert handed[0] == single_handed[0] == [T] * batch and end[0] == single_end[0] == [T + more] * batch
    for ways in ((handed[1], single_handed[1]), (end[1], single_end[1])):
        for i, (a, b) in enumerate(zip(*ways)):
            say(f"[stack] layer {i}: states off by {off(a, b, 1):.4f}")
            assert off(a, b, 1) < 0.05
    for name, a, b in (("prompt", prompt, single), ("after it", after, single_after)):
        a, b = a.transpose(0, 1), b.transpose(0, 1)  # a token of all sequences
        say(f"[stack] {name}: tokens off by up to {off(a, b, 1):.4f}")
        assert off(a, b, 1) < 0.05, name
