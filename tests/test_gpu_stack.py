"""The gated layer's operators together with the long convolution, as the example
serves them (needs an MI355X): a prompt in one pass and its tokens one by one
leave the same outputs and go on alike.

fp32 throughout: the two ways differ by roundings of the sums, 2e-5 of the
largest value an operator (the mixer's bound), which the layers hand on: each
normed, so that they add up: 2e-5 times six operators a layer."""
import os
import sys

import pytest
import torch

from gpu_harness import dev

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("layers,dim,batch,T,states,conv_every", [(4, 96, 3, 64, 20, 2), (3, 192, 2, 256, 64, 0), (2, 768, 1, 512, 128, 2)])
def test_prompt_and_tokens_agree(layers, dim, batch, T, states, conv_every):
    from gated_stack import GatedStack
    stack = GatedStack(layers, dim, batch, 2 * T + 8, T, states=states, conv_every=conv_every, dtype=torch.float32, seed=layers)
    g = torch.Generator(device=dev())
    g.manual_seed(1)
    x = torch.randn((batch, T + 3, dim), generator=g, device=dev())
    whole = [stack.prompt(x[:, :T].contiguous())] + [stack.step(x[:, T + k].contiguous()).unsqueeze(1) for k in range(3)]
    stack.reset()
    single = torch.stack([stack.step(x[:, t].contiguous()) for t in range(T + 3)], 1)
    whole = torch.cat(whole, 1)
    assert torch.isfinite(single).all()
    err = ((whole - single).abs().max() / single.abs().max()).item()
    assert err <= 2e-5 * 6 * layers, err
