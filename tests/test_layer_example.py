"""The example of a layer built from the operators: its gradient, its training and its single tokens."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_delta_layer.py")
    spec = importlib.util.spec_from_file_location("gated_delta_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradient_of_the_delta_rule(example):
    """Against autograd through the recursion token by token in 64 bits.  U, W, O and each gradient end in bf16 (2^-9 of a value each), and a gradient is the sum of
    two such (through the attention and through the inverse): 2^-9 times the root of the roundings in a row, six at most, taken twice; 2^-6 bounds it."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    B, T, H, d = 2, 128, 2, 64
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    unit = lambda x: torch.nn.functional.normalize(x, dim=-1).bfloat16()
    q, k, v = unit(rand(B, T, H, d)), unit(rand(B, T, H, d)), rand(B, T, H, d).bfloat16()
    beta, r = torch.sigmoid(rand(B, T, H)), -torch.nn.functional.softplus(rand(B, T, H) - 3)
    dO = rand(B, T, H, d).bfloat16()
    mine = [x.clone().requires_grad_() for x in (q, k, v, beta, r)]
    example.Delta.apply(*mine[:4], example.local(mine[4])).backward(dO)
    exact = [x.double().cpu().requires_grad_() for x in (q, k, v, beta, r)]
    S, out = torch.zeros(B, H, d, d, dtype=torch.float64), []
    for t in range(T):
        qt, kt, vt, bt, rt = (x[:, t] for x in exact)
        S = S * rt.exp()[..., None, None]
        S = S + (bt[..., None] * kt)[..., :, None] * (vt - (S * kt[..., :, None]).sum(-2))[..., None, :]
        out.append(d ** -0.5 * (S * qt[..., :, None]).sum(-2))
    torch.stack(out, 1).backward(dO.double().cpu())
    for name, a, b in zip("q k v beta r".split(), mine, exact):
        got, want = a.grad.double().cpu(), b.grad
        assert (got - want).norm() <= 2.0 ** -6 * want.norm(), name


def test_training_lowers_the_loss(example):
    torch.manual_seed(0)
    losses = example.train(example.Layer(256, 4))
    assert losses[-1] < 0.9 * losses[0]


def test_tokens_one_by_one_are_the_prompt(example):
    """Both end in bf16 behind bf16 factors: U, W, O, the projection (2^-9 each, the relative distance of a token's 256 outputs), on both sides; 2^-6 bounds it."""
    torch.manual_seed(0)
    assert example.answer(example.Layer(256, 4)) <= 2.0 ** -6
