"""The example that trains and decodes blocks made of linear attention and the block norms."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "linear_block.py")
    spec = importlib.util.spec_from_file_location("linear_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_training_lowers_the_loss(example):
    print("training 30 steps", flush=True)
    _, losses = example.train(steps=30)
    # a model that learns nothing stays at the entropy of 32 symbols, 3.47, or above it
    assert all(x == x for x in losses)
    assert sum(losses[-5:]) < sum(losses[:5])


@pytest.mark.parametrize("prompt", [1, 63, 64, 100])
def test_decoding_agrees_with_the_chunk_call(example, prompt):
    print(f"decoding after a prompt of {prompt}", flush=True)
    torch.manual_seed(1)
    model = example.Model().to("cuda")
    tokens = torch.randint(0, 32, (3, 130), device="cuda")
    with torch.no_grad():
        whole, _ = model(tokens)
    apart = example.decode(model, tokens, prompt)
    # both round the same eleven values to bfloat16 on their way (two blocks of projections, o, a,
    # y, n; the logits), each by 2^-9 relative at most in the mean square: sqrt(11) 2^-9 = 6.5e-3
    # if every rounding fell differently
    assert float((apart - whole).norm() / whole.norm()) < 6.5e-3


def test_gradients_follow_differences(example):
    """One step against the gradient lowers the loss by |gradient|^2 times its length, to first order."""
    torch.manual_seed(2)
    model = example.Model(blocks=1).to("cuda")
    tokens = torch.randint(0, 32, (2, 200), device="cuda")

    def loss():
        logits, _ = model(tokens[:, :-1])
        return torch.nn.functional.cross_entropy(logits.reshape(-1, 32), tokens[:, 1:].reshape(-1))

    a = loss()
    a.backward()
    size = sum(float((p.grad.double() ** 2).sum()) for p in model.parameters())
    step = 0.05 * float(a.detach()) / size  # a predicted fall of 5 %: well over bfloat16's 0.4 %, small beside curvature
    with torch.no_grad():
        for p in model.parameters():
            p -= step * p.grad
        b = loss()
    fall = (float(a.detach()) - float(b)) / (step * size)
    assert 0.5 < fall < 1.5, fall


def test_a_second_derivative_is_refused(example):
    """A penalty on a gradient raises instead of leaving out what goes through the operators."""
    print("second derivatives", flush=True)
    q, k, v, z = (torch.randn(1, 20, 2, 64, device="cuda").to(torch.bfloat16).requires_grad_(True) for _ in range(4))
    w = torch.ones(64, device="cuda", requires_grad=True)
    o, _ = example.Attention.apply(q, k, v, -torch.rand(1, 20, 2, device="cuda"), None)
    a, _ = example.BlockNorm.apply(v, w, z, None, None, None)
    for y, x in ((o, q), (a, v)):
        with pytest.raises(RuntimeError, match="second derivative"):
            d, = torch.autograd.grad(y.float().sum(), x, create_graph=True)
            (x.float() ** 2 + d.float() ** 2).sum().backward()
