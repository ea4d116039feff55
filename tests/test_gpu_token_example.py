"""The token model of examples/: its gradients against automatic differentiation of the same model in 64 bits, and its two
ways of reading a text (at once, and token by token) against each other.

Tolerance of the gradients: every one is a chain of six products over at most 60 numbers or tokens and 50 vocabulary
entries in fp32, whose relative errors (about sqrt(60) 2^-24 = 5e-7 each) add up to about 3e-6 in the 2-norm: 2e-5.
"""
import importlib.util
import os

import pytest

from conftest import ROOT

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("token_model", os.path.join(ROOT, "examples", "token_model.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_loss(model, W, tokens, positions, targets, starts, bonus):
    """The same model in plain 64-bit operations on the CPU."""
    h, d = model.heads, model.dim
    x = W["embedding"][tokens]
    q, k, v = (x @ W["qkv"]).view(-1, 3, h, d).unbind(1)
    angle = positions.double()[:, None] * model.frequencies.double().cpu()
    c, s = torch.cos(angle)[:, None] * model.magnitude, torch.sin(angle)[:, None] * model.magnitude

    def turn(t):
        u, w = t[..., :d // 2], t[..., d // 2:]
        return torch.cat([u * c - w * s, w * c + u * s], -1)
    q, k = turn(q), turn(k)
    rates = model.rates.double().cpu()
    outs = []
    for a, z in zip(starts[:-1], starts[1:]):
        t = torch.arange(z - a).double()
        weight = torch.exp(-rates[:, None, None] * (t[:, None] - t)).tril()
        map_ = model.scale * torch.einsum("thd,shd->hts", q[a:z], k[a:z]) * weight
        outs.append(torch.einsum("hts,shd->thd", map_, v[a:z]))
    hidden = x + torch.cat(outs).reshape(x.shape) @ W["out"]
    kernel = torch.exp(-(W["a"][:, :, None] - W["b"][:, None, :]).abs())
    logits = torch.einsum("q,qij,tj->ti", W["w"], kernel, hidden)
    logp = torch.log_softmax(logits, -1)
    given = targets >= 0
    entropy = -(logp.exp() * logp).sum(-1)
    return -((logp.gather(1, targets.clamp(min=0)[:, None])[:, 0] + bonus * entropy)[given]).mean()


def inputs(vocabulary, n, cut, seed=3):
    gen = torch.Generator().manual_seed(seed)
    tokens = torch.randint(0, vocabulary, (n,), generator=gen)
    targets = torch.randint(0, vocabulary, (n,), generator=gen)
    targets[cut - 1] = -1
    positions = torch.cat([torch.arange(cut), torch.arange(n - cut)])
    return tokens, positions, targets, torch.tensor([0, cut, n])


def test_gradients_of_the_model(example):
    model = example.TokenModel(50, 32, 2, operators=3, stretch=4.0, context=64)
    tokens, positions, targets, starts = inputs(50, 60, 23)
    loss, grads = model.gradients(tokens.cuda(), positions.cuda(), targets.cuda(), starts.cuda(), 0.1)
    W = {n: t.double().cpu().requires_grad_() for n, t in model.weights.items()}
    want = plain_loss(model, W, tokens, positions, targets, starts.tolist(), 0.1)
    want.backward()
    assert abs(float(loss) - want.item()) < 2e-5 * abs(want.item())
    for name, t in W.items():
        off = (grads[name].double().cpu() - t.grad).norm() / t.grad.norm()
        assert float(off) < 2e-5, f"{name}: {float(off):.2e}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_reading_at_once_and_token_by_token_agree(example, dtype):
    """After a prompt at once and after the same tokens one by one the state and the next token's alternatives agree."""
    model = example.TokenModel(300, 64, 4, dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    tokens = example.text(300, 90)
    positions = torch.arange(90, device="cuda")
    at_once, one_by_one = model.new_state(1), model.new_state(1)
    _, entropy, ids, alternatives = model.read(tokens, positions, state=at_once, top=4)
    for t in range(90):
        last = model.write(tokens[t:t + 1], positions[t:t + 1], one_by_one, top=4)
    # fp32: the states are sums of the same products in either order.  bf16: keys and values are the projection's results (a matrix product of 90 rows, and of
    # one) rounded to 8 bits, and either factor may have been rounded the other way
    assert float((at_once - one_by_one).norm() / at_once.norm()) < (1e-5 if dtype == "f32" else 2 * 2.0 ** -8)
    # bf16: the attention's results are rounded to 8 bits, and in the prompt its map and state as well
    bound = 1e-4 if dtype == "f32" else 2.0 ** -6 * float(alternatives.abs().max())
    assert float((alternatives[:, -1] - last[1][:, 0]).abs().max()) < bound
    if dtype == "f32":
        assert torch.equal(ids[:, -1], last[0][:, 0])


def test_training_lowers_the_loss(example):
    model = example.TokenModel(100, 64, 2, dtype=torch.bfloat16)
    tokens = example.text(100, 201)
    positions = torch.arange(200, device="cuda")
    losses = []
    for _ in range(15):
        loss, g = model.gradients(tokens[:-1], positions, tokens[1:])
        size = torch.sqrt(sum(t.square().sum() for t in g.values()))
        model.step(g, 1.0 / max(1.0, float(size)))
        losses.append(float(loss))
    assert losses[-1] < 0.8 * losses[0], losses
