"""The token model of examples/ around the gated delta rule: layer norms, the delta rule, the head, log probabilities and the check of drafts in one run.

Tolerances.  In fp32 a gradient is a chain of some 28 sums (norms, projections, attention, head, and back) over at most 60 numbers or tokens and 50 vocabulary entries, whose relative
errors (about sqrt(60) 2^-24 = 5e-7 each) add up to 1.4e-5 in the 2-norm: 5e-5.  A rate's gradient is a sum over the tokens behind it of terms of either sign, which
may leave an eighth of what they are: 4e-4 for the weights that the rates come from.
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
    """The same model in plain 64-bit operations on the CPU, token by token."""
    h, d = model.heads, model.dim
    x = W["embedding"][tokens]

    def norm(t):
        t = t - t.mean(-1, keepdim=True)
        return t / torch.sqrt(t.square().mean(-1, keepdim=True) + 1e-5)
    normed = norm(x) * W["norm"] + W["norm_bias"]
    q, k, v = (normed @ W["qkv"]).view(-1, 3, h, d).unbind(1)
    angle = positions.double()[:, None] * model.frequencies.double().cpu()
    c, s = torch.cos(angle)[:, None] * model.magnitude, torch.sin(angle)[:, None] * model.magnitude

    def turn(t):
        u, w = t[..., :d // 2], t[..., d // 2:]
        return torch.cat([u * c - w * s, w * c + u * s], -1)
    q, k = turn(norm(q) * d ** -0.5), turn(norm(k) * d ** -0.5)
    small = normed @ W["small"]
    decay, beta = torch.exp(-model.rates.double().cpu() * torch.exp(small[:, :h])), torch.sigmoid(small[:, h:])
    outs = []
    for a, z in zip(starts[:-1], starts[1:]):
        state = torch.zeros(h, d, d, dtype=torch.float64)
        for t in range(a, z):
            state = decay[t][:, None, None] * state
            u = beta[t][:, None] * (v[t] - (state * k[t][:, :, None]).sum(1))
            state = state + k[t][:, :, None] * u[:, None, :]
            outs.append((state * q[t][:, :, None]).sum(1))
    hidden = x + torch.stack(outs).reshape(x.shape) @ W["out"]
    kernel = torch.exp(-(W["a"][:, :, None] - W["b"][:, None, :]).abs())
    logits = torch.einsum("q,qij,tj->ti", W["w"], kernel, hidden)
    logp = torch.log_softmax(logits, -1)
    given = targets >= 0
    entropy = -(logp.exp() * logp).sum(-1)
    return -((logp.gather(1, targets.clamp(min=0)[:, None])[:, 0] + bonus * entropy)[given]).mean()


def test_gradients_of_the_model(example):
    model = example.DeltaTokenModel(50, 32, 2, operators=3)
    gen = torch.Generator().manual_seed(3)
    tokens, targets = torch.randint(0, 50, (60,), generator=gen), torch.randint(0, 50, (60,), generator=gen)
    targets[22] = -1
    positions, starts = torch.cat([torch.arange(23), torch.arange(37)]), torch.tensor([0, 23, 60])
    loss, grads = model.gradients(tokens.cuda(), positions.cuda(), targets.cuda(), starts.cuda(), 0.1)
    W = {n: t.double().cpu().requires_grad_() for n, t in model.weights.items()}
    want = plain_loss(model, W, tokens, positions, targets, starts.tolist(), 0.1)
    want.backward()
    assert abs(float(loss) - want.item()) < 2e-5 * abs(want.item())
    assert set(grads) == set(W)
    for name, t in W.items():
        off = (grads[name].double().cpu() - t.grad).norm() / t.grad.norm()
        assert float(off) < (4e-4 if name == "small" else 5e-5), f"{name}: {float(off):.2e}"


def test_drafts_checked_at_once_are_what_is_written_one_by_one(example):
    """Sequences whose drafts are right, wrong from the third on, and wrong at once: as many are kept, the next token is what writing gives, and the state that of the
    tokens that were kept."""
    model = example.DeltaTokenModel(300, 64, 4)
    lengths, columns = [40, 17, 90], 6
    starts = torch.tensor([0] + lengths).cumsum(0).cuda()
    tokens = example.text(300, sum(lengths))
    positions = torch.cat([torch.arange(n) for n in lengths]).cuda()
    state = model.new_state(3)
    _, _, ids, _ = model.read(tokens, positions, starts, state, top=1)
    current = ids[0, starts[1:] - 1]
    at = torch.tensor(lengths, device="cuda")
    chain, states, one_by_one = [current], [], state.clone()
    for i in range(columns):
        ids, alternatives, _ = model.write(chain[-1], at + i, one_by_one, top=2)
        # fp32 sums in another order move logits by 1e-5 of their size at most: the likeliest token is the same either way
        assert float((alternatives[0] - alternatives[1]).min()) > 1e-3
        states.append(one_by_one.clone())
        chain.append(ids[0])
    drafted = torch.stack(chain[:columns], 1)
    drafted[1, 3] = (drafted[1, 3] + 1) % 300
    drafted[2, 1] = (drafted[2, 1] + 1) % 300
    accepted, following = model.check(drafted, at[:, None] + torch.arange(columns, device="cuda"), state, drafted.roll(-1, 1))
    assert accepted.tolist() == [5, 2, 0]
    assert following.tolist() == [int(chain[a + 1][b]) for b, a in enumerate(accepted.tolist())]
    for b, a in enumerate(accepted.tolist()):
        assert float((state[b] - states[a][b]).norm() / states[a][b].norm()) < 1e-5


def test_drawn_tokens_have_the_models_distribution(example):
    """With drafts that are certain the first token is the draft where its chance is below its probability, and else one drawn from the rest: over equally
    spaced chances of either kind the frequencies are the probabilities, to the spacing."""
    model = example.DeltaTokenModel(30, 32, 2)
    prompt, positions = example.text(30, 20), torch.arange(20, device="cuda")
    state = model.new_state(1)
    _, _, ids, _ = model.read(prompt, positions, state=state, top=2)
    last = ids[0, -1]
    n = 64
    grid = (torch.arange(n, device="cuda").double() + 0.5) / n
    many = state.expand(n * n, -1, -1, -1).contiguous()
    draft = ids[1, -1]
    tokens = torch.stack([last, draft]).expand(n * n, 2).contiguous()
    drafts = torch.stack([draft, draft]).expand(n * n, 2).contiguous()
    chances = grid.repeat_interleave(n)[:, None].expand(n * n, 2).flatten().contiguous()
    accepted, following = model.check(tokens, torch.tensor([20, 21], device="cuda").expand(n * n, 2), many, drafts, chances, grid.repeat(n))
    first = torch.where(accepted > 0, draft, following)
    _, _, likeliest, logp = model.read(last[None], torch.tensor([20], device="cuda"), state=state.clone(), top=30)
    p = torch.zeros(30, device="cuda", dtype=torch.float64)
    p[likeliest[:, 0]] = logp[:, 0].double().exp()
    # of n equally spaced chances p(draft) n are below it, to one half; of those behind that draw a row has its share of n to one: 1.5 / n of all at most
    assert float((torch.bincount(first, minlength=30) / n ** 2 - p).abs().max()) < 2.0 / n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_commands_run(example, dtype, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["token_model.py", "--delta", "--steps", "2", "--length", "100", "--dtype", dtype])
    example.main()
    assert "drafts kept" in capsys.readouterr().out
