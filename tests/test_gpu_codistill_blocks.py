"""Training of residual blocks end to end: the operators together, the gradient of a round against autograd in 64 bits, generation that
continues what the whole-sequence forward pass says."""
import math

import pytest
import torch

import lm_block_reference as BR
from paper_2012_15198_amd import codistill

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


def reference_loss(model, x, tokens, labels, reset, teacher, tau, w_kl, w_ce):
    """The model in plain 64-bit operations, step by step: sum over workers of the mean loss."""
    W, V, D, T, K, N = model.W, model.V, model.D, reset.shape[1], model.K, model.S_
    n = tokens.shape[1]
    ids, t = teacher
    masks = [BR.factor(pair, W * n, D, model.p) for pair in model.rng.tolist()]
    fresh = (reset != 0).view(W, -1, T)
    norm = lambda s, w: s / (s.square().mean(1, keepdim=True) + model.EPS).sqrt() * w
    total = 0
    for w in range(W):
        rows, own = slice(w * n, (w + 1) * n), lambda at, *shape: x[w, at:at + math.prod(shape)].view(*shape)
        table = own(0, V, D)
        add, s = table[tokens[w].long()] * math.sqrt(D), 0
        for k, place in enumerate(model.at):
            s = s + add * masks[k][rows]
            into = norm(s, own(place["norm"], D)) @ own(place["into"], D, 2 * D)
            a, z = into[:, :D].reshape(-1, T, D), into[:, D:].reshape(-1, T, D)
            taps, bias = own(place["conv"], D, K), own(place["conv"] + D * K, D)
            seen, u = [torch.zeros_like(a[:, 0])] * (K - 1), []
            for i in range(T):
                seen = [torch.where(fresh[w, :, i, None], torch.zeros_like(v), v) for v in seen[-(K - 1):]] + [a[:, i]]
                v = bias + sum(taps[:, j] * seen[j] for j in range(K))
                u.append(v * torch.sigmoid(v))
            u = torch.stack(u, 1)
            steps = u @ own(place["steps"], D, D + 2 * N)
            rate, first, skip = own(place["scan"], D, N).exp(), own(place["scan"] + D * N, D), own(place["scan"] + D * (N + 1), D)
            h, ys = torch.zeros((u.shape[0], D, N), dtype=x.dtype), []
            for i in range(T):
                delta = torch.nn.functional.softplus(steps[:, i, :D] + first)
                h = (-delta[..., None] * rate).exp() * h * (~fresh[w, :, i]).to(x.dtype)[:, None, None]
                h = h + (delta * u[:, i])[..., None] * steps[:, i, None, D:D + N]
                ys.append(((h * steps[:, i, None, D + N:]).sum(2) + skip * u[:, i]) * z[:, i] * torch.sigmoid(z[:, i]))
            add = torch.stack(ys, 1).reshape(n, D) @ own(place["back"], D, D)
        y = norm(s + add * masks[model.blocks][rows], own(model.norm, D)) * masks[model.blocks + 1][rows]
        logits = y / math.sqrt(D) @ table.t()
        log_q = torch.log_softmax(t[rows].to(x.dtype) / tau, 1)
        kl = (log_q.exp() * (log_q - torch.log_softmax(logits / tau, 1).gather(1, ids[rows].long()))).sum(1)
        ce = -torch.log_softmax(logits, 1).gather(1, labels[rows].clamp(min=0).long()[:, None])[:, 0] * (labels[rows] >= 0)
        total = total + (w_kl * tau**2 * kl + w_ce * ce).mean()
    return total


@pytest.mark.parametrize("blocks,p", [(1, 0.0), (2, 0.3), (3, 0.1)])
def test_gradient_of_a_round_against_autograd(blocks, p):
    model = codistill.Blocks(2, 23, 6, blocks, p, seed=3)
    model.x[:, :model.P] += 0.1 * torch.randn((2, model.P), device=DEV, generator=torch.Generator(DEV).manual_seed(1))
    model.rng[:, 1] += 1_000_000_007
    tokens, labels, reset = codistill.text(2, 3, 19, 23, 4)
    gen = torch.Generator().manual_seed(2)
    ids = torch.stack([torch.randperm(23, generator=gen)[:4] for _ in range(2 * 57)]).int()
    t = torch.randn((2 * 57, 4), generator=gen)
    loss = model.gradient(tokens, labels, reset, (ids.to(DEV), t.to(DEV)), 2.0, 0.5, 1.0)
    x = model.x.cpu().double().requires_grad_()
    ref = reference_loss(model, x, tokens.cpu(), labels.cpu(), reset.cpu(), (ids, t), 2.0, 0.5, 1.0)
    ref.backward()
    assert abs(float(loss.sum()) - float(ref.detach())) < 1e-5 * abs(float(ref.detach()))
    got, want = model.g.cpu().double()[:, :model.P], x.grad[:, :model.P]
    assert float((got - want).abs().max()) < 5e-5 * float(want.abs().max())


@pytest.mark.parametrize("together", [True, False])
def test_rounds_run_and_draw_new_masks(together):
    model = codistill.Blocks(4, 31, 32, 2, 0.1, seed=5)
    held_out, draws = codistill.text(4, 4, 64, 31, 99), []
    for k in range(6):
        draws.append(model.rng[:, 1].tolist())
        loss = model.step(*codistill.text(4, 4, 64, 31, k), codistill=together)
        assert loss.isfinite().all() and model.x.isfinite().all() and model.g[:, :model.P].isfinite().all()
    assert len({d for row in draws for d in row}) == 6 * 4
    logp, entropy = model.score(*held_out)
    assert logp.isfinite().all() and entropy.isfinite().all()
    assert torch.equal(model.forward(model.x, *held_out[::2]), model.forward(model.x, *held_out[::2]))      # scores drop nothing


def test_generation_by_single_steps_follows_the_sequence():
    model = codistill.Blocks(2, 31, 16, 2, seed=7)
    for k in range(5):
        model.step(*codistill.text(2, 2, 32, 31, k))
    prompts = codistill.text(1, 3, 20, 31, 50)[0].view(3, 20)
    out = model.generate(1, prompts, 6)
    whole = torch.cat([prompts, out], 1)
    reset = torch.zeros((3, 26), dtype=torch.uint8, device=DEV)
    z = model.forward(model.x[1:2], whole.reshape(1, -1).contiguous(), reset).view(3, 26, 31)
    best = z[:, 19:25].max(2).values
    chosen = z[:, 19:25].gather(2, out.long()[..., None])[..., 0]
    assert ((best - chosen) < 1e-4).all()


def test_the_command_trains_blocks(capsys):
    codistill.main(["--workers", "4", "--steps", "2", "--vocab", "23", "--width", "16", "--batch", "2", "--length", "24", "--blocks", "2", "--dropout", "0.1"])
    assert '"round": 2' in capsys.readouterr().out
