"""Gossip training of small language models with codistillation: the language-model operators and the mixing step together.

W workers train replicas of one model on their own tokens.  The model is an embedding table (tied: also the output
projection), one gated recurrence over its rows and a residual connection; a worker's parameters are one flat row
[table V x D | projection D x 2 D].  A round:

    forward     cx_embed_lookup, projection, cx_gated_scan, output projection
    teacher     the same forward pass with the parameters of the peer that the round's topology gives each worker;
                cx_token_scores keeps its K most likely tokens
    loss        cx_distill_step: the label's cross entropy and the distance to the teacher, gradient over the logits
    backward    output projection, cx_gated_scan_grad, projection, cx_embed_grad added to the output projection's gradient
    update      cx_sgd_fused_mix: momentum SGD and segment-wise averaging with the peers

Blocks is the same with residual blocks in the recurrence's place, any number of them: norm, projection, short convolution, selective
scan with a gate, projection back, dropout on what is added to the residual:

    forward     cx_add_norm, projection, cx_short_conv, projection, cx_select_scan, projection, ..., cx_add_norm, cx_dropout
    backward    their gradients into the same flat rows, the masks drawn again from the counter

The matrix products in between are torch's.  `python -m paper_2012_15198_amd.codistill` trains on synthetic text (noisy
arithmetic sequences, packed documents) and prints the loss and the log probability of held-out text; --blocks 2 --dropout 0.1
trains two blocks with dropout.
"""
from __future__ import annotations

import argparse
import json
import math

import numpy as np
import torch

from . import cxlm as lm
from . import cxmix as cx
from .workloads import equal_seg_off


class Replicas:
    """W replicas with flat float32 parameters x [W][ld], momentum v and gradients g, on one GPU."""

    def __init__(self, W, V, D, S=4, seed=0, device="cuda:0"):
        self.W, self.V, self.D, self.S, self.seed, self.device = W, V, D, S, seed, device
        self.P = V * D + 2 * D * D
        ld = -(-self.P // 8) * 8
        gen = torch.Generator(device).manual_seed(seed)
        self.x = torch.zeros((W, ld), device=device)
        self.x[:, :self.P].normal_(0.0, 1.0 / math.sqrt(D), generator=gen)
        self.x[:, V * D:self.P] /= 2
        self.x[:] = self.x[0]                                    # replicas begin equal
        self.v, self.g = torch.zeros_like(self.x), torch.zeros_like(self.x)
        self.x2, self.v2 = torch.zeros_like(self.x), torch.zeros_like(self.x)
        offsets = equal_seg_off(self.P, S)
        cx.cx_check_segments(offsets, self.P)
        self.offsets, self.round = torch.from_numpy(offsets).to(device), 0

    def table(self, rows, w):
        return rows[w, :self.V * self.D].view(self.V, self.D)

    def projection(self, rows, w):
        return rows[w, self.V * self.D:self.P].view(self.D, 2 * self.D)

    def forward(self, x, tokens, reset, keep=False):
        """Logits [W * B * T][V] of tokens int32 [W][B * T]; reset: uint8 [W * B][T].  keep: also what the backward pass needs."""
        W, D, N, T = tokens.shape[0], self.D, tokens.shape[1], reset.shape[1]
        e = torch.empty((W * N, D), device=x.device)
        lm.cx_embed_lookup(x, tokens, e, 0, self.V, math.sqrt(D))
        fu = torch.empty((W * N, 2 * D), device=x.device)        # gates and inputs side by side
        for w in range(W):
            torch.mm(e[w * N:(w + 1) * N], self.projection(x, w), out=fu[w * N:(w + 1) * N])
        y = torch.empty_like(e)
        states = lm.scan_states(y, T) if keep else None
        lm.cx_gated_scan(fu[:, :D], fu[:, D:], y, T, reset=reset, states=states)
        s = (e + y) / math.sqrt(D)
        z = torch.empty((W * N, self.V), device=x.device)
        for w in range(W):
            torch.mm(s[w * N:(w + 1) * N], self.table(x, w).t(), out=z[w * N:(w + 1) * N])
        return (z, e, fu, s, states) if keep else z

    def gradient(self, tokens, labels, reset, teacher=None, tau=2.0, w_kl=0.5, w_ce=1.0):
        """Fills g; the mean loss of each worker.  labels: int32 [W * N] (-1: none); teacher: (ids, log probabilities) of K tokens."""
        W, D, N, T = self.W, self.D, tokens.shape[1], reset.shape[1]
        z, e, fu, s, states = self.forward(self.x, tokens, reset, keep=True)
        ids, t = teacher or (torch.empty((W * N, 0), dtype=torch.int32, device=z.device), torch.empty((W * N, 0), device=z.device))
        loss, gout = torch.empty(W * N, device=z.device), torch.full((W * N,), 1.0 / N, device=z.device)
        lm.cx_distill_step(z, ids, t, labels, gout, loss, z, tau, w_kl, w_ce)          # the gradient takes the logits' place
        ds = torch.empty_like(e)
        for w in range(W):
            rows = slice(w * N, (w + 1) * N)
            torch.mm(z[rows], self.table(self.x, w), out=ds[rows])
            torch.mm(z[rows].t(), s[rows], out=self.table(self.g, w))
        ds /= math.sqrt(D)
        dfu = torch.empty_like(fu)
        lm.cx_gated_scan_grad(fu[:, :D], fu[:, D:], ds, dfu[:, :D], dfu[:, D:], T, states, reset=reset)
        for w in range(W):
            rows = slice(w * N, (w + 1) * N)
            torch.mm(e[rows].t(), dfu[rows], out=self.projection(self.g, w))
            ds[rows].addmm_(dfu[rows], self.projection(self.x, w).t())
        lm.cx_embed_grad(ds, tokens, self.g, self.g, 0, self.V, math.sqrt(D))
        return loss.view(W, N).mean(1)

    def step(self, tokens, labels, reset, lr=0.1, mu=0.9, wd=0.0, K=8, codistill=True):
        """One round; the mean loss of each worker."""
        peers = cx.cx_topology_gen(self.seed, self.W, self.S, self.round, 1)[0]
        cx.cx_check_peers(peers)
        teacher = None
        if codistill:
            z = self.forward(self.x[torch.from_numpy(peers[0]).long().to(self.device)], tokens, reset)
            ids = torch.empty((z.shape[0], K), dtype=torch.int32, device=z.device)
            top = torch.empty((z.shape[0], K), device=z.device)
            lm.cx_token_scores(z, None, None, None, ids, top)
            teacher = ids, top
        loss = self.gradient(tokens, labels, reset, teacher)
        cx.cx_sgd_fused_mix(self.x, self.x2, self.v, self.v2, self.g, lr, mu, wd, self.P, self.offsets, torch.from_numpy(peers).to(self.device))
        self.x, self.x2, self.v, self.v2 = self.x2, self.x, self.v2, self.v
        self.round += 1
        return loss

    def score(self, tokens, labels, reset):
        """Mean log probability of the labels and mean entropy, per worker."""
        z = self.forward(self.x, tokens, reset)
        logp, entropy = (torch.empty(z.shape[0], device=z.device) for _ in range(2))
        lm.cx_token_scores(z, labels, logp, entropy)
        known = (labels >= 0).view(self.W, -1)
        return logp.view(self.W, -1).sum(1) / known.sum(1), entropy.view(self.W, -1).mean(1)

    def generate(self, w, prompts, steps):
        """Greedy continuation, int32 [B][steps], of prompts int32 [B][T] by worker w: one scan over the prompts, then a token
        at a time, the state updated in place."""
        x, D = self.x[w:w + 1], self.D
        B, T = prompts.shape
        state = torch.zeros((B, D), device=x.device)
        out = torch.empty((B, steps), dtype=torch.int32, device=x.device)
        tokens = prompts
        for k in range(steps):
            n = tokens.shape[1]
            e, y = (torch.empty((B * n, D), device=x.device) for _ in range(2))
            lm.cx_embed_lookup(x, tokens.reshape(1, -1), e, 0, self.V, math.sqrt(D))
            fu = e @ self.projection(x, 0)
            lm.cx_gated_scan(fu[:, :D], fu[:, D:], y, n, h0=state, h_last=state)
            z = ((e + y).view(B, n, D)[:, -1] / math.sqrt(D)) @ self.table(x, 0).t()
            ids, top = torch.empty((B, 1), dtype=torch.int32, device=x.device), torch.empty((B, 1), device=x.device)
            lm.cx_token_scores(z, None, None, None, ids, top)
            out[:, k] = ids[:, 0]
            tokens = ids
        return out


class Blocks(Replicas):
    """W replicas of a model of residual blocks.  A worker's flat row: table V x D; of each block norm D, projection D x 2 D, convolution
    D x K and D, projection D x (D + 2 S), scan D x S, D and D, projection D x D; norm D."""

    K, S_, EPS = 4, 8, 1e-6                                      # taps, states of a column

    def __init__(self, W, V, D, blocks=2, dropout=0.0, S=4, seed=0, device="cuda:0"):
        K, N, at = self.K, self.S_, V * D
        self.blocks, self.p, self.at = blocks, dropout, []
        for _ in range(blocks):
            place = {}
            for name, size in (("norm", D), ("into", 2 * D * D), ("conv", D * (K + 1)), ("steps", D * (D + 2 * N)), ("scan", D * (N + 2)), ("back", D * D)):
                place[name], at = at, at + size
            self.at.append(place)
        self.norm, self.P = at, at + D
        self.W, self.V, self.D, self.S, self.seed, self.device = W, V, D, S, seed, device
        gen = torch.Generator(device).manual_seed(seed)
        row = torch.empty(self.P, device=device).normal_(0.0, 1.0 / math.sqrt(D), generator=gen)
        row[self.norm:] = 1.0
        for place in self.at:
            row[place["norm"]:place["into"]] = 1.0
            row[place["conv"] + D * K:place["steps"]] = 0.0
            scan = row[place["scan"]:place["back"]]
            scan[:D * N] = (torch.arange(N, device=device) + 1.0).log().repeat(D)
            steps = (torch.rand(D, device=device, generator=gen) * math.log(100.0) + math.log(1e-3)).exp()
            scan[D * N:D * (N + 1)] = steps + (-(-steps).expm1()).log()          # softplus gives the steps
            scan[D * (N + 1):] = 1.0
        self.x = torch.zeros((W, -(-self.P // 8) * 8), device=device)
        self.x[:, :self.P] = row                                 # replicas begin equal
        self.v, self.g = torch.zeros_like(self.x), torch.zeros_like(self.x)
        self.x2, self.v2 = torch.zeros_like(self.x), torch.zeros_like(self.x)
        offsets = equal_seg_off(self.P, S)
        cx.cx_check_segments(offsets, self.P)
        self.offsets, self.round = torch.from_numpy(offsets).to(device), 0
        # key and draw of each mask: the embedding's, the blocks', the last one; a round's draws follow the round's before
        self.rng = torch.tensor([[seed, k] for k in range(blocks + 2)], dtype=torch.int64, device=device)

    def part(self, rows, w, at, columns):
        return rows[w, at:at + self.D * columns].view(self.D, columns)

    def product(self, x, at, columns, a):
        """a @ the workers' matrices [D][columns] at `at`, each on its own rows."""
        out, n = torch.empty((a.shape[0], columns), device=a.device), a.shape[0] // x.shape[0]
        for w in range(x.shape[0]):
            torch.mm(a[w * n:(w + 1) * n], self.part(x, w, at, columns), out=out[w * n:(w + 1) * n])
        return out

    def product_grad(self, at, columns, a, d):
        """Of product(): the gradient of a, and into g that of the matrices."""
        da, n = torch.empty_like(a), a.shape[0] // self.W
        for w in range(self.W):
            rows = slice(w * n, (w + 1) * n)
            torch.mm(a[rows].t(), d[rows], out=self.part(self.g, w, at, columns))
            torch.mm(d[rows], self.part(self.x, w, at, columns).t(), out=da[rows])
        return da

    def block(self, x, place, y, T, reset=None, states=None, before=None, h=None):
        """What a block adds to the residual, from the norm's output y; before and h: the state of generation, in place."""
        D, K, N = self.D, self.K, self.S_
        into = self.product(x, place["into"], 2 * D, y)
        u, v = torch.empty_like(y), torch.empty_like(y)
        lm.cx_short_conv(into[:, :D], x, place["conv"], u, T, K, before=before, after=before, reset=reset)
        steps = self.product(x, place["steps"], D + 2 * N, u)
        lm.cx_select_scan(u, steps[:, :D], steps[:, D:D + N], steps[:, D + N:], x, place["scan"], v, T, z=into[:, D:], h0=h, h_last=h, reset=reset, states=states)
        return self.product(x, place["back"], D, v), into, u, steps, v

    def forward(self, x, tokens, reset, keep=False):
        W, D, n, T = tokens.shape[0], self.D, tokens.shape[1], reset.shape[1]
        p = self.p if keep else 0.0                              # the teacher and scores drop nothing
        add, s, kept = torch.empty((W * n, D), device=x.device), None, []
        lm.cx_embed_lookup(x, tokens, add, 0, self.V, math.sqrt(D))
        for k, place in enumerate(self.at):
            total, y, inv = torch.empty_like(add), torch.empty_like(add), torch.empty(W * n, device=x.device)
            lm.cx_add_norm(add, s, x, place["norm"], total, y, self.EPS, inv=inv, p=p, rng=self.rng[k])
            states = lm.select_states(y, T, self.S_) if keep else None
            s, (add, into, u, steps, v) = total, self.block(x, place, y, T, reset, states)
            kept.append((s, y, inv, into, u, steps, v, states))
        total, y, inv = torch.empty_like(add), torch.empty_like(add), torch.empty(W * n, device=x.device)
        lm.cx_add_norm(add, s, x, self.norm, total, y, self.EPS, inv=inv, p=p, rng=self.rng[self.blocks])
        if p:
            lm.cx_dropout(y, self.rng[self.blocks + 1], y, p)
        y /= math.sqrt(D)
        z = torch.empty((W * n, self.V), device=x.device)
        for w in range(W):
            torch.mm(y[w * n:(w + 1) * n], self.table(x, w).t(), out=z[w * n:(w + 1) * n])
        return (z, (total, y, inv), kept) if keep else z

    def gradient(self, tokens, labels, reset, teacher=None, tau=2.0, w_kl=0.5, w_ce=1.0):
        W, D, N, n, T, p = self.W, self.D, self.S_, tokens.shape[1], reset.shape[1], self.p
        z, (s, y, inv), kept = self.forward(self.x, tokens, reset, keep=True)
        ids, t = teacher or (torch.empty((W * n, 0), dtype=torch.int32, device=z.device), torch.empty((W * n, 0), device=z.device))
        loss, gout = torch.empty(W * n, device=z.device), torch.full((W * n,), 1.0 / n, device=z.device)
        lm.cx_distill_step(z, ids, t, labels, gout, loss, z, tau, w_kl, w_ce)          # the gradient takes the logits' place
        dy = torch.empty_like(y)
        for w in range(W):
            rows = slice(w * n, (w + 1) * n)
            torch.mm(z[rows], self.table(self.x, w), out=dy[rows])
            torch.mm(z[rows].t(), y[rows], out=self.table(self.g, w))
        dy /= math.sqrt(D)
        if p:
            lm.cx_dropout(dy, self.rng[self.blocks + 1], dy, p)
        ds, dadd = torch.empty_like(dy), torch.empty_like(dy)
        lm.cx_add_norm_grad(dy, s, inv, self.x, self.norm, None, ds, None, self.g, dx=dadd, p=p, rng=self.rng[self.blocks])
        for k in range(self.blocks - 1, -1, -1):
            place, (s, y, inv, into, u, steps, v, states) = self.at[k], kept[k]
            dv = self.product_grad(place["back"], D, v, dadd)
            du, dinto, dsteps = torch.empty_like(u), torch.empty_like(into), torch.empty_like(steps)
            lm.cx_select_scan_grad(u, steps[:, :D], steps[:, D:D + N], steps[:, D + N:], self.x, place["scan"], dv, du, dsteps[:, :D], dsteps[:, D:D + N],
                                   dsteps[:, D + N:], None, self.g, T, states, z=into[:, D:], dz=dinto[:, D:], reset=reset)
            du += self.product_grad(place["steps"], D + 2 * N, u, dsteps)
            lm.cx_short_conv_grad(into[:, :D], du, self.x, place["conv"], dinto[:, :D], None, self.g, T, self.K, reset=reset)
            dy = self.product_grad(place["into"], 2 * D, y, dinto)
            lm.cx_add_norm_grad(dy, s, inv, self.x, place["norm"], ds, ds if k else None, None, self.g, dx=dadd, p=p, rng=self.rng[k])
        lm.cx_embed_grad(dadd, tokens, self.g, self.g, 0, self.V, math.sqrt(D))
        return loss.view(W, n).mean(1)

    def step(self, *args, **kw):
        loss = super().step(*args, **kw)
        self.rng[:, 1] += self.blocks + 2
        return loss

    def generate(self, w, prompts, steps):
        x, D, B = self.x[w:w + 1], self.D, prompts.shape[0]
        inputs = [torch.zeros((B, self.K - 1, D), device=x.device) for _ in self.at]
        states = [torch.zeros((B, D, self.S_), device=x.device) for _ in self.at]
        out, tokens = torch.empty((B, steps), dtype=torch.int32, device=x.device), prompts
        for k in range(steps):
            n = tokens.shape[1]
            add, s = torch.empty((B * n, D), device=x.device), None
            lm.cx_embed_lookup(x, tokens.reshape(1, -1), add, 0, self.V, math.sqrt(D))
            for place, before, h in zip(self.at, inputs, states):
                total, y = torch.empty_like(add), torch.empty_like(add)
                lm.cx_add_norm(add, s, x, place["norm"], total, y, self.EPS)
                s, add = total, self.block(x, place, y, n, before=before, h=h)[0]
            y = torch.empty_like(add)
            lm.cx_add_norm(add, s, x, self.norm, None, y, self.EPS)
            z = (y.view(B, n, D)[:, -1] / math.sqrt(D)) @ self.table(x, 0).t()
            ids, top = torch.empty((B, 1), dtype=torch.int32, device=x.device), torch.empty((B, 1), device=x.device)
            lm.cx_token_scores(z, None, None, None, ids, top)
            out[:, k] = ids[:, 0]
            tokens = ids
        return out


def text(W, B, T, V, seed, device="cuda:0"):
    """Packed documents for every worker: arithmetic sequences modulo V whose step is the document's own, one token in ten
    at random.  tokens int32 [W][B * T], labels int32 [W * B * T] (-1 where a document ends), reset uint8 [W * B][T]."""
    rng = np.random.default_rng(seed)
    reset = rng.random((W * B, T + 1)) < 0.05
    reset[:, 0] = True
    document = np.cumsum(reset, 1)
    begin, stride = rng.integers(0, V, (W * B, T + 2)), rng.integers(1, 4, (W * B, T + 2))
    place = np.arange(T + 1) - np.maximum.accumulate(np.where(reset, np.arange(T + 1), 0), 1)
    rows = np.arange(W * B)[:, None]
    tokens = (begin[rows, document] + stride[rows, document] * place) % V
    noise = rng.random(tokens.shape) < 0.1
    tokens = np.where(noise, rng.integers(0, V, tokens.shape), tokens).astype(np.int32)
    labels = np.where(reset[:, 1:], -1, tokens[:, 1:]).astype(np.int32)
    on = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
    return on(tokens[:, :-1].reshape(W, B * T)), on(labels.reshape(-1)), on(reset[:, :-1].astype(np.uint8))


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("workers", 8), ("steps", 100), ("vocab", 97), ("width", 64), ("batch", 4), ("length", 128), ("seed", 1)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--no-codistill", action="store_true", help="labels alone")
    ap.add_argument("--blocks", type=int, default=0, help="residual blocks in the gated recurrence's place")
    ap.add_argument("--dropout", type=float, default=0.0, help="share of what blocks add that is dropped")
    a = ap.parse_args(argv)
    if a.blocks < 0:
        ap.error("--blocks: a number of blocks")
    if a.dropout and not a.blocks:
        ap.error("--dropout: of --blocks")
    model = Blocks(a.workers, a.vocab, a.width, a.blocks, a.dropout, seed=a.seed) if a.blocks else Replicas(a.workers, a.vocab, a.width, seed=a.seed)
    held_out = text(a.workers, a.batch, a.length, a.vocab, 10**6 + a.seed)
    for k in range(a.steps + 1):
        if k % 20 == 0 or k == a.steps:
            logp, entropy = model.score(*held_out)
            print(json.dumps({"round": k, "held_out_logp": round(float(logp.mean()), 4), "entropy": round(float(entropy.mean()), 4),
                              "spread": round(float((model.x - model.x.mean(0)).norm() / model.x.norm()), 6)}), flush=True)
        if k < a.steps:
            model.step(*text(a.workers, a.batch, a.length, a.vocab, a.seed * 7919 + k), codistill=not a.no_codistill)


if __name__ == "__main__":
    main()
