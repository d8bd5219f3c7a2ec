"""The language-model operators inside captured graphs and on streams of their own: every replay equals the eager call, bit for bit."""
import pytest
import torch

from paper_2012_15198_amd import cxlm as lm

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


def calls():
    """name -> (inputs that change, outputs, call(workspace, stream), workspace bytes)"""
    gen = torch.Generator(DEV).manual_seed(3)
    normal = lambda *s, dtype=torch.float32: torch.randn(s, device=DEV, generator=gen).to(dtype)
    ints = lambda hi, *s: torch.randint(-1, hi, s, device=DEV, generator=gen).int()
    found = {}

    x, tokens, out = normal(3, 4000), ints(100, 3, 700), torch.empty((2100, 30), device=DEV)
    found["lookup"] = ([x, tokens], [out], lambda ws, st: lm.cx_embed_lookup(x, tokens, out, 500, 100, 2.0, stream=st), 0)
    dout, g = normal(2100, 30), torch.empty((3, 4000), device=DEV)
    found["embed_grad"] = ([dout, tokens], [g[:, 500:3500]], lambda ws, st: lm.cx_embed_grad(dout, tokens, None, g, 500, 100, 2.0, workspace=ws, stream=st),
                           lm.cx_embed_workspace(3, 700, 100, 30))
    B, T, D = 2, 900, 70
    f, u, dy = (normal(B * T, D, dtype=torch.bfloat16) for _ in range(3))
    y, df, du = (torch.empty_like(f) for _ in range(3))
    h0, h1, dh, dh0, states = normal(B, D), normal(B, D), normal(B, D), normal(B, D), lm.scan_states(f, T)
    reset = (torch.rand((B, T), device=DEV, generator=gen) < 0.02).to(torch.uint8)

    def scan(ws, st):
        lm.cx_gated_scan_bf16(f, u, y, T, h0=h0, h_last=h1, reset=reset, states=states, workspace=ws, stream=st)
        lm.cx_gated_scan_grad_bf16(f, u, dy, df, du, T, states, dh_last=dh, dh0=dh0, reset=reset, workspace=ws, stream=st)

    found["scan"] = ([f, u, dy, h0, dh], [y, h1, df, du, dh0], scan, lm.cx_scan_workspace(B, T, D))
    z, labels = normal(2, 70_001, dtype=torch.float16), ints(70_001, 2)
    logp, entropy, ids, top = torch.empty(2, device=DEV), torch.empty(2, device=DEV), torch.empty((2, 9), dtype=torch.int32, device=DEV), torch.empty((2, 9), device=DEV)
    found["scores"] = ([z, labels], [logp, entropy, ids, top], lambda ws, st: lm.cx_token_scores_f16(z, labels, logp, entropy, ids, top, workspace=ws, stream=st),
                       lm.cx_scores_workspace(2, 70_001, 9))
    z2, ids2, t2 = normal(1, 200_001), ints(200_001, 1, 5), normal(1, 5)
    gout, loss, dz, loss2, stats = normal(1), torch.empty(1, device=DEV), torch.empty_like(z2), torch.empty(1, device=DEV), torch.empty((1, 4), device=DEV)

    def distill(ws, st):
        lm.cx_distill_step(z2, ids2, t2, None, gout, loss, dz, 2.0, 1.0, 0.0, workspace=ws, stream=st)
        lm.cx_distill_loss(z2, ids2, t2, None, loss2, stats, 2.0, 1.0, 0.0, workspace=ws, stream=st)

    found["distill"] = ([z2, t2, gout], [loss, dz, loss2], distill, lm.cx_distill_workspace(1, 200_001))
    return found


NAMES = ["lookup", "embed_grad", "scan", "scores", "distill"]


@pytest.mark.parametrize("name", NAMES)
def test_replays_equal_eager_calls(name):
    inputs, outputs, call, needed = calls()[name]
    assert needed > 0 or name == "lookup"
    work = torch.empty(max(needed, 1), dtype=torch.uint8, device=DEV)
    call(work, None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(work, torch.cuda.current_stream())
    for k in range(4):
        for t in inputs:                                  # other data every time, eager work and synchronisation between the replays
            t.copy_(t.flip(0).roll(k + 1, -1))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outputs]
        for t in outputs:
            t.fill_(77)
        call(work, None)
        torch.cuda.synchronize()
        for a, b in zip(replayed, outputs):
            assert torch.equal(a, b)


@pytest.mark.parametrize("name", NAMES)
def test_calls_on_another_stream(name):
    inputs, outputs, call, needed = calls()[name]
    call(None, None)                                      # workspace from torch's allocator
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]
    for t in outputs:
        t.fill_(77)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    if needed:
        with pytest.raises(ValueError, match="brings its own workspace"):
            call(None, side)
    call(torch.empty(max(needed, 1), dtype=torch.uint8, device=DEV), side)
    side.synchronize()
    for a, b in zip(outputs, want):
        assert torch.equal(a, b)
    with torch.cuda.stream(side):
        for t in outputs:
            t.fill_(78)
        call(None, None)
    side.synchronize()
    for a, b in zip(outputs, want):
        assert torch.equal(a, b)
