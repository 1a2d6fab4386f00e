"""Dropout, the logits in 8-bit floating point, the selection of beams and their reordering in runs as a program makes them: a training step and a beam search,
call by call against the float64 definitions, and captured into graphs that are replayed between eager work."""
import numpy as np
import pytest
import torch

from oracle import beam_oracle, dropout_oracle, fp8_oracle
from paper_2603_25011_amd.beam import beam_reorder, beam_select
from paper_2603_25011_amd.dropout import dropout
from paper_2603_25011_amd.fp8 import Fp8Head, fp8_logits

from tests.test_gpu_fp8 import U, close, host, tolerance

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
P, SEED, OFFSET = 0.1, 3, 40


def step(H, W, bias, state, target):
    """Dropout on the hidden states, logits, the gradient of a cross entropy at them, and what comes back of it."""
    x = dropout(H, P, SEED, OFFSET, state)
    y = fp8_logits(x, W, bias, torch.bfloat16)
    g = torch.softmax(y.detach().float(), -1)
    g = (g - torch.nn.functional.one_hot(target, W.shape[0])).to(y.dtype)
    return (x.detach(), y.detach(), g, *torch.autograd.grad(y, (H, W, bias), g))


def leaves(gen, N, V, D, dtype):
    H = torch.randn(N, D, generator=gen).to(dtype).to(DEV).requires_grad_(True)
    W = (torch.randn(V, D, generator=gen) * 0.3).to(dtype).to(DEV).requires_grad_(True)
    return H, W, torch.randn(V, generator=gen).to(DEV).requires_grad_(True)


@pytest.mark.parametrize("N,V,D,dtype", [(1, 300, 100, torch.float32), (70, 1000, 312, torch.bfloat16), (300, 517, 129, torch.float32), (513, 2000, 768, torch.bfloat16)])
def test_a_training_step(N, V, D, dtype):
    gen = torch.Generator().manual_seed(N)
    H, W, bias = leaves(gen, N, V, D, dtype)
    state = torch.tensor([11, 7], device=DEV)
    x, y, g, dH, dW, db = step(H, W, bias, state, torch.randint(0, V, (N,), generator=gen).to(DEV))
    kept, factor = dropout_oracle.keep(N * D, P, SEED + 11, OFFSET + 7)
    kept = kept.reshape(N, D)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else U
    close(host(x), host(H) * kept * factor, (2 * U + half) * 1.01 * np.abs(host(H)) * factor, "dropout")
    hq, wq, gq = fp8_oracle.blocks(host(x), 1, 128)[0], fp8_oracle.blocks(host(W), 128, 128)[0], fp8_oracle.blocks(host(g), 1, 128)[0]
    ht, gt = fp8_oracle.blocks(host(x), 128, 1)[0], fp8_oracle.blocks(host(g), 128, 1)[0]
    want = hq @ wq.T + host(bias)
    close(host(y), want, tolerance(hq, wq, want, "bf16", host(bias)), "logits")
    out = "bf16" if dtype == torch.bfloat16 else "f32"
    # the gradient of the dropped states is rounded to their type, then multiplied and rounded once more
    want = gq @ wq
    tol = tolerance(gq, wq.T, want, out)
    close(host(dH), want * kept * factor, (tol + (2 * U + half) * 1.01 * (np.abs(want) + tol)) * kept * factor, "dH")
    close(host(dW), gt.T @ ht, tolerance(gt.T, ht.T, gt.T @ ht, out), "dW")
    close(host(db), host(g).sum(axis=0), 8 * U * (np.sqrt(N) + 1) * np.abs(host(g)).sum(axis=0), "db")


@pytest.mark.parametrize("N,V,D,dtype", [(200, 1000, 312, torch.bfloat16), (5, 3000, 129, torch.float32)])
def test_a_captured_training_step(N, V, D, dtype):
    gen = torch.Generator().manual_seed(N)
    H, W, bias = leaves(gen, N, V, D, dtype)
    state, target = torch.zeros(2, dtype=torch.int64, device=DEV), torch.randint(0, V, (N,), generator=gen).to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(H, W, bias, state, target)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(H, W, bias, state, target)
    seen = []
    for k in range(4):
        with torch.no_grad():
            state.copy_(torch.tensor([k, 5 * k], device=DEV))
            target.copy_(torch.randint(0, V, (N,), generator=gen))
            W.add_(torch.randn(V, D, generator=gen).to(W).mul(0.1))
            H.copy_(torch.randn(N, D, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        mine = [t.detach().clone().requires_grad_(True) for t in (H, W, bias)]
        want = step(*mine, state, target)
        for a, b, what in zip(got, want, ("dropped", "logits", "their gradient", "dH", "dW", "db")):
            assert torch.equal(a, b), (k, what)
        seen.append(got[3].clone())
    assert not any(torch.equal(seen[0], s) for s in seen[1:])


def search(head, table, hidden, caches, scores, finished, steps, end_id):
    """`steps` steps of a beam search whose states are summed embeddings: (scores, tokens [B, beams, steps], caches)."""
    B, beams, D = hidden.shape
    tokens = torch.zeros((B, beams, steps), dtype=torch.int32, device=DEV)
    for t in range(steps):
        logits = head.logits(hidden, torch.bfloat16 if t % 2 else torch.float32)
        scores, parents, chosen = beam_select(logits, scores, beams, 1.0, finished, end_id)
        hidden, tokens, finished, *caches = beam_reorder([hidden, tokens, finished, *caches], parents)
        tokens[:, :, t] = chosen
        finished = finished | (chosen == end_id)
        hidden = hidden + table[chosen.long().reshape(-1)].reshape(B, beams, D)
        for c in caches:
            c[:, :, :, t] = hidden[:, :, None, :c.shape[-1]].to(c.dtype)
        yield logits, scores, parents, chosen, tokens, finished, hidden, caches


def start(gen, B, beams, V, D, steps):
    W = torch.randn(V, D, generator=gen).to(DEV) * 0.3
    W[5] *= 2.0                                                    # an end that is chosen now and then
    head = Fp8Head(W, torch.randn(V, generator=gen).to(DEV))
    hidden = torch.randn(B, 1, D, generator=gen).expand(B, beams, D).contiguous().to(DEV)
    scores = torch.full((B, beams), -float("inf"))
    scores[:, 0] = 0                                               # all beams are alike at the first step
    caches = [torch.zeros(B, beams, 2, steps, 16, dtype=dt, device=DEV) for dt in (torch.float32, torch.bfloat16)]
    return head, W, hidden, caches, scores.to(DEV), torch.zeros(B, beams, dtype=torch.bool, device=DEV)


@pytest.mark.parametrize("B,beams,V,D", [(1, 1, 700, 64), (3, 4, 3000, 129), (9, 5, 517, 100), (1, 16, 30522, 64)])
def test_a_beam_search(B, beams, V, D):
    gen = torch.Generator().manual_seed(V)
    head, table, hidden, caches, scores, finished = start(gen, B, beams, V, D, 6)
    wq = fp8_oracle.unpack(head.W8.cpu().numpy(), head.exps.cpu().numpy(), D)
    before = (hidden, torch.zeros((B, beams, 6), dtype=torch.int32), finished, caches, scores)
    for t, (logits, scores, parents, chosen, tokens, finished, hidden, caches) in enumerate(search(head, table, hidden, caches, scores, finished, 6, 5)):
        last_hidden, last_tokens, last_finished, last_caches, last_scores = before
        hq = fp8_oracle.blocks(host(last_hidden).reshape(-1, D), 1, 128)[0]
        want = hq @ wq.T + host(head.bias)
        close(host(logits).reshape(-1, V), want, tolerance(hq, wq, want, "bf16" if t % 2 else "f32", host(head.bias)), "logits")
        best = beam_oracle.select(host(logits), host(last_scores), beams, 1.0, last_finished.cpu().numpy(), 5)
        assert np.array_equal(parents.cpu().numpy(), best[1]) and np.array_equal(chosen.cpu().numpy(), best[2])
        close(host(scores), best[0], U * np.abs(np.where(np.isfinite(best[0]), best[0], 0)) + 64 * U, "scores")
        p = parents.cpu().numpy()
        want = beam_oracle.reorder(last_tokens.cpu().numpy(), p)
        want[:, :, t] = best[2]
        assert np.array_equal(tokens.cpu().numpy(), want)
        for c, last in zip(caches, last_caches):
            assert np.array_equal(host(c)[:, :, :, :t], beam_oracle.reorder(host(last), p)[:, :, :, :t])
        before = tuple(x.clone() if isinstance(x, torch.Tensor) else [c.clone() for c in x] for x in (hidden, tokens, finished, caches, scores))
    assert len({tuple(r) for r in tokens[0].tolist()}) == beams


def test_a_captured_beam_search():
    gen = torch.Generator().manual_seed(2)
    B, beams, V, D, steps = 4, 5, 9001, 96, 4
    head, table, hidden, caches, scores, finished = start(gen, B, beams, V, D, steps)

    def run():
        *_, last = search(head, table, hidden, caches, scores, finished, steps, 5)
        return [last[1], last[4], last[5], *last[7]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for k in range(4):
        hidden.copy_(torch.randn(B, 1, D, generator=gen).expand(B, beams, D))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, run())), k


def test_two_streams_at_once():
    """Calls on two streams share no memory: the same results as one after the other."""
    gen = torch.Generator().manual_seed(6)
    work = [(torch.randn(300, 768, generator=gen).to(DEV), Fp8Head(torch.randn(5000, 768, generator=gen).to(DEV)), torch.zeros(60, 5, device=DEV)) for _ in range(2)]

    def run(H, head, scores):
        logits = head.logits(dropout(H, 0.2, 1, 1))
        return logits, *beam_select(logits.view(60, 5, -1), scores, 7)
    want = [run(*w) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(8):
        for w, s, g in zip(work, streams, got):
            with torch.cuda.stream(s):
                g.append(run(*w))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for one in g for a, b in zip(w, one))
