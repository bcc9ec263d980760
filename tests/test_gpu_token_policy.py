"""The token operators together, as a training step uses them (examples/token_policy_step.py): gradients against autograd, learning, a
captured step, another stream; and tensors of more than 2^31 values."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_1805_04170_amd as tt

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("token_policy_step", os.path.join(ROOT, "examples", "token_policy_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def inputs(example, policy, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    T, V = policy.tokens, policy.vocab
    ids = torch.randint(0, V, (T,), generator=g, device=DEV)
    actions = torch.randint(0, V, (T,), generator=g, device=DEV)
    logp = policy.logp(policy.forward(ids), actions)
    old = logp + torch.tensor([-0.5, -0.1, 0.05, 0.4], device=DEV)[torch.randint(0, 4, (T,), generator=g, device=DEV)]
    ref = logp + 0.2 * torch.randn(T, generator=g, device=DEV)
    advantage = torch.randn(T, generator=g, device=DEV)
    weight = torch.where(torch.rand(T, generator=g, device=DEV) < 0.2, 0.0, 1.0 / T)
    return ids, actions, old, ref, advantage, weight


def test_gradients_of_a_step_against_autograd(example):
    V, T, lo, hi, kl = 32, 64, 0.2, 0.25, 0.05
    p = example.TokenPolicy(V, (32, 64), T, 2, seed=3)
    ids, a, old, ref, adv, w = inputs(example, p, 4)
    loss, dE, dW = p.gradients(tt.policy(lo, hi, kl), ids, a, old, ref, adv, w)
    E = example.join(p.E, p.table, V, 32).double().requires_grad_()
    W = [example.join(s, t, r, c).double().requires_grad_() for s, t, r, c in zip(p.W, p.w, p.widths, p.widths[1:])]
    x = E[ids] * p.scale
    for i, m in enumerate(W):
        x = x @ m
        if i + 1 < len(W):
            x = torch.relu(x)
    logp = torch.log_softmax(x, 1)[torch.arange(T, device=DEV), a]
    ratio = torch.exp(logp - old)
    d = ref - logp
    want = (w * (-torch.minimum(ratio * adv, ratio.clamp(1 - lo, 1 + hi) * adv) + kl * (torch.exp(d) - 1 - d))).sum()
    want.backward()
    near = lambda got, ref: float((got.double() - ref).norm() / ref.norm())  # noqa: E731
    # the loss and the way back to the table see no 8-bit value but gates, which are exact: fp32 errors alone, some 1e-6
    assert abs(float(loss) - float(want.detach())) < 2e-5
    assert near(example.join(dE, p.table, V, 32), E.grad) < 1e-4
    # weight gradients read activations of 8 bits: a step is at most 1/64 of a block's largest value, off by a third of half of it
    for got, m, t in zip(dW, W, p.w):
        assert near(example.join(got, t, *m.shape), m.grad) < 2e-2


def test_training_learns(example):
    _, rewards = example.train(40, report=None)
    assert np.mean(rewards[-5:]) > 0.4 > 0.1 > np.mean(rewards[:2])


def test_a_step_in_a_graph_and_on_another_stream(example):
    p = example.TokenPolicy(64, (64, 256), 128, 2, seed=5)
    params = tt.policy(kl=0.1)
    sets = [inputs(example, p, s) for s in (6, 7, 8)]
    flat = lambda r: [r[0]] + r[1] + sum(r[2], [])  # noqa: E731
    want = [[t.clone() for t in flat(p.gradients(params, *s))] for s in sets]
    static = [t.clone() for t in sets[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = flat(p.gradients(params, *static))
    for turn in range(2):
        for s, ref in zip(sets, want):
            for a, b in zip(static, s):
                a.copy_(b)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, ref)), turn
            p.gradients(params, *s)         # (eager work between replays, in the same workspace)
            torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = flat(p.gradients(params, *sets[1]))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, want[1]))


def test_tables_of_more_values_than_31_bits_count():
    V, D, T = 70000, 32768, 300
    W = torch.empty((V, D), dtype=torch.bfloat16, device=DEV)
    W.view(torch.int16).copy_((torch.arange(V, device=DEV) % 997).to(torch.int16)[:, None].expand(V, D))     # row v holds the bits of v mod 997
    W[:, 5] = torch.arange(V, device=DEV).remainder(256).to(torch.bfloat16)
    ids = torch.randint(0, V, (T,), device=DEV)
    ids[:4] = torch.tensor([V - 1, 0, V - 1, 65536], device=DEV)
    X = torch.empty((T, D), dtype=torch.bfloat16, device=DEV)
    tt.tt_embed_forward(T, V, D, 0, "bf16", "", "", ids, 1.0, [W], [X])
    assert torch.equal(X[:, 5].float(), ids.remainder(256).float())
    assert torch.equal(X.view(torch.int16)[:, -1], (ids % 997).to(torch.int16))
    G = torch.randn((T, D), device=DEV).bfloat16()
    ws = torch.empty(tt.tt_embed_workspace_bytes(T, V, D, 0, "bf16", "", ""), dtype=torch.uint8, device=DEV)
    W.fill_(7)
    tt.tt_embed_backward(T, V, D, 0, "bf16", "", "", ids, 1.0, [G], [W], ws)
    rows = torch.unique(ids)
    want = torch.zeros((rows.numel(), D), device=DEV)
    want.index_add_(0, torch.searchsorted(rows, ids), G.float())
    got = W[rows].float()
    assert torch.all((got - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5)
    W[rows] = 0
    assert int(torch.count_nonzero(W.view(torch.int16)[:, ::61])) == 0 and int(torch.count_nonzero(W.view(torch.int16)[V - 5:])) == 0


def test_logits_of_more_values_than_31_bits_count():
    T, V = 20000, 120000
    X = torch.empty((T, V), dtype=torch.bfloat16, device=DEV).normal_(0, 2)
    a = torch.randint(0, V, (T,), device=DEV)
    one = torch.ones(T, device=DEV)
    rows = torch.tensor([0, 1, 17900, 17895, T - 2, T - 1], device=DEV)
    p = tt.policy(kl=0.1)

    def run(x, act, n):
        ws = torch.empty(tt.tt_policy_workspace_bytes(n, V, 0, "bf16", "", ""), dtype=torch.uint8, device=DEV)
        dX, logp, loss = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(1, device=DEV)
        tt.tt_policy_loss(p, n, V, 0, "bf16", "", "", [x], act, -12 * one[:n], -12 * one[:n], one[:n], one[:n], loss, logp, [dX], ws)
        return logp, dX
    logp, dX = run(X, a, T)
    few_logp, few_dX = run(X[rows].contiguous(), a[rows].contiguous(), rows.numel())
    # the same rows by themselves (other sums of the same 120000 terms)
    assert torch.all((logp[rows] - few_logp).abs() < 4e-5)
    assert torch.all((dX[rows].float() - few_dX.float()).abs() <= 2.0 ** -7 * few_dX.float().abs() + 1e-9)
    assert not torch.isnan(dX[:, ::997].float()).any()


def test_activations_of_more_values_than_31_bits_count():
    rows, cols = 66000, 32768
    X = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV).normal_(0, 1)
    Q, S = torch.empty((rows, cols), dtype=torch.int8, device=DEV), torch.empty((rows, cols // 32), dtype=torch.uint8, device=DEV)
    tt.tt_pack8(rows, cols, 0, "bf16", "", [X], [Q], [S])
    some = [0, 33000, 65535, 65536, rows - 1]
    x, q, s = (torch.stack([t[r] for r in some]).contiguous() for t in (X, Q, S))
    q2, s2 = torch.empty_like(q), torch.empty_like(s)
    tt.tt_pack8(len(some), cols, 0, "bf16", "", [x], [q2], [s2])
    assert torch.equal(q, q2) and torch.equal(s, s2)
    X.fill_(3)
    tt.tt_unpack8(rows, cols, 0, "bf16", "", [Q], [S], [X])
    back = torch.empty_like(x)
    tt.tt_unpack8(len(some), cols, 0, "bf16", "", [q2], [s2], [back])
    assert torch.equal(torch.stack([X[r] for r in some]), back)
    assert int((X[:, ::509] == 3).sum()) < X[:, ::509].numel() // 100
