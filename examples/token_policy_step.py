"""Training steps of a small token policy on a tiled chain of layers.

    python examples/token_policy_step.py [steps]

Each step: tokens come in, an embedding table's rows go through a chain of fully-connected layers under the planner's tilings, the
last layer's outputs are the logits over the vocabulary.  An action is drawn for every token and rewarded; the clipped policy loss
with its KL term gives the logits' gradient, the chain's backward pass reads its activations from 8 bits (the 16-bit or 32-bit
ones are gone by then), and the sum by token number is the table's gradient.  Several updates are made from the same draw, so
that the loss's ratios leave 1.

The task: the action that pays is (5 * token + 3) modulo the vocabulary.  The mean reward climbs from 1 / vocabulary towards 1.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1805_04170_amd as tt  # noqa: E402

DEV = "cuda:0"


def shard_count(t):
    return 1 << len(t)


def block_of(t, s):
    """(row block, column block) that shard s of tiling t holds"""
    r = c = 0
    for j, letter in enumerate(t):
        bit = (s >> (len(t) - 1 - j)) & 1
        r, c = (2 * r + bit, c) if letter == "R" else (r, 2 * c + bit) if letter == "C" else (r, c)
    return r, c


def cut(full, t):
    sr, sc = tt.tt_shard_shape(full.shape[0], full.shape[1], t)
    blocks = [block_of(t, s) for s in range(shard_count(t))]
    return [full[r * sr:(r + 1) * sr, c * sc:(c + 1) * sc].contiguous() for r, c in blocks]


def join(shards, t, rows, cols):
    out = torch.empty((rows, cols), dtype=shards[0].dtype, device=shards[0].device)
    for s, x in enumerate(shards):
        r, c = block_of(t, s)
        out[r * x.shape[0]:(r + 1) * x.shape[0], c * x.shape[1]:(c + 1) * x.shape[1]] = x
    return out


def empty(rows, cols, t, dtype):
    sr, sc = tt.tt_shard_shape(rows, cols, t)
    return [torch.empty((sr, sc), dtype=dtype, device=DEV) for _ in range(shard_count(t))]


class TokenPolicy:
    """An embedding table and a chain of layers, all tensors cut as the planner says; `table`: the table's own tiling."""

    def __init__(self, vocab, widths, tokens, k, dtype="f32", table=None, seed=0):
        self.vocab, self.widths, self.tokens, self.k, self.dtype = vocab, list(widths) + [vocab], tokens, k, dtype
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        L = self.layers = len(self.widths) - 1
        self.lay = [tt.layer("fc", "relu" if i < L - 1 else "none", self.widths[i], self.widths[i + 1]) for i in range(L)]
        plan = tt.tt_plan_chain(self.lay, tokens, k)
        self.x, self.g, self.w = plan.x(), plan.g(), plan.w()
        self.forms = [[plan.forms(i + 1, op) for op in range(3)] for i in range(L)]
        self.table = "C" * k if table is None else table
        gen = torch.Generator().manual_seed(seed)
        normal = lambda r, c, std: (torch.randn(r, c, generator=gen) * std).to(self.torch_dtype).to(DEV)  # noqa: E731
        self.E = cut(normal(vocab, self.widths[0], self.widths[0] ** -0.5), self.table)
        self.W = [cut(normal(a, b, (2.0 / a) ** 0.5 if i < L - 1 else 0.1 * a ** -0.5), self.w[i]) for i, (a, b) in enumerate(zip(self.widths, self.widths[1:]))]
        need = [tt.tt_policy_workspace_bytes(tokens, vocab, k, dtype, self.x[-1], self.g[-1]), tt.tt_policy_workspace_bytes(tokens, vocab, k, dtype, self.x[-1]),
                tt.tt_embed_workspace_bytes(tokens, vocab, self.widths[0], k, dtype, self.g[0], self.table)]
        for i in range(L):
            need.append(tt.tt_fc_workspace_bytes(self.lay[i], tokens, k, dtype, tt.TT_OP_FWD, self.x[i], self.w[i], self.x[i + 1], forms_a=self.forms[i][0]))
            need.append(tt.tt_fc_packed_workspace_bytes(self.lay[i], tokens, k, dtype, self.x[i], self.w[i], self.x[i + 1], self.g[i + 1], self.g[i],
                                                        self.forms[i][1], self.forms[i][2]))
        self.ws = torch.empty(max(256, max(need)), dtype=torch.uint8, device=DEV)
        self.scale = self.widths[0] ** 0.5

    def forward(self, ids, keep=False):
        """logits' shards; keep: also what the backward pass needs, every activation but the logits in 8 bits"""
        T, kept = self.tokens, []
        X = empty(T, self.widths[0], self.x[0], self.torch_dtype)
        tt.tt_embed_forward(T, self.vocab, self.widths[0], self.k, self.dtype, self.table, self.x[0], ids, self.scale, self.E, X)
        for i, lay in enumerate(self.lay):
            if keep:
                Q = [torch.empty(s.shape, dtype=torch.int8, device=DEV) for s in X]
                S = [torch.empty((s.shape[0], -(-s.shape[1] // tt.TT_PACK8_BLOCK)), dtype=torch.uint8, device=DEV) for s in X]
                tt.tt_pack8(T, self.widths[i], self.k, self.dtype, self.x[i], X, Q, S)
                kept.append((Q, S))
            Y = empty(T, self.widths[i + 1], self.x[i + 1], self.torch_dtype)
            tt.tt_fc_forward(lay, T, self.k, self.dtype, self.x[i], self.w[i], self.x[i + 1], self.forms[i][0], X, self.W[i], Y, self.ws)
            X = Y
        return (X, kept) if keep else X

    def logp(self, logits, actions):
        out = torch.empty(self.tokens, device=DEV)
        tt.tt_token_logp(self.tokens, self.vocab, self.k, self.dtype, self.x[-1], 1.0, logits, actions, out, self.ws)
        return out

    def gradients(self, params, ids, actions, old, ref, advantage, weight):
        """loss, and the gradients of the table and of the layers' weights"""
        T, k, dt = self.tokens, self.k, self.dtype
        logits, kept = self.forward(ids, keep=True)
        loss, logp = torch.empty(1, device=DEV), torch.empty(T, device=DEV)
        G = empty(T, self.vocab, self.g[-1], self.torch_dtype)
        tt.tt_policy_loss(params, T, self.vocab, k, dt, self.x[-1], self.g[-1], logits, actions, old, ref, advantage, weight, loss, logp, G, self.ws)
        dW = [None] * self.layers
        for i in reversed(range(self.layers)):
            dX = empty(T, self.widths[i], self.g[i], self.torch_dtype)
            dW[i] = empty(self.widths[i], self.widths[i + 1], self.w[i], self.torch_dtype)
            Q, S = kept[i]
            YQ, YS = kept[i + 1] if i + 1 < self.layers else (None, None)     # (no ReLU behind the last layer)
            tt.tt_fc_backward_packed(self.lay[i], T, k, dt, self.x[i], self.w[i], self.x[i + 1], self.g[i + 1], self.g[i], self.forms[i][1], self.forms[i][2],
                                     Q, S, self.W[i], YQ, YS, G, dX, dW[i], self.ws)
            G = dX
        dE = empty(self.vocab, self.widths[0], self.table, self.torch_dtype)
        tt.tt_embed_backward(T, self.vocab, self.widths[0], k, dt, self.g[0], self.table, ids, self.scale, G, dE, self.ws)
        return loss, dE, dW

    def descend(self, dE, dW, rate):
        for p, d in zip(self.E + sum(self.W, []), dE + sum(dW, [])):
            p.sub_(d, alpha=rate)


def train(steps=60, vocab=64, widths=(64, 256), tokens=1024, k=2, updates=4, rate=0.3, seed=1, report=print):
    policy = TokenPolicy(vocab, widths, tokens, k, seed=seed)
    params = tt.policy(clip_low=0.2, clip_high=0.3, kl=0.01)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rewards = []
    for step in range(steps):
        ids = torch.randint(0, vocab, (tokens,), generator=gen, device=DEV)
        logits = policy.forward(ids)
        z = join(logits, policy.x[-1], tokens, vocab).float()
        u = torch.rand(z.shape, generator=gen, device=DEV).clamp_(1e-9, 1 - 1e-7)
        actions = (z - torch.log(-torch.log(u))).argmax(1)      # (a draw from softmax(z))
        reward = (actions == (5 * ids + 3) % vocab).float()
        old = policy.logp(logits, actions)
        advantage = (reward - reward.mean()) / (reward.std() + 1e-3)
        weight = torch.full((tokens,), 1.0 / tokens, device=DEV)
        for _ in range(updates):
            loss, dE, dW = policy.gradients(params, ids, actions, old, old, advantage, weight)
            policy.descend(dE, dW, rate / (1 + 0.02 * step))
        rewards.append(reward.mean())
        if report and step % 10 == 0:
            report("step %3d  reward %.3f  loss %+.4f" % (step, float(rewards[-1]), float(loss)))
    return policy, [float(r) for r in rewards]


if __name__ == "__main__":
    _, r = train(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
    print("mean reward: first 10 steps %.3f, last 10 steps %.3f" % (sum(r[:10]) / 10, sum(r[-10:]) / 10))
