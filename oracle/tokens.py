"""Plain 64-bit forms of what surrounds a chain that trains a token model: the embedding and its table's gradient, token log
probabilities, the clipped policy loss with its KL term, and the 8-bit form of activations.  Untiled; loops over tokens and
blocks."""
import math

import numpy as np


def embed_forward(W, ids, scale):
    X = np.zeros((len(ids), W.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < W.shape[0]:
            X[t] = scale * W[v]
    return X


def embed_backward(dX, ids, vocab, scale):
    """returns the table's gradient and, for error bounds, the sums of magnitudes and the number of terms"""
    dW, mag, n = np.zeros((vocab, dX.shape[1])), np.zeros((vocab, dX.shape[1])), np.zeros(vocab, dtype=np.int64)
    for t, v in enumerate(ids):
        if 0 <= v < vocab:
            dW[v] += scale * dX[t]
            mag[v] += abs(scale) * np.abs(dX[t])
            n[v] += 1
    return dW, mag, n


def counts(x, a, w=1.0):
    """whether a token counts: a weight, a token of the vocabulary, a logit above -inf"""
    return w != 0 and 0 <= a < len(x) and not np.all(x == -np.inf)


def log_softmax(z):
    with np.errstate(invalid="ignore"):
        m = np.max(z)
        return z - m - math.log(np.sum(np.exp(z - m))) if not np.isnan(m) and m != np.inf else np.full(len(z), np.nan)


def token_logp(X, ids, scale):
    return np.array([log_softmax(scale * x)[a] if counts(x, a) else 0.0 for x, a in zip(X, ids)])


def policy_term(logp, old, ref, adv, clip_low, clip_high, kl):
    """a token's loss as a function of its log probability"""
    ratio = math.exp(logp - old)
    loss = -min(ratio * adv, min(max(ratio, 1 - clip_low), 1 + clip_high) * adv)
    if kl:
        loss += kl * (math.exp(ref - logp) - 1 - (ref - logp))
    return loss


def policy_loss(X, actions, old, ref, adv, weight, scale, clip_low, clip_high, kl):
    """(loss, log probabilities, gradient of the logits, derivative by the log probability of each token)"""
    T, V = X.shape
    loss, logp, dX, d = 0.0, np.zeros(T), np.zeros((T, V)), np.zeros(T)
    for t in range(T):
        if not counts(X[t], actions[t], weight[t]):
            continue
        a = int(actions[t])
        ls = log_softmax(scale * X[t])
        logp[t] = ls[a]
        r = ref[t] if kl else 0.0
        loss += weight[t] * policy_term(ls[a], old[t], r, adv[t], clip_low, clip_high, kl)
        ratio = math.exp(ls[a] - old[t])
        clipped = (adv[t] > 0 and ratio > 1 + clip_high) or (adv[t] < 0 and ratio < 1 - clip_low)
        d[t] = (0.0 if clipped else -ratio * adv[t]) + (kl * (1 - math.exp(r - ls[a])) if kl else 0.0)
        g = -np.exp(ls)
        g[a] += 1
        dX[t] = weight[t] * d[t] * scale * g
    return loss, logp, dX, d


def pack8(X, block=32):
    """(Q, S): whole steps, and the exponents of the steps plus 127, one per block of a row"""
    rows, cols = X.shape
    Q, S = np.zeros((rows, cols), dtype=np.int8), np.zeros((rows, -(-cols // block)), dtype=np.uint8)
    for r in range(rows):
        for b in range(S.shape[1]):
            x = X[r, b * block:(b + 1) * block]
            if not np.all(np.isfinite(x)):
                S[r, b] = 255
                continue
            e = -126
            while np.max(np.abs(x)) > 127 * 2.0 ** e:
                e += 1
            for i, v in enumerate(x):
                q = round(v / 2.0 ** e)                 # (to nearest, ties to even)
                Q[r, b * block + i] = q if q != 0 or v == 0 else (1 if v > 0 else -1)
            S[r, b] = e + 127
    return Q, S


def unpack8(Q, S, block=32):
    step = np.where(S == 255, np.nan, 2.0 ** (S.astype(np.float64) - 127))
    return Q.astype(np.float64) * np.repeat(step, block, axis=1)[:, :Q.shape[1]]
