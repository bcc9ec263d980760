"""The token operators (embedding and its gradient, policy loss, activations in 8 bits) against their plain 64-bit forms.

Bounds, from the arithmetic the kernels are said to do (eps = 2^-24, half a step of fp32 next to 1; a bf16 result adds half a step
of bf16, which has 8 significant bits: 2^-8 of its value):
  embedding            one fp32 product: eps |z|
  table gradient       n fp32 additions and one product: (n + 1) eps sum |terms|
  log probabilities    statistics in fp32.  The logits' factor and each exponent are rounded (2 eps of the distance from the
                       maximum: |logp| + log V covers it), the sum is one of chains of at most 256 additions and a tree over them,
                       the logarithm is good to a step: 4 eps (2 |logp| + 2 log V + 160)
  loss                 the terms' derivatives times that, and 64 eps of the sum of magnitudes
  logits' gradient     the derivative's error from the log probability's, and the softmax's relative one, eps-wise as above
  8-bit form           exact
"""
import ctypes
import math
import mmap

import numpy as np
import pytest
import torch

import paper_1805_04170_amd as tt
from oracle import layers as ly
from oracle import tiling as tl
from oracle import tokens as tk
from synthetic import bf16_bits_to_f64, normal_f32, to_bf16_bits

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
EPS = 2.0 ** -24
GUARD = "end"       # host runs: which side of a buffer the inaccessible page lies on
_libc = None


def _guarded(nbytes):
    """host memory whose neighbour page (behind it, or in front of it) cannot be touched"""
    global _libc
    _libc = _libc or ctypes.CDLL(None, use_errno=True)
    page = mmap.PAGESIZE
    body = max(page, -(-nbytes // page) * page)
    m = mmap.mmap(-1, body + 2 * page)
    raw = torch.frombuffer(m, dtype=torch.uint8)
    base = raw.data_ptr()
    for at in (base, base + page + body):
        assert _libc.mprotect(ctypes.c_void_p(at), ctypes.c_size_t(page), 0) == 0
    lo = page + (body - nbytes if GUARD == "end" else 0)
    return raw[lo:lo + nbytes]


def empty(shape, dtype, skew=0):
    """a buffer full of 0x5a bytes; skew: elements by which it is off a 256-byte boundary (device runs)"""
    e = torch.empty(0, dtype=dtype).element_size()
    n = int(np.prod(shape))
    if DEV == "cpu":
        raw = _guarded(n * e)
    else:
        raw = torch.empty(max(1, (n + skew) * e), dtype=torch.uint8, device=DEV)[skew * e:]
    raw.fill_(0x5a)
    if n == 0:
        return torch.empty(shape, dtype=dtype, device=DEV)
    return raw[:n * e].view(dtype).view(shape)


def up(a, skew=0):
    """numpy array to the device; uint16 travels as bf16"""
    t = torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16) if a.dtype == np.uint16 else torch.from_numpy(np.ascontiguousarray(a))
    out = empty(tuple(t.shape), t.dtype, skew)
    out.copy_(t)
    return out


def down(t):
    return bf16_bits_to_f64(t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)) if t.dtype == torch.bfloat16 else t.cpu().numpy()


def stored(a, dt):
    """what a tensor of type dt holds of the values: (array to upload, the same in 64 bits)"""
    a = a.astype(np.float32)
    if dt == "bf16":
        bits = to_bf16_bits(a)
        return bits, bf16_bits_to_f64(bits)
    return a, a.astype(np.float64)


def shards(a, t, skew=0):
    return [up(s, skew) for s in tl.tile(a, t)]


def outputs(rows, cols, t, dt, skew=0):
    sr, sc = tl.shard_shape(rows, cols, t)
    return [empty((sr, sc), torch.bfloat16 if dt == "bf16" else torch.float32, skew) for _ in range(1 << len(t))]


def full(sh, t, rows, cols):
    return tl.untile([down(s) for s in sh], t, rows, cols)


def workspace(nbytes):
    return empty((max(256, nbytes),), torch.uint8)


def out_eps(dt):
    return 2.0 ** -8 if dt == "bf16" else 0.0


def check(got, want, bound, what):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])


def ids_of(values, idt):
    return up(np.asarray(values, dtype=np.int32 if idt == "i32" else np.int64))


# --------------------------------------------------------------- embedding

def run_embed(T, V, D, dt, tW="", tX="", idt="i64", seed=1, ids=None, scale=None, skew=0):
    rng = np.random.default_rng(seed)
    k = len(tW)
    scale = math.sqrt(D) if scale is None else scale
    if ids is None:
        ids = np.minimum((np.exp(rng.random(T) * math.log(V + 1)) - 1).astype(np.int64), V - 1)
        ids = np.where(rng.random(T) < 0.1, -1, ids)
    W, Wf = stored(normal_f32(seed, 0, (V, D), 0.5), dt)
    G, Gf = stored(normal_f32(seed, 1, (T, D), 0.5), dt)
    d_ids = ids_of(ids, idt)
    Xs = outputs(T, D, tX, dt, skew)
    tt.tt_embed_forward(T, V, D, k, dt, tW, tX, d_ids, scale, shards(W, tW, skew), Xs)
    s32 = float(np.float32(scale))
    want = tk.embed_forward(Wf, ids, s32)
    check(full(Xs, tX, T, D), want, (EPS + out_eps(dt) * (1 + EPS)) * np.abs(want), "X")
    dWs = outputs(V, D, tW, dt, skew)
    ws = workspace(tt.tt_embed_workspace_bytes(T, V, D, k, dt, tX, tW))
    Gs = shards(G, tX, skew)
    tt.tt_embed_backward(T, V, D, k, dt, tX, tW, d_ids, scale, Gs, dWs, ws)
    want, mag, n = tk.embed_backward(Gf, ids, V, s32)
    err = (n[:, None] + 1) * EPS * mag
    check(full(dWs, tW, V, D), want, err + out_eps(dt) * (np.abs(want) + err), "dW")
    again = outputs(V, D, tW, dt, skew)
    ws.fill_(0xa5)
    tt.tt_embed_backward(T, V, D, k, dt, tX, tW, d_ids, scale, Gs, again, ws)
    for a, b in zip(dWs, again):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (1, 5, 8), (7, 40, 33), (65, 300, 64), (130, 17, 250), (257, 1031, 72)])
def test_embedding(T, V, D, dt):
    run_embed(T, V, D, dt, seed=T)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,D", [(40, 20, 600), (129, 300, 2052), (200, 3, 1031), (3, 1000, 4100)])
def test_embedding_of_wide_rows(T, V, D, dt):
    run_embed(T, V, D, dt, seed=D)


@pytest.mark.parametrize("tW,tX,D", [("C", "R", 1200), ("RC", "Cr", 2064), ("CC", "RR", 4200)])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_embedding_of_wide_rows_tiled(tW, tX, D, dt):
    run_embed(100, 40, D, dt, tW, tX, seed=D)


def test_embedding_of_large_vocabularies_and_many_tokens():
    run_embed(256, 1500, 300, "bf16", seed=5, ids=np.arange(256) % 3)
    run_embed(256, 1500, 30, "bf16", seed=5, ids=np.arange(256) // 100)
    run_embed(3000, 1500, 40, "f32", seed=5)
    run_embed(3000, 40, 600, "bf16", seed=5)
    run_embed(2000, 5000, 600, "f32", "RC", "CR", seed=6)
    run_embed(700, 270000, 3, "bf16", seed=6)      # more numbers than 256 workgroups' counters hold
    run_embed(20000, 7, 16, "f32", seed=7)


@pytest.mark.parametrize("tW,tX", [("R", "C"), ("C", "r"), ("r", "R"), ("RC", "CR"), ("rC", "Cr"), ("CC", "RR"), ("RCr", "CCC")])
@pytest.mark.parametrize("dt,D", [("bf16", 64), ("f32", 24), ("bf16", 40)])
def test_embedding_tiled(tW, tX, dt, D):
    run_embed(48, 96, D, dt, tW, tX, "i32", seed=len(tW) + D)


@pytest.mark.parametrize("what", ["one", "none", "two", "huge", "long_runs"])
def test_embedding_token_patterns(what):
    for T in (300, 200):
        run_patterns(T, what)


def run_patterns(T, what):
    V = 50
    rng = np.random.default_rng(4)
    ids = {"one": np.full(T, 49), "none": np.full(T, -1), "two": np.where(np.arange(T) % 2 == 0, 3, 4),
           "huge": np.where(np.arange(T) % 3 == 0, 2 ** 62, np.where(np.arange(T) % 3 == 1, -2 ** 62, V)),
           "long_runs": np.sort(rng.integers(0, 4, T))[::-1].copy()}[what].astype(np.int64)
    for D, dt in [(3, "f32"), (5, "bf16"), (20, "f32"), (140, "f32")]:
        run_embed(T, V, D, dt, ids=ids)


@pytest.mark.parametrize("T,V,D,dt", [(257, 1, 33, "bf16"), (256, 2, 40, "f32"), (300, 1, 7, "bf16"), (1024, 31, 9, "f32"), (16385, 3, 8, "bf16"), (258, 257, 1, "f32")])
def test_embedding_on_either_side_of_what_is_sorted(T, V, D, dt):
    run_embed(T, V, D, dt, seed=T)


@pytest.mark.parametrize("tW,tX,T", [("CCCCCC", "RRRRRR", 64), ("RCRCRC", "CrRrCR", 320), ("rrrrrr", "CCCCCC", 64)])
def test_embedding_of_six_cuts(tW, tX, T):
    run_embed(T, 64, 320, "bf16", tW, tX, seed=T)


def test_embedding_skewed_buffers():
    run_embed(33, 70, 48, "bf16", seed=8, skew=1)
    run_embed(34, 70, 48, "f32", "C", "R", seed=9, skew=3)


@pytest.mark.parametrize("scale", [math.inf, -math.inf, math.nan, -2.0])
@pytest.mark.parametrize("T", [40, 300])
def test_table_gradient_rows_without_tokens_are_zeros(T, scale):
    V = 50
    ids = np.where(np.arange(T) % 2 == 0, 3, np.arange(T) % 7 + 20)
    for D, dt in [(3, "f32"), (40, "bf16"), (300, "f32"), (1100, "bf16")]:
        G, Gf = stored(np.abs(normal_f32(D, 1, (T, D), 0.5)) + 0.25, dt)
        dW, ws = outputs(V, D, "", dt), workspace(tt.tt_embed_workspace_bytes(T, V, D, 0, dt, "", ""))
        tt.tt_embed_backward(T, V, D, 0, dt, "", "", ids_of(ids, "i32"), scale, [up(G)], dW, ws)
        there = np.isin(np.arange(V), ids)
        assert not dW[0].cpu()[torch.from_numpy(~there)].contiguous().view(torch.uint8).any(), (D, dt)     # (+0)
        with np.errstate(invalid="ignore"):
            want, mag, n = tk.embed_backward(Gf, ids, V, scale)
        if math.isfinite(scale):
            err = (n[:, None] + 1) * EPS * mag
            check(down(dW[0]), want, err + out_eps(dt) * (np.abs(want) + err), "dW")
        else:
            assert np.array_equal(down(dW[0])[there], want[there], equal_nan=True)


def test_a_workspace_for_many_tokens_covers_fewer():
    V, D = 40, 24
    G, dW = [up(normal_f32(3, 1, (16385, D), 0.5))], outputs(V, D, "", "f32")
    ws = workspace(tt.tt_embed_workspace_bytes(16385, V, D, 0, "f32", "", ""))
    ids = np.arange(16385) % V
    for T in (16385, 16384, 257, 100):
        tt.tt_embed_backward(T, V, D, 0, "f32", "", "", ids_of(ids[:T], "i64"), 1.0, [G[0][:T]], dW, ws)
        want, mag, n = tk.embed_backward(down(G[0])[:T].astype(float), ids[:T], V, 1.0)
        check(down(dW[0]), want, (n[:, None] + 1) * EPS * mag, T)
    T, V = 129, 20000
    raw, x = stored(normal_f32(4, 0, (T, V), 2.0), "bf16")
    a, ws = np.arange(T), workspace(tt.tt_policy_workspace_bytes(T, V, 0, "bf16", "", ""))
    want = tk.token_logp(x, a, 1.0)
    for n in (129, 128, 3):
        one, loss, logp, dX = np.ones(n, np.float32), empty((1,), torch.float32), empty((n,), torch.float32), outputs(n, V, "", "bf16")
        tt.tt_policy_loss(tt.policy(), n, V, 0, "bf16", "", "", [up(raw[:n])], ids_of(a[:n], "i64"), up(want[:n].astype(np.float32)), None, up(one), up(one), loss, logp, dX, ws)
        check(down(logp), want[:n], logp_bound(want[:n], V), n)


def test_embedding_without_tokens_is_a_gradient_of_zeros():
    dW = [empty((6, 5), torch.float32)]
    ws = workspace(tt.tt_embed_workspace_bytes(0, 6, 5, 0, "f32", "", ""))
    none = empty((1,), torch.int64)
    tt.tt_embed_backward(0, 6, 5, 0, "f32", "", "", none, 1.0, [empty((1, 5), torch.float32)], dW, ws)
    assert not down(dW[0]).any()


@pytest.mark.parametrize("T,V,D", [(0, 6, 5), (5, 0, 5), (0, 0, 5), (5, 6, 0)])
def test_embedding_of_tensors_without_values(T, V, D):
    none = lambda r, c: [torch.empty((r, c), dtype=torch.float32, device=DEV) if r * c == 0 else empty((r, c), torch.float32)]  # noqa: E731
    X, dW, ids = none(T, D), none(V, D), torch.zeros(T, dtype=torch.int64, device=DEV)
    tt.tt_embed_forward(T, V, D, 0, "f32", "", "", ids, 1.0, none(V, D), X)
    tt.tt_embed_backward(T, V, D, 0, "f32", "", "", ids, 1.0, none(T, D), dW, None)
    if V == 0 and T:
        assert not down(X[0]).any()
    if T == 0:
        assert not down(dW[0]).any()


# ------------------------------------------------------------- policy loss

def policy_inputs(T, V, dt, seed, scale, kl, masked):
    rng = np.random.default_rng(seed)
    raw, x = stored(normal_f32(seed, 0, (T, V), 2.0), dt)
    a = rng.integers(0, V, T)
    w = np.full(T, 1.0 / T, dtype=np.float32)
    if masked:
        def put(rows, cols, v):
            raw[rows, cols] = to_bf16_bits(np.full(1, v, np.float32))[0] if dt == "bf16" else v
            x[rows, cols] = v
        put(slice(None), slice(V - V // 7, None), -np.inf)
        a = rng.integers(0, max(1, V - V // 7), T)
        for t in range(T):
            if t % 5 == 1:
                w[t] = 0
                put(t, slice(None), [np.nan, np.inf, -np.inf, 1.0][t % 4])
            if t % 7 == 3:
                put(t, slice(None), -np.inf)
            if t % 11 == 6:
                a[t] = V if t % 2 else -1
            if t % 13 == 8:     # one logit left, and it is the action's
                keep = x[t, a[t]] if 0 <= a[t] < V else np.nan
                if np.isfinite(keep):
                    put(t, slice(None), -np.inf)
                    put(t, int(a[t]), keep)
    logp = tk.token_logp(np.where(np.isnan(x) | (x == np.inf), 0.0, x), a, scale)
    # ratios that stay away from where the clip begins, on both sides of it
    old = (logp - rng.choice([-0.5, -0.1, 0.0, 0.05, 0.4], T)).astype(np.float32)
    ref = (logp + rng.normal(0, 0.3, T)).astype(np.float32)
    adv = rng.normal(0, 1, T).astype(np.float32)
    adv[::9] = 0
    return raw, x, a, old, ref, adv, w


def logp_bound(logp, V):
    return 4 * EPS * (2 * np.abs(logp) + 2 * math.log(V + 1) + 160)


def run_policy(T, V, dt, tX="", tG="", idt="i64", seed=1, scale=1.0, kl=0.05, masked=False, with_dx=True, skew=0, clip=(0.2, 0.25)):
    k = len(tX)
    scale = float(np.float32(scale))
    raw, x, a, old, ref, adv, w = policy_inputs(T, V, dt, seed, scale, kl, masked)
    p = tt.policy(clip_low=clip[0], clip_high=clip[1], kl=kl, scale=scale)
    lo, hi, klf = (float(np.float32(v)) for v in (clip[0], clip[1], kl))
    loss, logp = empty((1,), torch.float32), empty((T,), torch.float32)
    Xs, dX = shards(raw, tX, skew), outputs(T, V, tG, dt, skew) if with_dx else None
    ws = workspace(tt.tt_policy_workspace_bytes(T, V, k, dt, tX, tG if with_dx else None))
    args = (up(old), up(ref) if kl else None, up(adv), up(w))
    d_a = ids_of(a, idt)
    tt.tt_policy_loss(p, T, V, k, dt, tX, tG, Xs, d_a, *args, loss, logp, dX, ws)
    want_loss, want_logp, want_dX, d = tk.policy_loss(x, a, old.astype(float), ref.astype(float), adv.astype(float), w.astype(float), scale, lo, hi, klf)
    live = np.array([tk.counts(x[t], a[t], w[t]) for t in range(T)])
    lb = np.where(live, logp_bound(want_logp, V), 0)
    check(down(logp), want_logp, lb, "logp")
    # dL/dlogp moves by (|ratio adv| + kl exp(ref - logp)) times the log probability's error; L itself by |dL/dlogp| times it
    ratio = np.exp(np.where(live, want_logp - old, 0))
    kle = klf * np.exp(np.where(live, ref - want_logp, 0)) if kl else 0 * ratio
    slope = np.abs(ratio * adv) + kle
    size = np.abs(ratio * adv) + kle * 2 + klf * np.abs(np.where(live, ref - want_logp, 0))
    wl = np.where(live, w, 0)
    check(down(loss)[0], want_loss, np.sum(wl * (slope * (lb + 16 * EPS) + 64 * EPS * size)), "loss")
    if with_dx:
        d_err = slope * (lb + 16 * EPS)
        z = np.where(np.isfinite(x) & live[:, None], scale * x, -np.inf)
        top = np.where(live, np.max(z, axis=1, initial=-1e30), 0)
        with np.errstate(invalid="ignore", divide="ignore"):
            away = np.where(np.isfinite(z), top[:, None] - z, 0)
            ls = np.where(live[:, None], z - top[:, None], -np.inf)
            prob = np.exp(ls) / np.maximum(np.sum(np.exp(ls), axis=1, keepdims=True), 1e-300)
        p_rel = 4 * EPS * (2 * away + 2 * math.log(V + 1) + 160)
        hot = np.zeros((T, V))
        hot[np.arange(T)[live], a[live]] = 1
        err = wl[:, None] * scale * (d_err[:, None] * (hot + prob) + np.abs(d)[:, None] * (prob * p_rel + 8 * EPS * hot)) + 1e-37
        check(full(dX, tG, T, V), want_dX, np.where(live[:, None], err + out_eps(dt) * (np.abs(want_dX) + err), 0), "dX")
        again, loss2, logp2 = outputs(T, V, tG, dt, skew), empty((1,), torch.float32), empty((T,), torch.float32)
        ws.fill_(0xa5)
        tt.tt_policy_loss(p, T, V, k, dt, tX, tG, Xs, d_a, *args, loss2, logp2, again, ws)
        for u, v in zip([loss, logp] + dX, [loss2, logp2] + again):
            assert torch.equal(u.view(torch.uint8), v.view(torch.uint8))
    return loss, logp


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", [(1, 1), (1, 2), (3, 7), (5, 64), (33, 1000), (4, 2051), (2, 8200)])
def test_policy_loss(T, V, dt):
    run_policy(T, V, dt, seed=T + V)


@pytest.mark.parametrize("T,V,dt", [(4300, 40, "f32"), (4200, 530, "bf16"), (2300, 1100, "f32"), (1100, 4200, "f32"), (560, 16600, "bf16"), (270, 66000, "bf16"),
                                    (258, 70000, "f32"), (3, 90000, "f32"), (2, 140001, "bf16"), (5, 160000, "bf16")])
def test_policy_loss_of_more_rows_than_workgroups_and_of_long_rows(T, V, dt):
    run_policy(T, V, dt, seed=V, masked=T < 4000)


@pytest.mark.parametrize("tX,tG,V", [("C", "R", 1100), ("CC", "RC", 4140), ("RC", "CC", 2084), ("CCCCC", "RRCCC", 17600)])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_policy_loss_of_long_rows_tiled(tX, tG, V, dt):
    run_policy(8, V, dt, tX, tG, "i32", seed=V, masked=True)


@pytest.mark.parametrize("tX,tG", [("C", "R"), ("R", "C"), ("r", "C"), ("CC", "RC"), ("CR", "rr"), ("rC", "Cr"), ("CCC", "RRC")])
@pytest.mark.parametrize("dt,V", [("bf16", 512), ("f32", 328), ("bf16", 104)])
def test_policy_loss_tiled(tX, tG, dt, V):
    run_policy(24, V, dt, tX, tG, "i32", seed=len(tX), masked=True, scale=0.7)


@pytest.mark.parametrize("tX,tG,V", [("CCCCCC", "RRRCCC", 640), ("RCRCRC", "CCCCCC", 4096 + 64), ("rrrrrr", "CrCrCr", 1024), ("CCCCCC", "CCCCCC", 64 * 600)])
def test_policy_loss_of_six_cuts(tX, tG, V):
    run_policy(64, V, "bf16", tX, tG, seed=V)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,kl", [(40, 50, 0.0), (60, 333, 0.05), (30, 1031, 0.3)])
def test_policy_loss_masked(T, V, kl, dt):
    run_policy(T, V, dt, seed=V, kl=kl, masked=True, scale=1.3)


def test_policy_loss_without_gradient_and_log_probabilities_alone():
    _, logp = run_policy(21, 300, "bf16", masked=False, with_dx=False)
    raw, x, a, *_ = policy_inputs(21, 300, "bf16", 1, 1.0, 0.05, False)
    out = empty((21,), torch.float32)
    ws = workspace(tt.tt_policy_workspace_bytes(21, 300, 0, "bf16", ""))
    tt.tt_token_logp(21, 300, 0, "bf16", "", 1.0, shards(raw, ""), ids_of(a, "i64"), out, ws)
    assert torch.equal(out, logp)


def run_logp(T, V, dt, tX="", seed=3, scale=1.0):
    rng = np.random.default_rng(seed)
    raw, x = stored(normal_f32(seed, 0, (T, V), 2.0), dt)
    a = rng.integers(-1, V + 1, T)
    out = empty((T,), torch.float32)
    ws = workspace(tt.tt_policy_workspace_bytes(T, V, len(tX), dt, tX))
    tt.tt_token_logp(T, V, len(tX), dt, tX, scale, shards(raw, tX), ids_of(a, "i32"), out, ws)
    want = tk.token_logp(x, a, float(np.float32(scale)))
    check(down(out), want, np.where((a >= 0) & (a < V), logp_bound(want, V), 0), "logp")


@pytest.mark.parametrize("T,V,dt,tX", [(1, 1, "f32", ""), (1, 4099, "bf16", ""), (3, 9000, "f32", ""), (8, 640, "bf16", "CC"), (6, 36, "bf16", "CR"), (4, 20, "f32", "CCr")])
def test_token_logp(T, V, dt, tX):
    run_logp(T, V, dt, tX, scale=0.8)


def test_policy_rows_that_count_show_their_nan():
    x = np.zeros((4, 40), np.float32)
    x[0, 3], x[1, 5], x[2, :] = np.nan, np.inf, np.nan
    one = np.ones(4, np.float32)
    loss, logp = empty((1,), torch.float32), empty((4,), torch.float32)
    dX, ws = outputs(4, 40, "", "f32"), workspace(tt.tt_policy_workspace_bytes(4, 40, 0, "f32", "", ""))
    tt.tt_policy_loss(tt.policy(), 4, 40, 0, "f32", "", "", shards(x, ""), ids_of([0] * 4, "i64"), up(0 * one), None, up(one), up(one), loss, logp, dX, ws)
    assert np.isnan(down(loss)).all()
    assert np.isnan(down(logp)[:3]).all() and abs(down(logp)[3] + math.log(40)) < 1e-5
    assert np.isnan(down(dX[0])[:3]).all() and np.isfinite(down(dX[0])[3]).all()


LOWEST = {"bf16": -3.3895313892515355e38, "f32": float(np.finfo(np.float32).min)}


def run_policy_of_large_logits(V, dt, mask, scale, tX="", tG="", with_dx=True):
    """Large finite logits, as masks leave them: rows of nothing but the mask, rows with a masked tail or with one entry left, an action
    that is ruled out, and rows whose largest logits are near the type's largest value.  No bound beyond run_policy's."""
    rng, T = np.random.default_rng(V), 8
    mask = LOWEST[dt] if mask is None else mask
    x = normal_f32(V, 0, (T, V), 2.0)
    a = rng.integers(0, max(1, V // 2), T)
    x[0] = mask
    x[1, V // 2:] = mask
    x[2] = mask
    x[2, a[2]] = 0.5
    x[3, 1:] = max(mask, -1e30)
    a[3] = V - 1                                # ruled out, unless it is all there is
    x[4, a[4]] = 2.5e38
    x[5] = 2.5e38
    x[6] = mask
    x[6, V // 3:] = mask / 2 if mask < -1e35 else mask - 1e4 * abs(mask) * 2.0 ** -8
    run_policy_of_logits(x, a, dt, scale, tX, tG, with_dx)


def run_policy_of_logits(x, a, dt, scale, tX="", tG="", with_dx=True):
    T, V = x.shape
    rng, scale, k = np.random.default_rng(V + T), float(np.float32(scale)), len(tX)
    raw, x = stored(x, dt)
    logp = tk.token_logp(x, a, scale)
    old = np.where(np.abs(logp) < 1e3, logp - rng.choice([-0.5, -0.1, 0.05, 0.4], T), 0).astype(np.float32)
    adv, w = rng.normal(0, 1, T).astype(np.float32), np.full(T, 1.0 / T, dtype=np.float32)
    p, lo, hi = tt.policy(clip_low=0.2, clip_high=0.25, scale=scale), float(np.float32(0.2)), float(np.float32(0.25))
    loss, got = empty((1,), torch.float32), empty((T,), torch.float32)
    dX = outputs(T, V, tG, dt) if with_dx else None
    Xs, d_a = shards(raw, tX), ids_of(a, "i64")
    ws = workspace(tt.tt_policy_workspace_bytes(T, V, k, dt, tX, tG if with_dx else None))
    tt.tt_policy_loss(p, T, V, k, dt, tX, tG, Xs, d_a, up(old), None, up(adv), up(w), loss, got, dX, ws)
    want_loss, want_logp, want_dX, d = tk.policy_loss(x, a, old.astype(float), old.astype(float), adv.astype(float), w.astype(float), scale, lo, hi, 0.0)
    lb = logp_bound(want_logp, V)

    def check_logp(got, what):      # (below the type's lowest value stands -inf)
        with np.errstate(over="ignore"):
            held = want_logp.astype(np.float32)
        low = np.isinf(held)
        assert np.array_equal(down(got)[low], held[low]), what
        check(down(got)[~low], want_logp[~low], lb[~low], what)
    check_logp(got, "logp")
    slope = np.abs(np.exp(want_logp - old) * adv)
    check(down(loss)[0], want_loss, np.sum(w * slope * (lb + 80 * EPS)), "loss")
    if with_dx:
        z = scale * x
        away = np.max(z, axis=1, keepdims=True) - z
        prob = np.exp(-away) / np.sum(np.exp(-away), axis=1, keepdims=True)
        hot = np.zeros((T, V))
        hot[np.arange(T), a] = 1
        p_rel = 4 * EPS * (2 * away + 2 * math.log(V + 1) + 160)
        err = w[:, None] * scale * ((slope * (lb + 16 * EPS))[:, None] * (hot + prob) + np.abs(d)[:, None] * (prob * p_rel + 8 * EPS * hot)) + 1e-37
        check(full(dX, tG, T, V), want_dX, err + out_eps(dt) * (np.abs(want_dX) + err), "dX")
    alone = empty((T,), torch.float32)
    ws = workspace(tt.tt_policy_workspace_bytes(T, V, k, dt, tX))
    tt.tt_token_logp(T, V, k, dt, tX, scale, Xs, d_a, alone, ws)
    check_logp(alone, "logp alone")


MASKS = [-5e9, -1e10, -1e15, -1e20, -1e30, -1e38, None]


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_policy_loss_of_large_finite_masks(dt, mask):
    for V, scale in [(40, 1.0), (600, 0.5), (600, 2.0), (4500, 1.0), (40, 4.0), (9, 1e-30)]:
        run_policy_of_large_logits(V, dt, mask, scale)
        run_policy_of_large_logits(V, dt, mask, scale, with_dx=False)


@pytest.mark.parametrize("mask", [-1e10, -1e30, None])
@pytest.mark.parametrize("V,dt,tX,tG", [(17000, "bf16", "", ""), (9000, "f32", "", ""), (90000, "f32", "", ""), (170000, "bf16", "", ""), (24, "bf16", "CC", "CC"),
                                        (4140, "f32", "CC", "RC"), (600, "bf16", "CCC", "RRr")])
def test_policy_loss_of_large_finite_masks_in_every_form(V, dt, tX, tG, mask):
    run_policy_of_large_logits(V, dt, mask, 1.0, tX, tG)
    run_policy_of_large_logits(V, dt, mask, 0.7, tX, tG, with_dx=False)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_policy_loss_of_large_finite_masks_many_rows(dt):
    """forms that take other kernels for many rows, each row a block of one mask and the rest ordinary"""
    for T, V in [(300, 40), (300, 2000), (260, 20000)]:
        x = normal_f32(T, 0, (T, V), 2.0)
        x[:, V // 2:] = np.array([-1e10, -1e20, LOWEST[dt], -np.inf], np.float32)[np.arange(T) % 4][:, None]
        whole = np.arange(T) % 7 == 3
        x[whole] = LOWEST[dt]
        raw, x = stored(x, dt)
        a = np.random.default_rng(T).integers(0, V // 2, T)
        want = tk.token_logp(x, a, 1.0)
        Xs, d_a, one = shards(raw, ""), ids_of(a, "i32"), np.ones(T, np.float32)
        for with_dx in (True, False):
            loss, logp, dX = empty((1,), torch.float32), empty((T,), torch.float32), outputs(T, V, "", dt) if with_dx else None
            ws = workspace(tt.tt_policy_workspace_bytes(T, V, 0, dt, "", "" if with_dx else None))
            tt.tt_policy_loss(tt.policy(), T, V, 0, dt, "", "", Xs, d_a, up(want.astype(np.float32)), None, up(one), up(one), loss, logp, dX, ws)
            check(down(logp), want, logp_bound(want, V), "logp")
            # all ratios are 1: the loss is -1 a row, the gradient p - onehot
            check(down(loss)[0], -float(T), T * (np.max(logp_bound(want, V)) + 64 * EPS), "loss")
            if with_dx:
                g = down(dX[0])
                lb = logp_bound(want, V)[:, None]
                prob = np.exp(x - np.max(x, 1, keepdims=True))
                prob /= np.sum(prob, 1, keepdims=True)
                prob[np.arange(T), a] -= 1
                away = np.minimum(np.max(x, 1, keepdims=True) - x, 200)
                err = np.abs(prob) * 4 * EPS * (2 * away + 2 * math.log(V + 1) + 160) + 2 * lb * np.abs(prob) + 1e-37
                err[np.arange(T), a] += 2 * lb[:, 0] + 8 * EPS
                check(g, prob, err + out_eps(dt) * (np.abs(prob) + err), "dX")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_policy_loss_of_large_logits_a_few_steps_apart(dt):
    step = 2.0 ** -8 if dt == "bf16" else 2.0 ** -23
    for V, scale in [(60, 1.0), (700, 0.3)]:
        base = np.array([1e2, -1e3, 3e4, -1e5, 9e5, -2e6, 5e7, -3e9, 7e12, -1e30, 1e38], np.float64)
        away = np.random.default_rng(V).integers(0, 6, (len(base), V))
        x = base[:, None] - np.exp2(np.floor(np.log2(np.abs(base))))[:, None] * step * away
        x[:, 3] = base
        run_policy_of_logits(x.astype(np.float32), np.full(len(base), 3), dt, scale)


def test_policy_loss_at_the_ends_of_the_scale():
    """a factor next to the type's largest value: the maximum has probability 1 over its number, everything else none"""
    x = np.zeros((2, 50), np.float32)
    x[0, 7] = 1.0
    raw, x = stored(x, "f32")
    for scale, want in [(3.4e38, [0.0, -math.log(50)]), (1e-45, [-math.log(50)] * 2)]:
        out, ws = empty((2,), torch.float32), workspace(tt.tt_policy_workspace_bytes(2, 50, 0, "f32", ""))
        tt.tt_token_logp(2, 50, 0, "f32", "", scale, shards(raw, ""), ids_of([7, 7], "i64"), out, ws)
        check(down(out), np.array(want), logp_bound(np.array(want), 50), "logp")


@pytest.mark.parametrize("V", [8000, 33000])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_log_probabilities_are_off_to_both_sides(dt, V):
    """No bias: the logits' factor is rounded (to 1.3e-8 of it here), but for the action and for the sum alike.  The mean error of 4096
    rows is within half a step of fp32 next to 1 (eps / 2 = 3e-8) and four times what roundings of single ones leave of it."""
    T = 4096
    x = normal_f32(V, 0, (T, V), 2.5)
    a = np.random.default_rng(V).integers(0, V, T)
    x[np.arange(T), a] += 8
    raw, x = stored(x, dt)
    z = torch.from_numpy(x).to(DEV)
    want = (z.gather(1, torch.from_numpy(a).to(DEV)[:, None])[:, 0] - torch.logsumexp(z, 1)).cpu().numpy()
    one, loss, logp, dX = np.ones(T, np.float32), empty((1,), torch.float32), empty((T,), torch.float32), outputs(T, V, "", dt)
    Xs, d_a = shards(raw, ""), ids_of(a, "i64")
    ws = workspace(max(tt.tt_policy_workspace_bytes(T, V, 0, dt, "", ""), tt.tt_policy_workspace_bytes(T, V, 0, dt, "")))
    tt.tt_policy_loss(tt.policy(), T, V, 0, dt, "", "", Xs, d_a, up(want.astype(np.float32)), None, up(one), up(one), loss, logp, dX, ws)
    alone = empty((T,), torch.float32)
    tt.tt_token_logp(T, V, 0, dt, "", 1.0, Xs, d_a, alone, ws)
    for got in (logp, alone):
        off = down(got).astype(np.float64) - want
        assert abs(np.mean(off)) < EPS / 2 + 4 * np.std(off) / math.sqrt(T), np.mean(off)


@pytest.mark.parametrize("dt,V", [("bf16", 8000), ("bf16", 60000), ("f32", 8000)])
def test_what_rounding_leaves_out_of_joined_sums_is_not_the_same_in_every_row(dt, V):
    """bf16's largest logits lie at a few distances from each other, whose products with the factor are rounded alike in all rows.  Of
    16384 rows' mean error an eighth of a step of fp32 is left for what is common to them, and four times what single roundings leave."""
    T, kind = 16384, torch.bfloat16 if dt == "bf16" else torch.float32
    gen = torch.Generator(device=DEV).manual_seed(V)
    x = torch.empty((T, V), dtype=kind, device=DEV).normal_(0, 2.5, generator=gen)
    a = torch.randint(0, V, (T,), generator=gen, device=DEV)
    x[torch.arange(T, device=DEV), a] = torch.empty(T, dtype=kind, device=DEV).normal_(8, 2.5, generator=gen)
    want = torch.cat([(z.gather(1, i[:, None])[:, 0] - torch.logsumexp(z, 1)) for z, i in ((x[t:t + 1024].double(), a[t:t + 1024]) for t in range(0, T, 1024))])
    logp, ws = empty((T,), torch.float32), workspace(tt.tt_policy_workspace_bytes(T, V, 0, dt, "", ""))
    one, loss, dX = torch.ones(T, device=DEV), empty((1,), torch.float32), [torch.empty_like(x)]
    tt.tt_policy_loss(tt.policy(), T, V, 0, dt, "", "", [x], a, want.float(), None, one, one, loss, logp, dX, ws)
    off = (logp.double() - want).cpu().numpy()
    assert abs(np.mean(off)) < EPS / 8 + 4 * np.std(off) / math.sqrt(T), np.mean(off)


def test_policy_loss_of_no_tokens_is_zero():
    loss = empty((1,), torch.float32)
    none = empty((1,), torch.float32)
    tt.tt_policy_loss(tt.policy(), 0, 40, 0, "f32", "", "", [none], empty((1,), torch.int64), none, None, none, none, loss, none, [none], workspace(256))
    assert down(loss)[0] == 0


@pytest.mark.parametrize("T,V", [(0, 40), (3, 0), (0, 0)])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_policy_loss_of_tensors_without_values(T, V, dt):
    name = "f32" if dt == torch.float32 else "bf16"
    X, per, a = [torch.empty((T, V), dtype=dt, device=DEV)], torch.ones(T, device=DEV), torch.zeros(T, dtype=torch.int64, device=DEV)
    loss, logp, dX = empty((1,), torch.float32), empty((T,), torch.float32), [torch.empty((T, V), dtype=dt, device=DEV)]
    ws = workspace(tt.tt_policy_workspace_bytes(T, V, 0, name, "", ""))
    tt.tt_policy_loss(tt.policy(kl=0.1), T, V, 0, name, "", "", X, a, per, per, per, per, loss, logp, dX, ws)
    assert down(loss)[0] == 0 and not down(logp).any()
    tt.tt_token_logp(T, V, 0, name, "", 1.0, X, a, logp, ws)
    assert not down(logp).any()


# ------------------------------------------------ activations in 8 bits

def run_pack(rows, cols, dt, t="", seed=1, values=None, skew=0):
    k = len(t)
    a = normal_f32(seed, 0, (rows, cols), 1.0) * np.exp(normal_f32(seed, 1, (1, cols), 2.0)) if values is None else values
    raw, x = stored(a, dt)
    sr, sc = tl.shard_shape(rows, cols, t)
    n = 1 << k
    Q, S = [empty((sr, sc), torch.int8) for _ in range(n)], [empty((sr, -(-sc // 32)), torch.uint8) for _ in range(n)]
    tt.tt_pack8(rows, cols, k, dt, t, shards(raw, t, skew), Q, S)
    X = outputs(rows, cols, t, dt, skew)
    tt.tt_unpack8(rows, cols, k, dt, t, Q, S, X)
    for s, xs in enumerate(tl.tile(x, t)):
        q, e = tk.pack8(xs)
        assert np.array_equal(down(S[s]), e), s
        assert np.array_equal(down(Q[s]), q), s
        v = tk.unpack8(q, e)
        got = down(X[s])
        assert np.array_equal(got, v, equal_nan=True), s
        fine = np.isfinite(v)
        assert np.array_equal(np.sign(v[fine]), np.sign(xs[fine]))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 16), (3, 31), (5, 33), (7, 64), (2, 200), (9, 47)])
def test_pack8(rows, cols, dt):
    run_pack(rows, cols, dt, seed=cols)


@pytest.mark.parametrize("t", ["R", "C", "r", "RC", "CCr", "RCRCRC"])
def test_pack8_tiled(t):
    run_pack(16, 96 if len(t) < 6 else 320, "bf16", t)
    run_pack(16, 88, "f32", t)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_pack8_values_at_the_edges(dt):
    tiny, big = 1e-45, 3.3e38
    rows = [[127.0, 126.5, 0.5, -0.5, 1.5, 2.5, 0.4, -0.4, 1e-30], [127.00001, 1, -1, 0.2], [255, 254, 253, -127.5], [128, 64.5, 63.5], [0] * 5, [-0.0, 0.0],
            [tiny, 2 * tiny, -tiny], [big, -big, 1, tiny], [np.nan, 1, 2], [np.inf, 1], [1, -np.inf], [2.0 ** -120, 2.0 ** -126, 2.0 ** -119.3],
            [1.984375], [1.98438], [1.9843], [63.5 * 2.0 ** 121]]
    a = np.zeros((len(rows), 40), np.float32)
    for i, r in enumerate(rows):
        a[i, :len(r)] = r
        a[i, 39] = 3.0
    run_pack(len(rows), 40, dt, values=a)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [64, 40])
def test_unpack8_takes_any_step(cols, dt):
    """all bytes as Q under all scales, those that packing never makes too; the backward pass's gates go by the same values"""
    S = np.repeat(np.arange(256, dtype=np.uint8)[:, None], -(-cols // 32), axis=1)
    Q = np.arange(-128, 128)[(np.arange(256)[:, None] * 7 + np.arange(cols)) % 256].astype(np.int8)
    X = outputs(256, cols, "", dt)
    tt.tt_unpack8(256, cols, 0, dt, "", [up(Q)], [up(S)], X)
    want = tk.unpack8(Q, S)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    assert np.array_equal(down(X[0]), want, equal_nan=True)
    lay, (W, Wf) = tt.layer("fc", "relu", 16, cols), stored(np.ones((16, cols), np.float32), dt)
    XQ, XS, (dY, dYf) = np.zeros((256, 16), np.int8), np.full((256, 1), 127, np.uint8), stored(normal_f32(1, 0, (256, cols), 1.0), dt)
    XQ[np.arange(256), np.arange(256) % 16] = 1
    dX, dW = outputs(256, 16, "", dt), outputs(16, cols, "", dt)
    ws = workspace(tt.tt_fc_packed_workspace_bytes(lay, 256, 0, dt, "", "", "", "", ""))
    tt.tt_fc_backward_packed(lay, 256, 0, dt, "", "", "", "", "", None, None, [up(XQ)], [up(XS)], [up(W)], [up(Q)], [up(S)], [up(dY)], dX, dW, ws)
    with np.errstate(invalid="ignore"):
        G = dYf * (want > 0)
    bound = lambda v, m: (1e-4 if dt == "bf16" else 1e-5) * m + 2 * out_eps(dt) * np.abs(v)  # noqa: E731
    check(down(dX[0]), G @ Wf.T, bound(G @ Wf.T, ly.abs_product(G, Wf.T)), "dX")


def test_pack8_skewed_buffers():
    run_pack(6, 70, "bf16", skew=1)
    run_pack(6, 70, "f32", skew=3)


def run_packed_backward(b, ni, no, dt, relu, tX, tW, tY, tdY, tdX, fd=None, fw=None, with_dx=True, seed=1, nan=False):
    k = len(tX)
    lay = tt.layer("fc", "relu" if relu else "none", ni, no)
    pack = lambda a, t: [tk.pack8(s) for s in tl.tile(a, t)]  # noqa: E731
    value = lambda ps, t, r, c: tl.untile([tk.unpack8(*p) for p in ps], t, r, c)  # noqa: E731
    Y = normal_f32(seed, 1, (b, no), 1.0)
    if nan:
        Y[1, 3] = np.inf
    X8, Y8 = pack(stored(normal_f32(seed, 0, (b, ni), 1.0), dt)[1], tX), pack(stored(Y, dt)[1], tY)
    W, Wf = stored(normal_f32(seed, 2, (ni, no), 0.1), dt)
    dY, dYf = stored(normal_f32(seed, 3, (b, no), 1.0), dt)
    dX, dW = outputs(b, ni, tdX, dt) if with_dx else None, outputs(ni, no, tW, dt)
    ws = workspace(tt.tt_fc_packed_workspace_bytes(lay, b, k, dt, tX, tW, tY, tdY, tdX, fd, fw, with_dx))
    lists = [[up(p[i]) for p in ps] for ps in (X8, Y8) for i in (0, 1)]
    Ws, dYs = shards(W, tW), shards(dY, tdY)
    tt.tt_fc_backward_packed(lay, b, k, dt, tX, tW, tY, tdY, tdX, fd, fw, lists[0], lists[1], Ws, lists[2] if relu else None, lists[3] if relu else None,
                             dYs, dX, dW, ws)
    Xv, Yv = value(X8, tX, b, ni), value(Y8, tY, b, no)
    with np.errstate(invalid="ignore"):
        G = dYf * (Yv > 0) if relu else dYf
    rel = 1e-4 if dt == "bf16" else 1e-5        # the shard products' own bounds
    if with_dx:
        want = G @ Wf.T
        check(full(dX, tdX, b, ni), want, rel * ly.abs_product(G, Wf.T) + 2 * out_eps(dt) * np.abs(want), "dX")
    want = Xv.T @ G
    check(full(dW, tW, ni, no), want, rel * ly.abs_product(Xv.T, G) + 2 * out_eps(dt) * np.abs(want), "dW")
    # and the 16-bit pass on the unpacked activations, bit for bit
    def unpacked(q, s, r, c, t):
        out = outputs(r, c, t, dt)
        tt.tt_unpack8(r, c, k, dt, t, q, s, out)
        return out
    Xu, Yu = unpacked(lists[0], lists[1], b, ni, tX), unpacked(lists[2], lists[3], b, no, tY)
    dX2, dW2 = outputs(b, ni, tdX, dt) if with_dx else None, outputs(ni, no, tW, dt)
    ws2 = workspace(tt.tt_fc_workspace_bytes(lay, b, k, dt, tt.TT_OP_DGRAD, tX, tW, tY, tdY, tdX, fd, fw, with_dx))
    tt.tt_fc_backward(lay, b, k, dt, tX, tW, tY, tdY, tdX, fd, fw, Xu, Ws, Yu, dYs, dX2, dW2, ws2)
    for u, v in zip((dX or []) + dW, (dX2 or []) + dW2):
        assert torch.equal(u.view(torch.uint8), v.view(torch.uint8))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("relu", [True, False])
def test_packed_backward_untiled(dt, relu):
    run_packed_backward(24, 48, 40, dt, relu, "", "", "", "", "")
    run_packed_backward(5, 17, 9, dt, relu, "", "", "", "", "", with_dx=False)


@pytest.mark.parametrize("t", [("R", "r", "R", "R", "R"), ("r", "C", "C", "C", "R"), ("C", "R", "r", "R", "C"), ("CC", "RR", "CR", "RC", "Cr"),
                               ("CCC", "RRR", "CCr", "CCr", "CCC")])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_packed_backward_tiled(t, dt):
    run_packed_backward(16, 64, 72 if len(t[0]) < 3 else 64, dt, True, *t, seed=len(t[0]))


def test_packed_backward_gates_out_what_is_not_a_number():
    run_packed_backward(8, 32, 64, "bf16", True, "", "", "", "", "", nan=True)
    run_packed_backward(8, 32, 64, "bf16", True, "R", "r", "C", "R", "R", nan=True)
