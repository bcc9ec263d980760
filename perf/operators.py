"""The operators of a token model's training step, as they are timed: the ends of a chain of layers and what lies between its
forward and its backward pass.

  embed_fwd, embed_bwd   rows of an embedding table by token, scaled, and the table's gradient
  policy, logp           the clipped policy loss with a KL term on the chain's logits and its gradient; the tokens' log
                         probabilities alone
  pack, packed_bwd       activations kept in 8 bits (blocks of 32 values with a power of two each), and a fully-connected
                         layer's backward pass that reads them

`listed()` names the cases; `draw()` gives further ones of the same ranges.  `prepare()` makes what a training program has in
hand: the shards of its tensors under their tilings (strings over "RCr", one letter a cut: rows, columns, replicated), tokens
and per-token values.  `run()` is one pass: the library's calls, or the same formulas in elementary torch operations.
`exact()` is the formulas in 64 bits.
"""
import functools
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
BLOCK = 32          # values that share a scale in the 8-bit form


def listed():
    return [
        # The next tokens of 16 sequences that are being generated: 16 rows of a large table, all latency.
        dict(name="embed_fwd_decode", op="embed_fwd", dtype="bf16", T=16, V=131072, D=4096, k=0, tW="", tX="", ids="i64", pad=False),
        # A training step's tokens, every position of 8 sequences of 2048.
        dict(name="embed_fwd_step", op="embed_fwd", dtype="bf16", T=16384, V=65536, D=4096, k=0, tW="", tX="", ids="i64", pad=True),
        # Sizes that are no round numbers, rows that are not whole 16-byte vectors.
        dict(name="embed_bwd_ragged", op="embed_bwd", dtype="bf16", T=2999, V=50021, D=1500, k=0, tW="", tX="", ids="i32", pad=True),
        # A training step's table gradient over 8 shards: the table by rows and columns, the activations by rows and columns.
        dict(name="embed_bwd_step", op="embed_bwd", dtype="bf16", T=16384, V=65536, D=8192, k=3, tW="RCC", tX="RRC", ids="i64", pad=False),
        # A small fp32 head (the output width of AlexNet's classifier): what a debugging run costs.
        dict(name="policy_small", op="policy", dtype="f32", T=100, V=1000, k=0, tX="", tG="", ids="i64", masked=False, kl=0.05),
        # An odd vocabulary, a tenth of the tokens masked, some vocabulary entries ruled out.
        dict(name="policy_ragged", op="policy", dtype="bf16", T=1000, V=50021, k=0, tX="", tG="", ids="i32", masked=True, kl=0.05),
        # A training step's tokens over a large vocabulary, nothing cut.
        dict(name="policy_step", op="policy", dtype="bf16", T=4096, V=131072, k=0, tX="", tG="", ids="i64", masked=False, kl=0.0),
        # The vocabulary cut over 8 shards, as a column-cut last layer leaves it; its gradient cut by rows and columns.
        dict(name="policy_sharded", op="policy", dtype="bf16", T=2048, V=32768, k=3, tX="CCC", tG="RRC", ids="i64", masked=True, kl=0.05),
        # Log probabilities of the tokens that 16 sequences have just been given.
        dict(name="logp_decode", op="logp", dtype="bf16", T=16, V=131072, k=0, tX="", ids="i64", masked=False),
        # A wide layer's activations into 8 bits and back.
        dict(name="pack_wide", op="pack", dtype="bf16", rows=8192, cols=8192, k=0, tX="", relu=True),
        # The first VGG-16 classifier layer's backward pass over 8 shards as the planner cuts it, from 8-bit activations.
        dict(name="packed_bwd_vgg16", op="packed_bwd", dtype="bf16", T=256, n_in=25088, n_out=4096, k=3, tX="CCC", tW="RRR",
             tY="CCr", tdY="CCr", tdX="CCC", relu=True),
        # One wide layer at a large batch, nothing cut: two large products.
        dict(name="packed_bwd_wide", op="packed_bwd", dtype="bf16", T=2048, n_in=8192, n_out=8192, k=0, tX="", tW="", tY="",
             tdY="", tdX="", relu=True),
    ]


# ------------------------------------------------------------------------------------------------- further cases

def _log_int(rng, lo, hi, step=1):
    """an integer between lo and hi, spread over the logarithm, a multiple of step"""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(round(v / step)) * step)


def _tiling(rng, k):
    return "".join(rng.choice("RRCCr") for _ in range(k))


# tilings of a layer's X, W, Y, dY, dX for one cut: data parallel, columns of the weight, rows of the weight
_LAYER_CUTS = {"data": "RrRRR", "columns": "rCCCr", "rows": "CRrrC"}


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "embed_bwd", "policy", "policy", "policy", "logp", "pack", "packed_bwd", "packed_bwd"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    e = 2 if dtype == "bf16" else 4
    while True:
        k = rng.choice([0, 0, 0, 1, 2, 3])
        n = 1 << k
        step = n * rng.choice([1, 8, 64])
        if op in ("embed_fwd", "embed_bwd"):
            c = dict(op=op, dtype=dtype, T=_log_int(rng, 1, 32768, 1 if k == 0 else n), V=_log_int(rng, 500, 200000, n), D=_log_int(rng, 64, 8192, step),
                     k=k, tW=_tiling(rng, k), tX=_tiling(rng, k), ids=rng.choice(["i32", "i64"]), pad=rng.random() < 0.5)
            copies = (1 << c["tW"].count("r"), 1 << c["tX"].count("r"))
            if e * c["D"] * (c["V"] * copies[0] + c["T"] * copies[1]) > 1.2e9:
                continue
        elif op == "policy":
            c = dict(op=op, dtype=dtype, T=_log_int(rng, 1, 8192, 1 if k == 0 else n), V=_log_int(rng, 500, 200000, step), k=k, tX=_tiling(rng, k),
                     tG=_tiling(rng, k), ids=rng.choice(["i32", "i64"]), masked=rng.random() < 0.5, kl=rng.choice([0.0, 0.05]))
            if e * c["T"] * c["V"] * (1 << max(c["tX"].count("r"), c["tG"].count("r"))) > 1.0e9:
                continue
        elif op == "logp":
            c = dict(op=op, dtype=dtype, T=_log_int(rng, 1, 4096, 1 if k == 0 else n), V=_log_int(rng, 500, 200000, step), k=k, tX=_tiling(rng, k),
                     ids=rng.choice(["i32", "i64"]), masked=rng.random() < 0.5)
            if e * c["T"] * c["V"] * (1 << c["tX"].count("r")) > 1.0e9:
                continue
        elif op == "pack":
            c = dict(op=op, dtype=dtype, rows=_log_int(rng, 1, 16384, 1 if k == 0 else n), cols=_log_int(rng, 16, 16384, step), k=k, tX=_tiling(rng, k),
                     relu=rng.random() < 0.5)
            if c["rows"] * c["cols"] * (1 << c["tX"].count("r")) > 7e7:
                continue
        else:
            cuts = [_LAYER_CUTS[rng.choice(sorted(_LAYER_CUTS))] for _ in range(k)]
            tX, tW, tY, tdY, tdX = ("".join(x[i] for x in cuts) for i in range(5))
            hi = 8192 if dtype == "bf16" else 1024
            c = dict(op=op, dtype=dtype, T=_log_int(rng, 8 * n, 4096 if dtype == "bf16" else 512, n), n_in=_log_int(rng, 64, hi, step),
                     n_out=_log_int(rng, 64, hi, step), k=k, tX=tX, tW=tW, tY=tY, tdY=tdY, tdX=tdX, relu=rng.random() < 0.7)
            if 4.0 * c["T"] * c["n_in"] * c["n_out"] > 5e11:
                continue
        tilings = [(t, c.get(a), c.get(b)) for t, a, b in (("tW", "V", "D"), ("tX", "T", "D"), ("tX", "T", "V"), ("tG", "T", "V"), ("tX", "rows", "cols"))
                   if t in c and a in c and b in c]
        if any(rows % (1 << c[t].count("R")) or cols % (1 << c[t].count("C")) for t, rows, cols in tilings):
            continue
        if 3072 in c.values():      # (a size that no workload here has)
            continue
        return c


# -------------------------------------------------------------------------------------------------------- tensors

def _torch_dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _block_of(t, s):
    """(row block, column block) that shard s of tiling t holds"""
    k = len(t)
    bits = [(s >> (k - 1 - j)) & 1 for j in range(k)]
    number = lambda letter: functools.reduce(lambda a, j: 2 * a + bits[j] if t[j] == letter else a, range(k), 0)  # noqa: E731
    return number("R"), number("C")


def _cut(full, t):
    """the 2^k shards of a tensor, each a dense buffer of its own"""
    sr, sc = full.shape[0] >> t.count("R"), full.shape[1] >> t.count("C")
    at = [_block_of(t, s) for s in range(1 << len(t))]
    return [full[r * sr:(r + 1) * sr, c * sc:(c + 1) * sc].clone(memory_format=torch.contiguous_format) for r, c in at]


def _join(shards, t):
    """the tensor that shards hold (replicas are equal: the last one is taken)"""
    if len(shards) == 1:
        return shards[0]
    held = {_block_of(t, s): shards[s] for s in range(len(shards))}
    rows, cols = 1 << t.count("R"), 1 << t.count("C")
    return torch.cat([torch.cat([held[r, c] for c in range(cols)], 1) for r in range(rows)], 0)


def _empty(rows, cols, t, dtype):
    sr, sc = rows >> t.count("R"), cols >> t.count("C")
    return [torch.empty((sr, sc), dtype=dtype, device=DEVICE) for _ in range(1 << len(t))]


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(g, rows, cols, std=1.0):
    return torch.empty((rows, cols), dtype=torch.float32, device=DEVICE).normal_(0.0, std, generator=g)


def _tokens(g, T, V, ids, pad=False):
    """Token numbers as text has them: the v-th most frequent one about 1 / v as often as the first.  pad: a sixteenth of the
    positions hold no token (-1)."""
    u = torch.rand(T, generator=g, device=DEVICE, dtype=torch.float64)
    t = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    if pad:
        t = torch.where(torch.rand(T, generator=g, device=DEVICE) < 1 / 16, torch.full_like(t, -1), t)
    return t.to(torch.int32 if ids == "i32" else torch.int64)


def _logits(c, g):
    """logits (fp32 values that the case's type holds), tokens, weights.  masked: a tenth of the tokens have weight 0, and NaN or
    infinities in their logits as often as not; the last entries of the vocabulary are ruled out (-inf); now and then a token
    has nothing left."""
    T, V = c["T"], c["V"]
    x = _normal(g, T, V, 2.5)
    a = torch.randint(0, max(1, V - V // 50), (T,), generator=g, device=DEVICE)
    rows = torch.arange(T, device=DEVICE)
    x[rows, a] += 8.0
    w = torch.full((T,), 1.0 / T, device=DEVICE)
    if c["masked"]:
        x[:, V - V // 50:] = -math.inf
        u = torch.rand(T, generator=g, device=DEVICE)
        w = torch.where(u < 0.1, torch.zeros_like(w), w)
        x[u < 0.05, :] = math.nan
        x[u < 0.02, :] = math.inf
        x[(u > 0.5) & (u < 0.505), :] = -math.inf
    return x.to(_torch_dtype(c["dtype"])), a.to(torch.int32 if c["ids"] == "i32" else torch.int64), w


# ------------------------------------------------------------------------------------------- the formulas, in 32 bits

def _pack(x):
    """8-bit form of x (rows x cols): blocks of 32 values of a row share a power of two 2^(S - 127), the smallest one that keeps
    them within 127 steps; a value that is not zero is at least one step; blocks with a value that is not finite have S = 255."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    top = b.abs().amax(2)
    bits = top.contiguous().view(torch.int32)
    e = (bits >> 23) - 127 - 6 + ((bits & 0x7fffff) > 0x7e0000).int()
    e = e.clamp(min=-126)
    fine = (bits < 0x7f800000)
    e = torch.where(fine, e, torch.zeros_like(e))
    inv = ((127 - e) << 23).contiguous().view(torch.float32)
    v = torch.where(fine[..., None], b, torch.zeros_like(b))
    q = torch.round(v * inv[..., None])
    q = torch.where((q == 0) & (v != 0), torch.sign(v), q)
    S = torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8)
    return q.view(rows, -1)[:, :cols].to(torch.int8).contiguous(), S


def _unpack(Q, S):
    rows, cols = Q.shape
    s = S.int()
    scale = torch.where(s == 255, torch.full_like(s, 0x7fc00000), s << 23).contiguous().view(torch.float32)
    return (torch.nn.functional.pad(Q.float(), (0, -cols % BLOCK)).view(rows, -1, BLOCK) * scale[..., None]).view(rows, -1)[:, :cols]


def _live(x, a, w):
    """tokens that count: a weight, a token of the vocabulary, and something left to choose from"""
    return (w != 0) & (a >= 0) & (a < x.shape[1]) & ~(x == -math.inf).all(1)


def _token_logp(x, a, live):
    """log softmax at the tokens, and the softmax's parts"""
    z = torch.where(live[:, None], x, torch.zeros_like(x))
    m = z.amax(1)
    p = torch.exp(z - m[:, None])
    s = p.sum(1)
    at = torch.where(live, a.long(), torch.zeros_like(a, dtype=torch.long))[:, None]
    logp = z.gather(1, at)[:, 0] - m - torch.log(s)
    return torch.where(live, logp, torch.zeros_like(logp)), p, s, at


def _policy(x, a, old, ref, adv, w, c):
    """loss, log probabilities and the logits' gradient, in the type that x has"""
    live = _live(x, a, w)
    logp, p, s, at = _token_logp(x, a, live)
    w = torch.where(live, w, torch.zeros_like(w))
    ratio = torch.exp(logp - old)
    loss = -torch.minimum(ratio * adv, ratio.clamp(1 - CLIP, 1 + CLIP) * adv)
    held = ((adv > 0) & (ratio > 1 + CLIP)) | ((adv < 0) & (ratio < 1 - CLIP))
    d = torch.where(held, torch.zeros_like(ratio), -ratio * adv)
    if c["kl"]:
        diff = ref - logp
        loss = loss + c["kl"] * (torch.expm1(diff) - diff)
        d = d - c["kl"] * torch.expm1(diff)
    loss = torch.where(live, w * loss, torch.zeros_like(loss)).sum()
    d = torch.where(live, w * d, torch.zeros_like(d))
    G = p * (-d / s)[:, None]
    G.scatter_add_(1, at, d[:, None])
    return loss, logp, torch.where(live[:, None], G, torch.zeros_like(G))


CLIP = 0.2


# -------------------------------------------------------------------------------------------------------------- cases

def prepare(case, seed):
    c = dict(case)
    g, dt = _gen(seed), _torch_dtype(c["dtype"])
    s = {"case": c}
    if c["op"] == "embed_fwd":
        s["ids"] = _tokens(g, c["T"], c["V"], c["ids"], c["pad"])
        s["W"] = _cut(_normal(g, c["V"], c["D"], 0.02).to(dt), c["tW"])
    elif c["op"] == "embed_bwd":
        s["ids"] = _tokens(g, c["T"], c["V"], c["ids"], c["pad"])
        s["dX"] = _cut(_normal(g, c["T"], c["D"], 0.01).to(dt), c["tX"])
    elif c["op"] in ("policy", "logp"):
        x, s["a"], s["w"] = _logits(c, g)
        if c["op"] == "policy":
            live = _live(x, s["a"], s["w"])
            step = max(1, (1 << 28) // c["V"])
            logp = torch.cat([_token_logp(x[i:i + step].float(), s["a"][i:i + step], live[i:i + step])[0] for i in range(0, c["T"], step)])
            noise = _normal(g, 3, c["T"])
            s["old"], s["ref"], s["adv"] = logp + 0.15 * noise[0], logp + 0.2 * noise[1], noise[2].contiguous()
        s["X"] = _cut(x, c["tX"])
    elif c["op"] == "pack":
        x = _normal(g, c["rows"], c["cols"])
        x = (x.clamp(min=0) if c["relu"] else x) * torch.exp(_normal(g, 1, c["cols"]))     # channels of unlike size
        s["X"] = _cut(x.to(dt), c["tX"])
    else:
        X, Y = _normal(g, c["T"], c["n_in"]).clamp(min=0).to(dt), _normal(g, c["T"], c["n_out"])
        s["X"] = [_pack(t) for t in _cut(X, c["tX"])]
        s["Y"] = [_pack(t) for t in _cut((Y.clamp(min=0) if c["relu"] else Y).to(dt), c["tY"])]
        s["W"] = _cut(_normal(g, c["n_in"], c["n_out"], c["n_in"] ** -0.5).to(dt), c["tW"])
        s["dY"] = _cut(_normal(g, c["T"], c["n_out"], 0.01).to(dt), c["tdY"])
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(s):
    c = s["case"]
    dt = _torch_dtype(c["dtype"])
    if c["op"] == "embed_fwd":
        ids, W = s["ids"].long(), _join(s["W"], c["tW"])
        fine = (ids >= 0) & (ids < c["V"])
        x = W[ids.clamp(0, c["V"] - 1)].float() * math.sqrt(c["D"])
        return _cut(torch.where(fine[:, None], x, torch.zeros_like(x)).to(dt), c["tX"])
    if c["op"] == "embed_bwd":
        ids, dX = s["ids"].long(), _join(s["dX"], c["tX"]).float()
        fine = (ids >= 0) & (ids < c["V"])
        dW = torch.zeros((c["V"], c["D"]), device=DEVICE)
        dW.index_add_(0, ids.clamp(0, c["V"] - 1), torch.where(fine[:, None], dX, torch.zeros_like(dX)))
        return _cut((dW * math.sqrt(c["D"])).to(dt), c["tW"])
    if c["op"] == "policy":
        x = _join(s["X"], c["tX"]).float()
        loss, logp, G = _policy(x, s["a"], s["old"], s["ref"], s["adv"], s["w"], c)
        return {"loss": loss.view(1), "logp": logp, "dX": _cut(G.to(dt), c["tG"])}
    if c["op"] == "logp":
        x = _join(s["X"], c["tX"]).float()
        live = _live(x, s["a"], torch.ones_like(s["w"]))
        return _token_logp(x, s["a"], live)[0]
    if c["op"] == "pack":
        return [_unpack(*_pack(x)).to(dt) for x in s["X"]]
    X = _join([_unpack(*p) for p in s["X"]], c["tX"])
    G = _join(s["dY"], c["tdY"]).float()
    if c["relu"]:
        Y = _join([_unpack(*p) for p in s["Y"]], c["tY"])
        G = torch.where(Y > 0, G, torch.zeros_like(G))
    W = _join(s["W"], c["tW"]).float()
    return {"dX": _cut((G @ W.T).to(dt), c["tdX"]), "dW": _cut((X.T @ G).to(dt), c["tW"])}


def _kept(s, name, make):
    """buffers that a program keeps from step to step: results and workspaces"""
    if name not in s:
        s[name] = make()
    return s[name]


def _workspace(nbytes):
    return torch.empty(max(256, nbytes), dtype=torch.uint8, device=DEVICE)


def _run_own(s):
    import paper_1805_04170_amd as tt
    c = s["case"]
    k, dn, dt = c["k"], c["dtype"], _torch_dtype(c["dtype"])
    if c["op"] == "embed_fwd":
        X = _kept(s, "Xout", lambda: _empty(c["T"], c["D"], c["tX"], dt))
        tt.tt_embed_forward(c["T"], c["V"], c["D"], k, dn, c["tW"], c["tX"], s["ids"], math.sqrt(c["D"]), s["W"], X)
        return X
    if c["op"] == "embed_bwd":
        dW = _kept(s, "dW", lambda: _empty(c["V"], c["D"], c["tW"], dt))
        ws = _kept(s, "ws", lambda: _workspace(tt.tt_embed_workspace_bytes(c["T"], c["V"], c["D"], k, dn, c["tX"], c["tW"])))
        tt.tt_embed_backward(c["T"], c["V"], c["D"], k, dn, c["tX"], c["tW"], s["ids"], math.sqrt(c["D"]), s["dX"], dW, ws)
        return dW
    if c["op"] == "policy":
        out = _kept(s, "out", lambda: (torch.empty(1, device=DEVICE), torch.empty(c["T"], device=DEVICE), _empty(c["T"], c["V"], c["tG"], dt)))
        ws = _kept(s, "ws", lambda: _workspace(tt.tt_policy_workspace_bytes(c["T"], c["V"], k, dn, c["tX"], c["tG"])))
        p = _kept(s, "params", lambda: tt.policy(clip_low=CLIP, clip_high=CLIP, kl=c["kl"]))
        tt.tt_policy_loss(p, c["T"], c["V"], k, dn, c["tX"], c["tG"], s["X"], s["a"], s["old"], s["ref"], s["adv"], s["w"],
                          out[0], out[1], out[2], ws)
        return {"loss": out[0], "logp": out[1], "dX": out[2]}
    if c["op"] == "logp":
        logp = _kept(s, "out", lambda: torch.empty(c["T"], device=DEVICE))
        ws = _kept(s, "ws", lambda: _workspace(tt.tt_policy_workspace_bytes(c["T"], c["V"], k, dn, c["tX"])))
        tt.tt_token_logp(c["T"], c["V"], k, dn, c["tX"], 1.0, s["X"], s["a"], logp, ws)
        return logp
    if c["op"] == "pack":
        def make():
            sr, sc = c["rows"] >> c["tX"].count("R"), c["cols"] >> c["tX"].count("C")
            n = 1 << k
            return ([torch.empty((sr, sc), dtype=torch.int8, device=DEVICE) for _ in range(n)],
                    [torch.empty((sr, -(-sc // BLOCK)), dtype=torch.uint8, device=DEVICE) for _ in range(n)], _empty(c["rows"], c["cols"], c["tX"], dt))
        Q, S, X = _kept(s, "out", make)
        tt.tt_pack8(c["rows"], c["cols"], k, dn, c["tX"], s["X"], Q, S)
        tt.tt_unpack8(c["rows"], c["cols"], k, dn, c["tX"], Q, S, X)
        return X
    lay = _kept(s, "layer", lambda: tt.layer("fc", "relu" if c["relu"] else "none", c["n_in"], c["n_out"]))
    tilings = (c["tX"], c["tW"], c["tY"], c["tdY"], c["tdX"])
    dX, dW = _kept(s, "out", lambda: (_empty(c["T"], c["n_in"], c["tdX"], dt), _empty(c["n_in"], c["n_out"], c["tW"], dt)))
    ws = _kept(s, "ws", lambda: _workspace(tt.tt_fc_packed_workspace_bytes(lay, c["T"], k, dn, *tilings)))
    lists = _kept(s, "lists", lambda: [[p[i] for p in s[n]] for n in ("X", "Y") for i in (0, 1)])
    tt.tt_fc_backward_packed(lay, c["T"], k, dn, *tilings, None, None, lists[0], lists[1], s["W"], lists[2], lists[3], s["dY"],
                             dX, dW, ws)
    return {"dX": dX, "dW": dW}


@functools.lru_cache(maxsize=256)
def _distinct(T, V):
    """expected number of different tokens among T"""
    v = np.arange(1, V + 1, dtype=np.float64)
    p = np.log1p(1.0 / v) / math.log(V + 1.0)
    return float(np.sum(-np.expm1(T * np.log1p(-p))))


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    copies = lambda t: 1 << t.count("r")  # noqa: E731
    if c["op"] in ("embed_fwd", "embed_bwd"):
        ids = c["T"] * (4 if c["ids"] == "i32" else 8)
        if c["op"] == "embed_fwd":
            return {"bytes": ids + e * c["D"] * (_distinct(c["T"], c["V"]) + c["T"] * copies(c["tX"])), "flops": c["T"] * c["D"]}
        return {"bytes": ids + e * c["D"] * (c["T"] + c["V"] * copies(c["tW"])), "flops": c["T"] * c["D"]}
    if c["op"] == "policy":
        return {"bytes": e * c["T"] * c["V"] * (1 + copies(c["tG"])) + 28 * c["T"], "flops": 8 * c["T"] * c["V"]}
    if c["op"] == "logp":
        return {"bytes": e * c["T"] * c["V"] + 12 * c["T"], "flops": 4 * c["T"] * c["V"]}
    if c["op"] == "pack":
        n = c["rows"] * c["cols"] * copies(c["tX"])
        return {"bytes": n * (2 * e + 2 * (1 + 1 / BLOCK)), "flops": 4 * n}
    x, y, w = c["T"] * c["n_in"], c["T"] * c["n_out"], c["n_in"] * c["n_out"]
    b = x * (1 + 1 / BLOCK) + e * (y + w) + e * (x * copies(c["tdX"]) + w * copies(c["tW"])) + (y * (1 + 1 / BLOCK) if c["relu"] else 0)
    return {"bytes": b, "flops": 4.0 * c["T"] * c["n_in"] * c["n_out"]}


# ----------------------------------------------------------------------------------------- the definitions, in 64 bits

def _exact_pack(x):
    """the values that the 8-bit form of x stands for"""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x.double(), (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    top = b.abs().amax(2, keepdim=True)
    step = torch.exp2(torch.ceil(torch.log2(top / 127.0)).clamp(min=-126.0, max=127.0))
    # (the logarithm may miss by one where top / 127 is next to a power of two)
    step = torch.where(step * 127.0 < top, 2 * step, step)
    step = torch.where((step * 63.5 >= top) & (step > 2.0 ** -126), step / 2, step)
    n = b / step
    q = torch.where(b == 0, torch.zeros_like(b), torch.sign(b) * torch.clamp(torch.round(n).abs(), min=1.0))
    return (q * step).view(rows, -1)[:, :cols]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "embed_fwd":
        W, ids = _join(s["W"], c["tW"]), s["ids"].long()
        x = torch.zeros((c["T"], c["D"]), dtype=torch.float64, device=DEVICE)
        at = ((ids >= 0) & (ids < c["V"])).nonzero()[:, 0]
        x[at] = torch.index_select(W, 0, ids[at]).double() * c["D"] ** 0.5
        return _cut(x, c["tX"])
    if c["op"] == "embed_bwd":
        dX, ids = _join(s["dX"], c["tX"]), s["ids"].long()
        at = ((ids >= 0) & (ids < c["V"])).nonzero()[:, 0]
        dW = torch.zeros((c["V"], c["D"]), dtype=torch.float64, device=DEVICE)
        dW.index_put_((ids[at],), dX[at].double() * c["D"] ** 0.5, accumulate=True)
        return _cut(dW, c["tW"])
    if c["op"] in ("policy", "logp"):
        full = _join(s["X"], c["tX"])
        a = s["a"].long()
        w = s["w"].double() if c["op"] == "policy" else torch.ones(c["T"], dtype=torch.float64, device=DEVICE)
        loss, logps, grads = 0.0, [], []
        step = max(1, (1 << 26) // c["V"])
        for i in range(0, c["T"], step):
            x, ai, wi = full[i:i + step].double(), a[i:i + step], w[i:i + step]
            n = x.shape[0]
            ok = (wi != 0) & (ai >= 0) & (ai < c["V"]) & (x.isnan() | (x > -math.inf)).any(1)
            lp = torch.zeros(n, dtype=torch.float64, device=DEVICE)
            rows = ok.nonzero()[:, 0]
            lsm = x[rows] - torch.logsumexp(x[rows], 1, keepdim=True)
            lp[rows] = lsm[torch.arange(rows.numel(), device=DEVICE), ai[rows]]
            logps.append(lp)
            if c["op"] == "policy":
                old, ref, adv = (s[m][i:i + step].double()[rows] for m in ("old", "ref", "adv"))
                l, wr = lp[rows], wi[rows]
                r = torch.exp(l - old)
                lo, hi = torch.full_like(r, 1 - CLIP), torch.full_like(r, 1 + CLIP)
                surrogate = torch.where(adv >= 0, torch.minimum(r, hi), torch.maximum(r, lo)) * adv
                free = torch.where(adv >= 0, r <= hi, r >= lo)
                kl = torch.exp(ref - l) - 1.0 - (ref - l)
                loss = loss + (wr * (c["kl"] * kl - surrogate)).sum()
                dl = wr * (c["kl"] * (1.0 - torch.exp(ref - l)) - free * r * adv)
                G = torch.zeros_like(x)
                onehot = torch.nn.functional.one_hot(ai[rows], c["V"]).double()
                G[rows] = dl[:, None] * (onehot - torch.exp(lsm))
                grads.append(G)
        if c["op"] == "logp":
            return torch.cat(logps)
        return {"loss": torch.as_tensor(loss, device=DEVICE).view(1), "logp": torch.cat(logps), "dX": _cut(torch.cat(grads), c["tG"])}
    if c["op"] == "pack":
        return [_exact_pack(x) for x in s["X"]]
    value = lambda p: p[0].double() * torch.exp2(p[1].double() - 127.0).repeat_interleave(BLOCK, 1)[:, :p[0].shape[1]]  # noqa: E731
    X, W, G = _join([value(p) for p in s["X"]], c["tX"]), _join(s["W"], c["tW"]).double(), _join(s["dY"], c["tdY"]).double()
    if c["relu"]:
        G = G * (_join([value(p) for p in s["Y"]], c["tY"]) > 0)
    return {"dX": _cut(torch.matmul(G, W.transpose(0, 1).contiguous()), c["tdX"]), "dW": _cut(torch.matmul(X.transpose(0, 1).contiguous(), G), c["tW"])}
