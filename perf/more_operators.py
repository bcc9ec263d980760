"""What stands between the layers of a residual block, and layers in 8 bits, as they are timed.

  drop              dropout whose mask comes from a counter-based generator (the backward pass is the same call)
  norm, norm_bwd    the residual's addition (with dropout of the branch) and the root-mean-square norm behind it; the gradients
  norm8             the same for answering: the norm's output in 8 bits with a scale for each token, and its values
  fc8               a fully-connected layer in 8-bit integers, a scale for each token and for each output channel; `quant`: its
                    input comes in the tensors' type, as the layer before leaves it

`listed()` names the cases; `draw()` gives further ones of the same ranges.  `prepare()` makes what a program has in hand: the
shards of its tensors under their tilings (strings over "RCr", one letter a cut: rows, columns, replicated), and weights in 8 bits.
`run()` is one pass: the library's calls, or the same formulas in elementary torch operations.  `exact()` is the formulas in 64 bits.

An 8-bit row begins every `_pitch(columns)` bytes, with zeros behind its values; an 8-bit weight is kept transposed, a row for each
output channel.
"""
import functools
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-5


def listed():
    return [
        # A training step's activations: every position of 8 sequences of 2048, a tenth dropped.
        dict(name="drop_step", op="drop", dtype="bf16", T=16384, D=4096, k=0, tX="", tY="", p=0.1),
        # A small fp32 run on sizes that are no round numbers, rows on the one side and columns on the other.
        dict(name="drop_ragged", op="drop", dtype="f32", T=502, D=1500, k=1, tX="R", tY="C", p=0.25),
        # A training step's residual sum and norm.
        dict(name="norm_step", op="norm", dtype="bf16", T=16384, D=4096, k=0, tX="", tY="", p=0.1, res=True),
        # A small fp32 block without dropout: what a debugging run costs.
        dict(name="norm_small", op="norm", dtype="f32", T=100, D=1000, k=0, tX="", tY="", p=0.0, res=True),
        # The backward pass of a wider block over 8 shards, cut differently on the two sides of the norm.
        dict(name="norm_bwd_step", op="norm_bwd", dtype="bf16", T=16384, D=8192, k=3, tX="RRC", tY="RCC", p=0.1, res=True),
        # Rows that are not whole 16-byte vectors, a norm without a residual.
        dict(name="norm_bwd_ragged", op="norm_bwd", dtype="bf16", T=2999, D=1500, k=0, tX="", tY="", p=0.0, res=False),
        # The next tokens of 16 sequences that are being answered: all latency.
        dict(name="norm8_decode", op="norm8", dtype="bf16", T=16, D=8192, k=0, tX="", tY="", res=True),
        # Whole prompts at once, their columns over 2 shards.
        dict(name="norm8_prompt", op="norm8", dtype="bf16", T=8192, D=8192, k=1, tX="C", tY="C", res=True),
        # The layer behind the norm, for 16 tokens: the weight is read once.
        dict(name="fc8_decode", op="fc8", dtype="bf16", T=16, n_in=4096, n_out=16384, k=0, tX="", tW="", tY="", relu=True, quant=False),
        # Sizes that are no round numbers, fp32 results.
        dict(name="fc8_ragged", op="fc8", dtype="f32", T=333, n_in=1500, n_out=2999, k=0, tX="", tW="", tY="", relu=False, quant=True),
        # The first VGG-16 classifier layer over 8 shards as the planner cuts it.
        dict(name="fc8_vgg16", op="fc8", dtype="bf16", T=256, n_in=25088, n_out=4096, k=3, tX="CCC", tW="RRR", tY="CCr", relu=True, quant=True),
        # One wide layer over whole prompts, nothing cut: a large product.
        dict(name="fc8_wide", op="fc8", dtype="bf16", T=4096, n_in=8192, n_out=8192, k=0, tX="", tW="", tY="", relu=True, quant=True),
    ]


# ------------------------------------------------------------------------------------------------- further cases

def _log_int(rng, lo, hi, step=1):
    """an integer between lo and hi, spread over the logarithm, a multiple of step"""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(round(v / step)) * step)


def _tiling(rng, k):
    return "".join(rng.choice("RRCCr") for _ in range(k))


def _copies(t):
    return 1 << t.count("r")


def draw(rng):
    op = rng.choice(["drop", "norm", "norm", "norm_bwd", "norm_bwd", "norm8", "norm8", "fc8", "fc8", "fc8", "fc8"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    e = 2 if dtype == "bf16" else 4
    while True:
        k = rng.choice([0, 0, 0, 1, 2, 3])
        n = 1 << k
        step = n * rng.choice([1, 8, 64])
        rows = 1 if k == 0 else n
        c = dict(op=op, dtype=dtype, k=k, tX=_tiling(rng, k), tY=_tiling(rng, k))
        if op == "fc8":
            c.update(T=_log_int(rng, 1, 8192, rows), n_in=_log_int(rng, 64, 16384, step), n_out=_log_int(rng, 64, 16384, step), tW=_tiling(rng, k),
                     relu=rng.random() < 0.5, quant=rng.random() < 0.5)
            if 2.0 * c["T"] * c["n_in"] * c["n_out"] > 5e11 or c["n_in"] * c["n_out"] * _copies(c["tW"]) > 3e8:
                continue
        else:
            c.update(T=_log_int(rng, 1, 32768, rows), D=_log_int(rng, 64, 16384, step))
            if op != "norm8":
                c["p"] = rng.choice([0.0, 0.1, 0.1, 0.5]) if op != "drop" else rng.choice([0.05, 0.1, 0.5])
            if op != "drop":
                c["res"] = rng.random() < 0.7
            if e * c["T"] * c["D"] * max(_copies(c["tX"]), _copies(c["tY"])) > 2.7e8:
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


def _pitch(cols):
    return -(-cols // 128) * 128


def _rows8(full, t):
    """8-bit shards: rows that begin every _pitch() bytes"""
    return [torch.nn.functional.pad(s, (0, _pitch(s.shape[1]) - s.shape[1])).contiguous() for s in _cut(full, t)]


def _weights8(full, t):
    """8-bit shards of a weight, transposed"""
    return [torch.nn.functional.pad(s.T, (0, _pitch(s.shape[0]) - s.shape[0])).contiguous() for s in _cut(full, t)]


def _empty(rows, cols, t, dtype):
    sr, sc = rows >> t.count("R"), cols >> t.count("C")
    return [torch.empty((sr, sc), dtype=dtype, device=DEVICE) for _ in range(1 << len(t))]


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(g, rows, cols, std=1.0):
    return torch.empty((rows, cols), dtype=torch.float32, device=DEVICE).normal_(0.0, std, generator=g)


def _activations(g, rows, cols):
    """values as layers leave them: channels of unlike size"""
    return _normal(g, rows, cols) * torch.exp(0.5 * _normal(g, 1, cols))


def prepare(case, seed):
    c = dict(case)
    g, dt = _gen(seed), _torch_dtype(c["dtype"])
    s = {"case": c}
    if c["op"] == "fc8":
        if c["quant"]:
            s["X"] = _cut(_activations(g, c["T"], c["n_in"]).clamp(min=0).to(dt), c["tX"])
        else:
            x = _activations(g, c["T"], c["n_in"])
            s["XS"] = x.abs().amax(1) / 127.0
            s["XQ"] = _rows8(torch.round(x / s["XS"][:, None]).to(torch.int8), c["tX"])
        w = _normal(g, c["n_in"], c["n_out"], c["n_in"] ** -0.5)
        s["WS"] = w.abs().amax(0) / 127.0
        s["WQ"] = _weights8(torch.round(w / s["WS"]).to(torch.int8), c["tW"])
        return s
    T, D = c["T"], c["D"]
    s["X"] = _cut(_activations(g, T, D).to(dt), c["tX"])
    if c.get("p"):
        # seed and offset as a program gives them to a layer; the step's number lies in device memory, where a captured graph finds it
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 ^ (seed * 0x1000003), 7
        s["step"] = torch.randint(0, 1 << 40, (1,), generator=g, device=DEVICE)
    if c["op"] == "drop":
        return s
    s["gain"] = (1.0 + 0.2 * _normal(g, 1, D)[0]).to(dt)
    s["R"] = _cut((2.0 * _activations(g, T, D)).to(dt), c["tX"]) if c["res"] and c["op"] != "norm_bwd" else None
    if c["op"] == "norm_bwd":       # (X is the sum that the forward pass left)
        s["dY"] = _cut(_normal(g, T, D, 0.01).to(dt), c["tY"])
        s["dH"] = _cut(_normal(g, T, D, 0.01).to(dt), c["tX"]) if c["res"] else None
    return s


# ------------------------------------------------------------------------------------------- the formulas, in 32 bits

_M0, _M1, _W0, _W1, _LOW = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85, 0xFFFFFFFF


def _kept(s, rows, cols):
    """The dropout mask: Philox4x32-10 of the counter (column / 8, row, offset) under the seed, 16 bits a value."""
    groups = -(-cols // 8)
    at = int(s["offset"]) + s["step"]           # (of the device; as 64 bits)
    x0 = torch.arange(groups, device=DEVICE).expand(rows, groups)
    x1 = torch.arange(rows, device=DEVICE)[:, None].expand(rows, groups)
    x2, x3 = (at & _LOW).expand(rows, groups), (at >> 32 & _LOW).expand(rows, groups)
    k0, k1 = s["seed"] & _LOW, s["seed"] >> 32 & _LOW
    for _ in range(10):
        a, b = x0 * _M0, x2 * _M1               # (the low 64 bits, which are all of them)
        x0, x1, x2, x3 = (b >> 32 & _LOW) ^ x1 ^ k0, b & _LOW, (a >> 32 & _LOW) ^ x3 ^ k1, a & _LOW
        k0, k1 = (k0 + _W0) & _LOW, (k1 + _W1) & _LOW
    u = torch.stack([x0 & 65535, x0 >> 16, x1 & 65535, x1 >> 16, x2 & 65535, x2 >> 16, x3 & 65535, x3 >> 16], 2)
    return u.view(rows, groups * 8)[:, :cols] >= _threshold(s["case"]["p"])


def _threshold(p):
    return int(p * 65536.0 + 0.5)


def _dropped(x, s):
    """x with dropout, in the type that it has"""
    c = s["case"]
    if not c["p"]:
        return x
    return torch.where(_kept(s, c["T"], c["D"]), x * (65536.0 / (65536 - _threshold(c["p"]))), torch.zeros_like(x))


def _q8(u):
    """(steps, largest magnitude) of the rows of u, in 64 bits: a value may lie next to the border of two steps"""
    m = u.abs().amax(1, keepdim=True)
    q = torch.where(m > 0, torch.round(u * 127.0 / m), torch.zeros_like(u))
    return q, m


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(s):
    c = s["case"]
    dt = _torch_dtype(c["dtype"])
    if c["op"] == "drop":
        return _cut(_dropped(_join(s["X"], c["tX"]).float(), s).to(dt), c["tY"])
    if c["op"] == "fc8":
        if c["quant"]:
            q, m = _q8(_join(s["X"], c["tX"]).double())
            q, xs = q.float(), (m[:, 0] / 127.0).float()
        else:
            q, xs = _join([x[:, :c["n_in"] >> c["tX"].count("C")] for x in s["XQ"]], c["tX"]).float(), s["XS"]
        w = _join([x[:, :c["n_in"] >> c["tW"].count("R")].T for x in s["WQ"]], c["tW"]).float()
        y = (q @ w) * xs[:, None] * s["WS"]
        return _cut((y.clamp(min=0) if c["relu"] else y).to(dt), c["tY"])
    gain = s["gain"].float()
    X = _join(s["X"], c["tX"]).float()
    if c["op"] == "norm_bwd":
        dY = _join(s["dY"], c["tY"]).float()
        r = torch.rsqrt((X * X).mean(1, keepdim=True) + EPS)
        n, gy = X * r, dY * gain
        dS = r * (gy - n * (gy * n).mean(1, keepdim=True))
        if c["res"]:
            dS = dS + _join(s["dH"], c["tX"]).float()
        out = {"dS": _cut(dS.to(dt), c["tX"]), "dgain": (dY * n).sum(0)}
        if c["p"]:
            out["dX"] = _cut(_dropped(dS, s).to(dt), c["tX"])
        return out
    H = X if c["op"] == "norm8" else _dropped(X, s)
    if c["res"]:
        H = H + _join(s["R"], c["tX"]).float()
    H = H.to(dt)            # the sum as it is kept: its norm is taken
    h = H.float()
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    if c["op"] == "norm":
        return {"H": _cut(H, c["tX"]), "Y": _cut((h * r * gain).to(dt), c["tY"])}
    q, m = _q8(h.double() * gain.double())
    S = m[:, 0].float() * r[:, 0] / 127.0
    return {"H": _cut(H, c["tX"]), "S": S, "Y": _cut((q.float() * S[:, None]).to(dt), c["tY"])}


def _held(s, name, make):
    """what a program keeps from step to step: results, workspaces, descriptions"""
    if name not in s:
        s[name] = make()
    return s[name]


def _workspace(nbytes):
    return torch.empty(max(256, nbytes), dtype=torch.uint8, device=DEVICE)


def _empty8(rows, cols, t):
    return [torch.empty((rows >> t.count("R"), _pitch(cols >> t.count("C"))), dtype=torch.int8, device=DEVICE) for _ in range(1 << len(t))]


def _run_own(s):
    import paper_1805_04170_amd as tt
    c = s["case"]
    k, dn, dt, T = c["k"], c["dtype"], _torch_dtype(c["dtype"]), c["T"]
    if c["op"] == "fc8":
        lay = _held(s, "layer", lambda: tt.layer("fc", "relu" if c["relu"] else "none", c["n_in"], c["n_out"]))
        Y = _held(s, "Yout", lambda: _empty(T, c["n_out"], c["tY"], dt))
        ws = _held(s, "ws", lambda: _workspace(tt.tt_fc8_workspace_bytes(lay, T, k, dn, c["tX"], c["tW"], c["tY"])))
        XQ, XS = s.get("XQ"), s.get("XS")
        if c["quant"]:
            XQ, XS = _held(s, "q", lambda: (_empty8(T, c["n_in"], c["tX"]), torch.empty(T, device=DEVICE)))
            tt.tt_rows8(T, c["n_in"], k, dn, c["tX"], c["tX"], s["X"], XQ, XS)
        tt.tt_fc_forward8(lay, T, k, dn, c["tX"], c["tW"], c["tY"], XQ, XS, s["WQ"], s["WS"], Y, ws)
        return Y
    D = c["D"]
    drop = _held(s, "drop", lambda: tt.drop(c["p"], s["seed"], s["offset"], s["step"])) if c.get("p") else None
    if c["op"] == "drop":
        Y = _held(s, "Yout", lambda: _empty(T, D, c["tY"], dt))
        tt.tt_dropout(drop, T, D, k, dn, c["tX"], c["tY"], s["X"], Y)
        return Y
    if c["op"] == "norm":
        H, Y = _held(s, "out", lambda: (_empty(T, D, c["tX"], dt), _empty(T, D, c["tY"], dt)))
        tt.tt_norm_forward(T, D, k, dn, c["tX"], c["tY"], EPS, s["X"], s["R"], s["gain"], H, Y, drop)
        return {"H": H, "Y": Y}
    if c["op"] == "norm_bwd":
        dS, dX, dgain = _held(s, "out", lambda: (_empty(T, D, c["tX"], dt), _empty(T, D, c["tX"], dt) if c["p"] else None, torch.empty(D, device=DEVICE)))
        ws = _held(s, "ws", lambda: _workspace(tt.tt_norm_workspace_bytes(T, D, k, dn, c["tX"], c["tY"])))
        tt.tt_norm_backward(T, D, k, dn, c["tX"], c["tY"], EPS, s["X"], s["gain"], s["dY"], s["dH"], dS, dX, dgain, ws, drop)
        return {"dS": dS, "dgain": dgain, "dX": dX} if c["p"] else {"dS": dS, "dgain": dgain}
    H, Q, S, Y = _held(s, "out", lambda: (_empty(T, D, c["tX"], dt), _empty8(T, D, c["tY"]), torch.empty(T, device=DEVICE), _empty(T, D, c["tY"], dt)))
    tt.tt_norm_forward8(T, D, k, dn, c["tX"], c["tY"], EPS, s["X"], s["R"], s["gain"], H, Q, S)
    tt.tt_unrows8(T, D, k, dn, c["tY"], c["tY"], Q, S, Y)
    return {"H": H, "S": S, "Y": Y}


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "fc8":
        x, w, y = c["T"] * c["n_in"], c["n_in"] * c["n_out"], c["T"] * c["n_out"]
        quant = x * (e + _copies(c["tX"])) if c["quant"] else 0
        return {"bytes": quant + x + w + e * y * _copies(c["tY"]) + 4 * (c["T"] + c["n_out"]), "flops": 2.0 * c["T"] * c["n_in"] * c["n_out"]}
    n, x, y = c["T"] * c["D"], _copies(c["tX"]), _copies(c["tY"])
    if c["op"] == "drop":
        return {"bytes": e * n * (1 + y), "flops": 2 * n}
    if c["op"] == "norm":
        return {"bytes": e * n * (1 + c["res"] + x + y) + e * c["D"], "flops": 6 * n}
    if c["op"] == "norm_bwd":
        return {"bytes": e * n * (2 + c["res"] + x * (2 if c["p"] else 1)) + (4 + e) * c["D"], "flops": 12 * n}
    return {"bytes": e * n * (1 + c["res"] + x) + n * y + (n + e * n * y) + e * c["D"] + 8 * c["T"], "flops": 8 * n}


# ----------------------------------------------------------------------------------------- the definitions, in 64 bits

def _philox(counter, key):
    """four words of 32 bits for each counter (Philox4x32, ten rounds), on the host"""
    mul = [np.uint64(0xD2511F53), np.uint64(0xCD9E8D57)]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    for i in range(10):
        keys = [np.uint64((key[0] + i * 0x9E3779B9) % 2 ** 32), np.uint64((key[1] + i * 0xBB67AE85) % 2 ** 32)]
        p = [mul[0] * c[0], mul[1] * c[2]]
        c = [(p[1] >> half) ^ c[1] ^ keys[0], p[1] & low, (p[0] >> half) ^ c[3] ^ keys[1], p[0] & low]
    return c


def _exact_factor(s, rows, cols):
    """what dropout multiplies each value by"""
    p = s["case"]["p"]
    if not p:
        return torch.ones((rows, 1), dtype=torch.float64, device=DEVICE)
    zero_below = round(p * 2 ** 16)
    at = (s["offset"] + int(s["step"].item())) % 2 ** 64
    seed = s["seed"] % 2 ** 64
    groups, parts = (cols + 7) // 8, []
    for first in range(0, rows, 2048):
        n = min(2048, rows - first)
        shape = (n, groups)
        words = _philox([np.broadcast_to(np.arange(groups, dtype=np.uint64)[None], shape), np.broadcast_to(np.arange(first, first + n, dtype=np.uint64)[:, None], shape),
                         np.full(shape, at % 2 ** 32, dtype=np.uint64), np.full(shape, at // 2 ** 32, dtype=np.uint64)], (seed % 2 ** 32, seed // 2 ** 32))
        halves = np.stack(words, 2).astype("<u4").view("<u2").reshape(n, groups * 8)[:, :cols]
        parts.append(torch.from_numpy(halves >= zero_below).to(DEVICE))
    return torch.cat(parts).double() / (1.0 - zero_below / 2 ** 16)


def _exact_steps(u):
    """round(127 u / largest) of each row, and the largest"""
    top = torch.linalg.vector_norm(u, ord=math.inf, dim=1, keepdim=True)
    t = torch.where(top == 0, torch.zeros_like(u), 127.0 * u / top)
    return torch.round(t), top[:, 0]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    dt = _torch_dtype(c["dtype"])
    if c["op"] == "drop":
        return _cut(_join(s["X"], c["tX"]).double() * _exact_factor(s, c["T"], c["D"]), c["tY"])
    if c["op"] == "fc8":
        if c["quant"]:
            q, top = _exact_steps(_join(s["X"], c["tX"]).double())
            xs = top / 127.0
        else:
            q, xs = _join([x[:, :c["n_in"] >> c["tX"].count("C")] for x in s["XQ"]], c["tX"]), s["XS"].double()
        w = _join([x[:, :c["n_in"] >> c["tW"].count("R")].T for x in s["WQ"]], c["tW"])
        y = torch.zeros((c["T"], c["n_out"]), dtype=torch.float64, device=DEVICE)
        for i in range(0, c["n_in"], 1024):     # (sums of 1024 products of 7 bits each stay whole numbers in 24 bits)
            y += torch.mm(q[:, i:i + 1024].float(), w[i:i + 1024].float().contiguous()).double()
        y = y * torch.outer(xs, s["WS"].double())
        return _cut(torch.relu(y) if c["relu"] else y, c["tY"])
    gain, X = s["gain"].double(), _join(s["X"], c["tX"]).double()
    if c["op"] == "norm_bwd":
        dY = _join(s["dY"], c["tY"]).double()
        rms = torch.sqrt(X.square().sum(1) / c["D"] + EPS)
        n = X / rms[:, None]
        along = torch.einsum("td,td->t", gain * dY, n) / c["D"]
        dS = (gain * dY - along[:, None] * n) / rms[:, None] + (_join(s["dH"], c["tX"]).double() if c["res"] else 0.0)
        out = {"dS": _cut(dS, c["tX"]), "dgain": (dY * n).sum(0)}
        if c["p"]:
            out["dX"] = _cut(dS * _exact_factor(s, c["T"], c["D"]), c["tX"])
        return out
    total = X if c["op"] == "norm8" else X * _exact_factor(s, c["T"], c["D"])
    if c["res"]:
        total = total + _join(s["R"], c["tX"]).double()
    h = total.to(dt).double()       # (the sum in the tensors' type is what the norm is defined on)
    rms = torch.sqrt(h.square().sum(1) / c["D"] + EPS)
    if c["op"] == "norm":
        return {"H": _cut(total, c["tX"]), "Y": _cut(h / rms[:, None] * gain, c["tY"])}
    q, top = _exact_steps(h * gain)
    S = top / rms / 127.0
    return {"H": _cut(total, c["tX"]), "S": S, "Y": _cut(q * S[:, None], c["tY"])}
