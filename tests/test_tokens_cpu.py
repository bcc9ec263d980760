"""CPU-side checks of the token operators: exported symbols, refusals (nothing is launched), workspace sizes, and the plain
64-bit forms against differences and against torch."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_1805_04170_amd as tt
from oracle import tokens as tk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = [1 << 20]           # an address that no refused call reads
P2 = [1 << 20] * 2
A = 1 << 20


def refused(status, fn, *args, **kw):
    with pytest.raises(tt.TilingError) as e:
        fn(*args, **kw)
    assert tt.STATUS_NAMES[e.value.status] == status, e.value


class Bytes:
    """a workspace of so many bytes at an address"""

    def __init__(self, n, at=A):
        self.n, self.at = n, at

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def element_size(self):
        return 1


class Asked:
    """an object that has a tensor's methods and is none"""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        if name not in ("data_ptr", "dtype", "numel", "is_contiguous"):
            raise AttributeError(name)
        return getattr(self.t, name)


def test_every_declared_symbol_is_exported_and_bound():
    header = open(os.path.join(ROOT, "include", "tensor_tiling_tokens.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(tt_[a-z0-9_]+)\s*\(", header))
    assert declared == set(tt.TOKEN_EXPORTS)
    L = ctypes.CDLL(tt.binding.LIB_PATH)
    for name in declared:
        assert hasattr(L, name) and hasattr(tt, name), name


def test_embedding_refusals():
    f = lambda T=8, V=8, D=8, k=0, dt="f32", tW="", tX="", ids=A, W=P, X=P, idt="i64": tt.tt_embed_forward(  # noqa: E731
        T, V, D, k, dt, tW, tX, ids, 1.0, W, X, stream=1, id_dtype=idt)
    for bad in (dict(T=-1), dict(V=-1), dict(D=-1), dict(k=7), dict(k=-1), dict(dt=5), dict(k=1, tW="X", tX="R", W=P2, X=P2), dict(ids=None), dict(ids=A + 4),
                dict(idt=9), dict(W=None), dict(X=None), dict(W=[0]), dict(X=[A + 2]), dict(dt="bf16", X=[A + 1]), dict(k=1, tW="R", tX="R", W=P2, X=P)):
        refused("TT_EINVAL", f, **bad)
    refused("TT_EINFEASIBLE", f, V=9, k=1, tW="R", tX="R", W=P2, X=P2)
    refused("TT_EINFEASIBLE", f, T=9, k=1, tW="R", tX="R", W=P2, X=P2)
    for bad in (dict(T=1 << 31), dict(V=1 << 31), dict(D=1 << 31), dict(T=(1 << 31) - 1, D=4096)):
        refused("TT_EUNSUPPORTED", f, **bad)
    f(T=0, ids=None)
    f(D=0)
    with pytest.raises(tt.TilingError):
        tt.tt_embed_forward(8, 8, 8, 0, "f32", "", "", torch.zeros(8), 1.0, P, P, stream=1)    # token numbers that are not whole


def test_embedding_gradient_refusals():
    need = tt.tt_embed_workspace_bytes(1000, 8, 8, 0, "f32", "", "")
    assert need > 0 and tt.tt_embed_workspace_bytes(100, 8, 8, 0, "f32", "", "") == 0      # (few tokens are not sorted)
    f = lambda T=1000, V=8, D=8, k=0, dt="f32", tX="", tW="", ids=A, dX=P, dW=P, ws=Bytes(need): tt.tt_embed_backward(  # noqa: E731
        T, V, D, k, dt, tX, tW, ids, 1.0, dX, dW, ws, stream=1, id_dtype="i32")
    for bad in (dict(T=-1), dict(k=7), dict(dt=2), dict(ids=None), dict(ids=A + 2), dict(dX=None), dict(dW=[0]), dict(dW=[A + 2])):
        refused("TT_EINVAL", f, **bad)
    refused("TT_EINFEASIBLE", f, T=1001, k=1, tX="R", tW="R", dX=P2, dW=P2)
    for ws in (None, Bytes(need - 1), Bytes(need, A + 128)):
        refused("TT_EWORKSPACE", f, ws=ws)
    refused("TT_EINVAL", tt.tt_embed_workspace_bytes, 8, 8, -1, 0, "f32", "", "")
    refused("TT_EINFEASIBLE", tt.tt_embed_workspace_bytes, 8, 9, 8, 1, "f32", "R", "R")
    refused("TT_EUNSUPPORTED", tt.tt_embed_workspace_bytes, 1 << 31, 9, 8, 0, "f32", "", "")
    f(V=0)
    f(D=0)


def test_policy_refusals():
    need = tt.tt_policy_workspace_bytes(8, 16, 0, "f32", "", "")
    ok = tt.policy(kl=0.1)

    def f(p=ok, T=8, V=16, k=0, dt="f32", tX="", tG="", X=P, a=A, old=A, ref=A, adv=A, w=A, loss=A, logp=A, dX=P, ws=Bytes(need), idt="i64"):
        tt.tt_policy_loss(p, T, V, k, dt, tX, tG, X, a, old, ref, adv, w, loss, logp, dX, ws, stream=1, id_dtype=idt)
    nan, inf = math.nan, math.inf
    for bad in (dict(T=-1), dict(V=-1), dict(k=7), dict(dt=3), dict(X=None), dict(X=[A + 2]), dict(dX=[0]), dict(a=None), dict(a=A + 4), dict(old=None), dict(ref=None),
                dict(adv=A + 1), dict(w=None), dict(loss=None), dict(loss=A + 2), dict(logp=A + 2), dict(idt=0), dict(k=1, tX="R", tG="q", X=P2, dX=P2),
                dict(p=tt.policy(scale=0)), dict(p=tt.policy(scale=-1)), dict(p=tt.policy(scale=nan)), dict(p=tt.policy(scale=inf)),
                dict(p=tt.policy(clip_low=-0.1)), dict(p=tt.policy(clip_high=nan)), dict(p=tt.policy(kl=nan)), dict(p=tt.policy(kl=inf))):
        refused("TT_EINVAL", f, **bad)
    refused("TT_EINFEASIBLE", f, V=17, k=1, tX="C", tG="R", X=P2, dX=P2)
    refused("TT_EINFEASIBLE", f, T=9, k=1, tX="C", tG="R", X=P2, dX=P2)
    for bad in (dict(T=1 << 22), dict(V=1 << 31)):
        refused("TT_EUNSUPPORTED", f, **bad)
    for ws in (None, Bytes(need - 1), Bytes(need, A + 64)):
        refused("TT_EWORKSPACE", f, ws=ws)
    refused("TT_EINVAL", tt.tt_policy_workspace_bytes, 8, 16, 1, "f32", "R", "z")
    refused("TT_EINFEASIBLE", tt.tt_policy_workspace_bytes, 8, 17, 1, "f32", "R", "C")


def test_token_logp_refusals():
    need = tt.tt_policy_workspace_bytes(8, 16, 0, "f32", "")

    def f(T=8, V=16, k=0, dt="f32", tX="", scale=1.0, X=P, ids=A, logp=A, ws=Bytes(need), idt="i32"):
        tt.tt_token_logp(T, V, k, dt, tX, scale, X, ids, logp, ws, stream=1, id_dtype=idt)
    for bad in (dict(T=-1), dict(k=7), dict(dt=3), dict(X=None), dict(ids=None), dict(ids=A + 1), dict(logp=None), dict(scale=0.0), dict(scale=math.nan), dict(idt=1)):
        refused("TT_EINVAL", f, **bad)
    refused("TT_EINFEASIBLE", f, V=17, k=1, tX="C", X=P2)
    refused("TT_EWORKSPACE", f, ws=None)
    f(T=0, ids=None, logp=None)


def test_pack_refusals():
    for fn in (tt.tt_pack8, tt.tt_unpack8):
        f = lambda rows=8, cols=8, k=0, dt="f32", t="", a=P, b=P, c=P: fn(rows, cols, k, dt, t, a, b, c, stream=1)  # noqa: E731,B023
        for bad in (dict(rows=-1), dict(cols=-1), dict(k=9), dict(dt=7), dict(a=None), dict(b=[0]), dict(c=None), dict(k=1, t="x", a=P2, b=P2, c=P2)):
            refused("TT_EINVAL", f, **bad)
        refused("TT_EINFEASIBLE", f, rows=9, k=1, t="R", a=P2, b=P2, c=P2)
        for bad in (dict(rows=1 << 31), dict(cols=1 << 31), dict(rows=1 << 30, cols=1 << 30)):
            refused("TT_EUNSUPPORTED", f, **bad)
        f(rows=0)
        f(cols=0)
    refused("TT_EINVAL", tt.tt_pack8, 8, 8, 0, "bf16", "", [A + 1], P, P, stream=1)
    refused("TT_EINVAL", tt.tt_unpack8, 8, 8, 0, "bf16", "", P, P, [A + 1], stream=1)


def test_packed_backward_refusals():
    lay = tt.layer("fc", "relu", 32, 32)
    need = tt.tt_fc_packed_workspace_bytes(lay, 8, 0, "bf16", "", "", "", "", "")

    def f(lay=lay, b=8, k=0, dt="bf16", t=("",) * 5, fd=None, xq=P, xs=P, w=P, yq=P, ys=P, dy=P, dx=P, dw=P, ws=Bytes(need)):
        tt.tt_fc_backward_packed(lay, b, k, dt, *t, fd, None, xq, xs, w, yq, ys, dy, dx, dw, ws, stream=1)
    for bad in (dict(lay=tt.layer("conv", "none", 8, 8, 4, 4, 3, 3, 1)), dict(b=0), dict(k=7), dict(dt=9), dict(xq=None), dict(xs=[0]), dict(w=None), dict(yq=None),
                dict(ys=None), dict(dy=[A + 1]), dict(dx=[A + 1]), dict(dw=None)):
        refused("TT_EINVAL", f, **bad)
    refused("TT_EINFEASIBLE", f, b=9, k=1, t=("R",) * 5, xq=P2, xs=P2, w=P2, yq=P2, ys=P2, dy=P2, dx=P2, dw=P2)
    for ws in (None, Bytes(need - 1), Bytes(need, A + 16)):
        refused("TT_EWORKSPACE", f, ws=ws)
    assert need > tt.tt_fc_packed_workspace_bytes(tt.layer("fc", "none", 32, 32), 8, 0, "bf16", "", "", "", "", "")


def test_per_token_arrays_are_dense_and_long_enough():
    """what slicing leaves is refused before anything is launched: strides, other types, fewer entries than tokens"""
    T, V, D = 8, 16, 8
    i64, f32 = torch.zeros(T, dtype=torch.int64), torch.zeros(T)
    grid, wide = torch.zeros((T, 4), dtype=torch.int64), torch.zeros((T, 4))
    # a workspace of no bytes: calls whose arrays are accepted end at it, nothing is launched
    none = Bytes(0)
    fwd = lambda ids, idt=None: tt.tt_embed_forward(T, V, 0, 0, "f32", "", "", ids, 1.0, P, P, stream=1, id_dtype=idt)  # noqa: E731
    bwd = lambda ids, idt=None: tt.tt_embed_backward(T, V, 0, 0, "f32", "", "", ids, 1.0, P, P, none, stream=1, id_dtype=idt)  # noqa: E731
    logp = lambda ids, out=f32, idt=None: tt.tt_token_logp(T, V, 0, "f32", "", 1.0, P, ids, out, none, stream=1, id_dtype=idt)  # noqa: E731

    def loss(actions=i64, old=f32, ref=f32, adv=f32, w=f32, value=torch.zeros(1), lp=f32, idt=None):
        tt.tt_policy_loss(tt.policy(kl=0.1), T, V, 0, "f32", "", "", P, actions, old, ref, adv, w, value, lp, P, none, stream=1, id_dtype=idt)
    for fn in (fwd, bwd):
        for ok in (i64, i64.int(), torch.zeros(T + 3, dtype=torch.int64), grid[:2], grid[0].expand(1, 4).repeat(2, 1)):
            fn(ok)                          # (no columns: TT_OK, nothing is launched)
        fn(i64, "i64")
        fn(A, "i32")
    plain = Asked(f32)
    refused("TT_EWORKSPACE", loss, old=plain, adv=torch.nn.Parameter(f32.clone()), w=f32.clone().requires_grad_())
    for bad in (wide[:, 1], f32.double(), f32[:T - 1]):
        refused("TT_EINVAL", loss, old=Asked(bad))
        refused("TT_EINVAL", loss, old=torch.nn.Parameter(bad))
    for ok in (dict(), dict(actions=i64.int()), dict(ref=None), dict(old=torch.zeros(T + 1)), dict(lp=None), dict(old=A, adv=A)):
        refused("TT_EWORKSPACE" if ok.get("ref", 0) is not None else "TT_EINVAL", loss, **ok)
    refused("TT_EWORKSPACE", logp, i64)
    for bad in (grid[:, -1], grid.int()[:, 0], i64[::2], i64[:T - 1], torch.zeros(1, dtype=torch.int64).expand(T), i64.short(), f32):
        for fn in (fwd, bwd, logp, loss):
            refused("TT_EINVAL", fn, bad)
    for fn in (fwd, bwd, logp):
        refused("TT_EINVAL", fn, i64.int(), idt="i64")
        refused("TT_EINVAL", fn, i64, idt="i32")
    for name in ("old", "ref", "adv", "w", "lp"):
        for bad in (wide[:, 1], f32.double(), f32.bfloat16(), f32[:T - 1], f32[:1].expand(T), f32.int()):
            refused("TT_EINVAL", loss, **{name: bad})
    for bad in (wide[:, 1], f32.double(), f32[1:]):
        refused("TT_EINVAL", logp, i64, bad)
    for bad in (torch.zeros(0), torch.zeros(1).double()):
        refused("TT_EINVAL", loss, value=bad)


def test_an_array_that_is_not_read_may_be_anything():
    i64, f32 = torch.zeros(8, dtype=torch.int64), torch.zeros(8)
    for ref in (None, f32.bfloat16(), f32[:3], torch.zeros((8, 2))[:, 0]):
        refused("TT_EWORKSPACE", tt.tt_policy_loss, tt.policy(), 8, 16, 0, "f32", "", "", P, i64, f32, ref, f32, f32, torch.zeros(1), f32, P, Bytes(0), stream=1)


def test_tensors_without_values_have_no_buffers():
    """torch's empty tensors have a NULL address; nothing is launched for them"""
    none = lambda r, c, dt=torch.float32: [torch.empty((r, c), dtype=dt)]  # noqa: E731
    ids = torch.empty(0, dtype=torch.int64)
    assert none(0, 8)[0].data_ptr() == 0
    for W in (P, none(0, 8)):
        tt.tt_embed_forward(0, 8 if W is P else 0, 8, 0, "f32", "", "", ids, 1.0, W, none(0, 8), stream=1)
    tt.tt_embed_forward(8, 8, 0, 0, "f32", "", "", A, 1.0, none(8, 0), none(8, 0), stream=1, id_dtype="i64")
    tt.tt_embed_backward(8, 0, 8, 0, "f32", "", "", A, 1.0, P, none(0, 8), None, stream=1, id_dtype="i32")
    tt.tt_embed_backward(0, 8, 0, 0, "f32", "", "", ids, 1.0, none(0, 0), none(8, 0), None, stream=1)
    tt.tt_token_logp(0, 16, 0, "f32", "", 1.0, none(0, 16), ids, torch.empty(0), None, stream=1)
    for fn, dts in ((tt.tt_pack8, (torch.float32, torch.int8, torch.uint8)), (tt.tt_unpack8, (torch.int8, torch.uint8, torch.float32))):
        fn(0, 64, 0, "f32", "", *[none(0, 64, d) for d in dts], stream=1)
        fn(4, 0, 1, "f32", "R", *[none(2, 0, d) * 2 for d in dts], stream=1)
        refused("TT_EINVAL", fn, 0, 64, 0, "f32", "", P, None, P, stream=1)
    refused("TT_EINVAL", tt.tt_embed_forward, 8, 0, 8, 0, "f32", "", "", A, 1.0, none(0, 8), none(0, 8), stream=1, id_dtype="i64")
    refused("TT_EINVAL", tt.tt_embed_backward, 0, 8, 8, 0, "f32", "", "", ids, 1.0, none(0, 8), none(0, 8), None, stream=1)
    refused("TT_EINVAL", tt.tt_token_logp, 4, 16, 0, "f32", "", 1.0, none(0, 16), A, A, Bytes(4096), stream=1, id_dtype="i64")


def test_a_workspace_for_many_tokens_covers_fewer():
    counts = [0, 1, 64, 127, 128, 129, 130, 256, 257, 300, 4096, 16383, 16384, 16385, 20000, 32768, 40000, 65535, 65536, 65537, 70000, 131072, 131073, 1 << 20, (1 << 22) - 1]
    for V, D in [(65536, 8192), (300, 1), (50021, 1500)]:
        sizes = [tt.tt_embed_workspace_bytes(T, V, D, 0, "bf16", "", "") for T in counts]
        assert sizes == sorted(sizes), (V, D)
    for V in (0, 5, 1000, 17000, 131072, 600000, (1 << 31) - 1):
        for dt in ("bf16", "f32"):
            for tdX in (None, ""):
                at = counts + [t + d for p in (1, 2, 3, 8, 37, 64) for t in [((1 << 22) - 1) // p] for d in (-1, 0)]
                sizes = [tt.tt_policy_workspace_bytes(T, V, 0, dt, "", tdX) for T in sorted(at)]
                assert sizes == sorted(sizes), (V, dt, tdX)


def test_plain_policy_gradient_against_differences():
    rng = np.random.default_rng(5)
    T, V, h = 12, 9, 1e-5
    X, a = rng.normal(0, 1.5, (T, V)), rng.integers(0, V, T)
    logp = tk.token_logp(X, a, 0.9)
    old, ref, adv, w = logp - rng.choice([-0.5, -0.1, 0.05, 0.4], T), logp + rng.normal(0, 0.3, T), rng.normal(0, 1, T), rng.random(T)
    w[3] = 0
    f = lambda Z: tk.policy_loss(Z, a, old, ref, adv, w, 0.9, 0.2, 0.25, 0.1)  # noqa: E731
    g = f(X)[2]
    for t in range(T):
        for v in range(V):
            d = np.zeros_like(X)
            d[t, v] = h
            # central differences: h^2 / 6 times the third derivative (of order 10 here), and rounding 1e-16 / h
            assert abs((f(X + d)[0] - f(X - d)[0]) / (2 * h) - g[t, v]) < 1e-8


def test_plain_forms_against_torch():
    rng = np.random.default_rng(6)
    W, ids = torch.tensor(rng.normal(size=(7, 5)), requires_grad=True), torch.tensor([3, 0, 3, 6, 3])
    X = 1.5 * torch.nn.functional.embedding(ids, W)
    dX = torch.tensor(rng.normal(size=(5, 5)))
    X.backward(dX)
    assert np.allclose(tk.embed_forward(W.detach().numpy(), ids.numpy(), 1.5), X.detach().numpy(), atol=1e-14)
    assert np.allclose(tk.embed_backward(dX.numpy(), ids.numpy(), 7, 1.5)[0], W.grad.numpy(), atol=1e-13)
    z = torch.tensor(rng.normal(size=(6, 11)))
    a = torch.tensor(rng.integers(0, 11, 6))
    assert np.allclose(tk.token_logp(z.numpy(), a.numpy(), 0.5), torch.log_softmax(0.5 * z, 1)[torch.arange(6), a].numpy(), atol=1e-13)


def test_plain_8_bit_form():
    x = np.array([[127.0, -3.5, 0.49, -0.2, 0.0, 2.5]])
    q, s = tk.pack8(x)
    assert s[0, 0] == 127 and q.tolist() == [[127, -4, 1, -1, 0, 2]]
    assert tk.unpack8(*tk.pack8(2 * x + 128))[0, 0] == 384      # 382 is 95.5 steps of 4: ties go to the even step, 96
    q, s = tk.pack8(np.array([[128.0, 1.0]]))
    assert s[0, 0] == 128 and q.tolist() == [[64, 1]]
