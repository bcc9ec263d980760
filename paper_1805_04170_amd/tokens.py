"""Binding of include/tensor_tiling_tokens.h, same names: the embedding in front of a chain of layers, the policy loss behind it,
activations in 8 bits between its passes.  Argument marshalling only, as in binding.py; the calls go through the extension
module _calls.

Per-token arrays (token numbers, log probabilities, weights) are dense torch tensors with an entry for every token at least, or
integer device addresses; the type of token numbers is taken from the tensor (torch.int32, torch.int64) or given as id_dtype ("i32",
"i64"), all others are torch.float32.  A tensor of another type, a strided one (tokens[:, -1] without .contiguous()) or a short
one is refused (TT_EINVAL).
"""
import ctypes

from . import binding as _b
from .binding import TilingError

TT_I32, TT_I64 = 2, 3
TT_PACK8_BLOCK = 32
TOKEN_EXPORTS = [
    "tt_embed_forward", "tt_embed_workspace_bytes", "tt_embed_backward", "tt_policy_workspace_bytes", "tt_policy_loss", "tt_token_logp",
    "tt_pack8", "tt_unpack8", "tt_fc_packed_workspace_bytes", "tt_fc_backward_packed",
]
__all__ = TOKEN_EXPORTS + ["TT_I32", "TT_I64", "TT_PACK8_BLOCK", "TOKEN_EXPORTS", "tt_policy", "policy"]


class tt_policy(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("clip_low", ctypes.c_float), ("clip_high", ctypes.c_float), ("kl", ctypes.c_float)]


def policy(clip_low=0.2, clip_high=0.2, kl=0.0, scale=1.0):
    return tt_policy(scale, clip_low, clip_high, kl)


def _fn(name):
    """the address of a function of the loaded library"""
    L = _b._lib or _b.lib()
    try:
        return L.token_addresses[name]
    except AttributeError:
        L.token_addresses = {n: ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in TOKEN_EXPORTS}
        _b._address("tt_retile")        # (makes the extension module known)
        return L.token_addresses[name]


_id_types = {}


def _id_dtype(ids, given):
    if given is not None:
        given = {"i32": TT_I32, "i64": TT_I64}.get(given, given)
        if not hasattr(ids, "dtype"):       # (an address, or None)
            return given
    if not _id_types:
        import torch
        _id_types.update({torch.int32: TT_I32, torch.int64: TT_I64})
    t = _id_types.get(getattr(ids, "dtype", None))
    if t is None or given not in (None, t):
        raise TilingError(1, "token numbers of type %s" % (getattr(ids, "dtype", None),))
    return t


# --------------------------------------------------------------- embedding

def tt_embed_forward(tokens, vocab, width, k, dtype, tW, tX, ids, scale, W, X, stream=None, id_dtype=None):
    fn = _fn("tt_embed_forward")
    _b._check(_b._calls.embed_forward(fn, tokens, vocab, width, k, dtype, tW, tX, _id_dtype(ids, id_dtype), ids, scale, W, X,
                                      _b._stream(stream)), "tt_embed_forward")


def _sized(name, *args):
    out = ctypes.c_size_t()
    _b._check(getattr(_b.lib(), name)(*args, ctypes.byref(out)), name)
    return out.value


def tt_embed_workspace_bytes(tokens, vocab, width, k, dtype, tdX, tdW):
    i = ctypes.c_int64
    return _sized("tt_embed_workspace_bytes", i(tokens), i(vocab), i(width), k, _b._dtype(dtype), _b._tiling(tdX), _b._tiling(tdW))


def tt_embed_backward(tokens, vocab, width, k, dtype, tdX, tdW, ids, scale, dX, dW, workspace, stream=None, id_dtype=None):
    fn = _fn("tt_embed_backward")
    _b._check(_b._calls.embed_backward(fn, tokens, vocab, width, k, dtype, tdX, tdW, _id_dtype(ids, id_dtype), ids, scale, dX, dW, workspace,
                                       _b._stream(stream)), "tt_embed_backward")


# ------------------------------------------------------------- policy loss

def tt_policy_workspace_bytes(tokens, vocab, k, dtype, tX, tdX=None):
    """tdX None: a call without the logits' gradient"""
    i = ctypes.c_int64
    return _sized("tt_policy_workspace_bytes", i(tokens), i(vocab), k, _b._dtype(dtype), _b._tiling(tX), _b._t_or(tdX, tX), 0 if tdX is None else 1)


def tt_policy_loss(params, tokens, vocab, k, dtype, tX, tdX, X, actions, old_logp, ref_logp, advantage, weight, loss, logp, dX, workspace,
                   stream=None, id_dtype=None):
    fn = _fn("tt_policy_loss")
    _b._check(_b._calls.policy_loss(fn, params, tokens, vocab, k, dtype, tX, tX if tdX is None else tdX, X, _id_dtype(actions, id_dtype), actions,
                                    old_logp, ref_logp, advantage, weight, loss, logp, dX, workspace, _b._stream(stream)), "tt_policy_loss")


def tt_token_logp(tokens, vocab, k, dtype, tX, scale, X, ids, logp, workspace, stream=None, id_dtype=None):
    fn = _fn("tt_token_logp")
    _b._check(_b._calls.token_logp(fn, tokens, vocab, k, dtype, tX, scale, X, _id_dtype(ids, id_dtype), ids, logp, workspace, _b._stream(stream)),
              "tt_token_logp")


# ------------------------------------------------ activations kept in 8 bits

def tt_pack8(rows, cols, k, dtype, t, X, Q, S, stream=None):
    fn = _fn("tt_pack8")
    _b._check(_b._calls.pack8(fn, rows, cols, k, dtype, t, X, Q, S, _b._stream(stream)), "tt_pack8")


def tt_unpack8(rows, cols, k, dtype, t, Q, S, X, stream=None):
    fn = _fn("tt_unpack8")
    _b._check(_b._calls.pack8(fn, rows, cols, k, dtype, t, Q, S, X, _b._stream(stream)), "tt_unpack8")


def tt_fc_packed_workspace_bytes(lay, batch, k, dtype, tX, tW, tY, tdY=None, tdX=None, forms_dgrad=None, forms_wgrad=None, with_dx=True):
    t = _b._tiling
    return _sized("tt_fc_packed_workspace_bytes", ctypes.byref(lay), ctypes.c_int64(batch), k, _b._dtype(dtype), t(tX), t(tW), t(tY),
                  _b._t_or(tdY, tY), _b._t_or(tdX, tX), _b._forms(forms_dgrad), _b._forms(forms_wgrad), 1 if with_dx else 0)


def tt_fc_backward_packed(lay, batch, k, dtype, tX, tW, tY, tdY, tdX, forms_dgrad, forms_wgrad, XQ, XS, W, YQ, YS, dY, dX, dW,
                          workspace=None, stream=None):
    fn = _fn("tt_fc_backward_packed")
    _b._check(_b._calls.backward_packed(fn, lay, batch, k, dtype, tX, tW, tY, tdY, tX if tdX is None else tdX, forms_dgrad, forms_wgrad, XQ, XS, W,
                                        YQ, YS, dY, dX, dW, workspace, _b._stream(stream)), "tt_fc_backward_packed")
