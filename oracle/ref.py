"""Python face of the fp64 oracle -- TEST INFRASTRUCTURE ONLY (see wmdec_oracle.c).

Every function takes and returns float64 numpy arrays in logical NCHW order.
The per-operator arithmetic lives in wmdec_oracle.c (direct loops); this file
only composes operators into the blocks and the decoder graph.  The operator
list is the one the paper's vertical fusion names (Sec. IV-B-1: Upsample,
Conv2d, GroupNorm, SiLU); by the paper's cost model (Eq. 8 against Eq. 9) the
fused path must produce the values of the unfused graph, which is what is
written here.  The decoder topology is not given by the paper; the reading used
is documented at `decoder`.
"""
import ctypes
import math
import os

import numpy as np

from . import build as _build

_lib = None
_D = ctypes.POINTER(ctypes.c_double)


def _load():
    global _lib
    if _lib is None:
        path = _build.build(force=False)
        _lib = ctypes.CDLL(path)
        for name in ("orc_gn_stats", "orc_silu", "orc_gn_apply", "orc_conv2d",
                     "orc_upsample2x", "orc_attention_core"):
            getattr(_lib, name).restype = None
    return _lib


def _p(a):
    return a.ctypes.data_as(_D)


def _f64(a):
    return np.ascontiguousarray(a, dtype=np.float64)


def gn_stats(x, groups, eps):
    """Per (sample, group) mean and 1/sqrt(biased var + eps): two passes."""
    x = _f64(x)
    n, c, h, w = x.shape
    assert c % groups == 0
    mean = np.empty((n, groups))
    rstd = np.empty((n, groups))
    _load().orc_gn_stats(_p(x), n, c, h, w, groups, ctypes.c_double(eps), _p(mean), _p(rstd))
    return mean, rstd


def silu(x):
    x = _f64(x)
    y = np.empty_like(x)
    _load().orc_silu(_p(x), ctypes.c_size_t(x.size), _p(y))
    return y


def group_norm(x, groups, eps, gamma, beta, apply_silu=False):
    """gamma*(x-mean)*rstd+beta per channel, optionally followed by SiLU."""
    x = _f64(x)
    n, c, h, w = x.shape
    mean, rstd = gn_stats(x, groups, eps)
    gamma = _f64(gamma)
    beta = _f64(beta)
    assert gamma.shape == (c,) and beta.shape == (c,)
    y = np.empty_like(x)
    _load().orc_gn_apply(_p(x), n, c, h, w, groups, _p(mean), _p(rstd), _p(gamma), _p(beta),
                         1 if apply_silu else 0, _p(y))
    return y


def conv2d(x, w, b=None):
    """k x k cross-correlation, stride 1, zero padding k//2 (k in {1,3})."""
    x = _f64(x)
    w = _f64(w)
    n, cin, h, wd = x.shape
    cout, cin2, k, k2 = w.shape
    assert cin == cin2 and k == k2 and k in (1, 3)
    bp = None
    if b is not None:
        b = _f64(b)
        assert b.shape == (cout,)
        bp = _p(b)
    y = np.empty((n, cout, h, wd))
    _load().orc_conv2d(_p(x), _p(w), bp, n, cin, cout, h, wd, k, _p(y))
    return y


def upsample2x(x):
    """Nearest 2x: out[.., y, x] = in[.., y//2, x//2]."""
    x = _f64(x)
    n, c, h, w = x.shape
    y = np.empty((n, c, 2 * h, 2 * w))
    _load().orc_upsample2x(_p(x), n, c, h, w, _p(y))
    return y


def upconv(x, w, b=None):
    """3x3 conv of the materialised 2x-upsampled tensor (padding on the upsampled grid)."""
    return conv2d(upsample2x(x), w, b)


def resblock(x, p, groups=32, eps=1e-6):
    """x -> S(x) + conv2(SiLU(GN2(conv1(SiLU(GN1(x)))))); S = 1x1 conv iff 'shortcut.w' present.

    p maps 'norm1.gamma', 'norm1.beta', 'conv1.w', 'conv1.b', 'norm2.*', 'conv2.*'
    (and optionally 'shortcut.w', 'shortcut.b') to arrays.
    """
    h = group_norm(x, groups, eps, p["norm1.gamma"], p["norm1.beta"], apply_silu=True)
    h = conv2d(h, p["conv1.w"], p["conv1.b"])
    h = group_norm(h, groups, eps, p["norm2.gamma"], p["norm2.beta"], apply_silu=True)
    h = conv2d(h, p["conv2.w"], p["conv2.b"])
    s = conv2d(x, p["shortcut.w"], p["shortcut.b"]) if "shortcut.w" in p else _f64(x)
    return s + h


def attention_core(q, k, v, scale):
    """softmax_rows(q k^T * scale) v for token-major [T, d] matrices."""
    q, k, v = _f64(q), _f64(k), _f64(v)
    t, d = q.shape
    assert k.shape == (t, d) and v.shape == (t, d)
    o = np.empty((t, d))
    _load().orc_attention_core(_p(q), _p(k), _p(v), t, d, ctypes.c_double(scale), _p(o))
    return o


def attention_block(x, p, groups=32, eps=1e-6):
    """Single-head spatial self-attention with residual.

    h = GN(x) (no SiLU); q,k,v = 1x1 convs of h with bias; tokens are the pixels
    in row-major (y*W + x) order; scores scaled by 1/sqrt(C); out = x + proj(o).
    p maps 'norm.gamma', 'norm.beta', 'q.w','q.b','k.w','k.b','v.w','v.b','proj.w','proj.b'.
    """
    x = _f64(x)
    n, c, hh, ww = x.shape
    h = group_norm(x, groups, eps, p["norm.gamma"], p["norm.beta"], apply_silu=False)
    q = conv2d(h, p["q.w"], p["q.b"])
    k = conv2d(h, p["k.w"], p["k.b"])
    v = conv2d(h, p["v.w"], p["v.b"])
    o = np.empty_like(x)
    for i in range(n):
        tok = lambda a: np.ascontiguousarray(a[i].reshape(c, hh * ww).T)  # [T, C]
        oi = attention_core(tok(q), tok(k), tok(v), 1.0 / math.sqrt(c))
        o[i] = oi.T.reshape(c, hh, ww)
    return x + conv2d(o, p["proj.w"], p["proj.b"])


def _sub(weights, prefix):
    pl = len(prefix) + 1
    return {k[pl:]: v for k, v in weights.items() if k.startswith(prefix + ".")}


def decoder(z, weights, level_channels=(512, 512, 256, 128), resblocks_per_level=3,
            groups=32, eps=1e-6):
    """Latent z[N,Cz,h,w] -> frame [N,Cout,8h,8w].

    Topology (the paper gives none; this is the reading of the workload
    description): conv_in 3x3 Cz->C0; mid = ResBlock(C0), attention, ResBlock(C0);
    for each level l: `resblocks_per_level` ResBlocks, the first one mapping the
    previous level's channels to this level's (1x1 conv shortcut when they
    differ), then -- except after the last level -- nearest-2x upsample followed
    by a 3x3 conv that keeps the channel count; finally GN -> SiLU -> conv_out.
    """
    x = conv2d(z, weights["conv_in.w"], weights["conv_in.b"])
    x = resblock(x, _sub(weights, "mid.res1"), groups, eps)
    x = attention_block(x, _sub(weights, "mid.attn"), groups, eps)
    x = resblock(x, _sub(weights, "mid.res2"), groups, eps)
    nlev = len(level_channels)
    for l in range(nlev):
        for i in range(resblocks_per_level):
            x = resblock(x, _sub(weights, f"up.{l}.res{i}"), groups, eps)
        if l + 1 < nlev:
            x = upconv(x, weights[f"up.{l}.upsample.w"], weights[f"up.{l}.upsample.b"])
    x = group_norm(x, groups, eps, weights["norm_out.gamma"], weights["norm_out.beta"], apply_silu=True)
    return conv2d(x, weights["conv_out.w"], weights["conv_out.b"])


def latent_extrapolate(z_prev, v_prev, lam):
    """Hit branch of the latent-extrapolation algorithm (Sec. IV-C, Alg. 2): the world model is skipped and the
    next latent is the first-order Taylor step of that section, z_t = z_{t-1} + lambda * v_{t-1}, with the motion
    vector v_{t-1} = z_{t-1} - z_{t-2} standing in for dz/dt."""
    return _f64(z_prev) + float(lam) * _f64(v_prev)


def extrapolated_latents(z_prev, v_prev, lam, hits):
    """`hits` consecutive hit steps of Alg. 2.  The motion vector is only updated on a miss, so every step adds the
    same lambda * v to the latent the previous step produced.  Returns [hits, ...]: the latent of every step."""
    z = _f64(z_prev)
    out = []
    for _ in range(int(hits)):
        z = latent_extrapolate(z, v_prev, lam)
        out.append(z)
    return np.stack(out) if out else np.empty((0,) + z.shape)


def adaln_modulation(c, p, apply_silu=True):
    """The AdaLN block's three small projections of the conditioning vector as the unfused graph runs them
    (Sec. IV-B-2: one small product per parameter): with a = SiLU(c) (the usual activation in front of the
    modulation; a = c if apply_silu is false),
        shift = W_shift a + b_shift,   scale = W_scale a + b_scale,   gate = W_gate a + b_gate.
    c: [batch, d_cond]; p maps 'shift.w', 'scale.w', 'gate.w' ([d_model, d_cond]) and '.b' ([d_model]).
    Returns (shift, scale, gate), each [batch, d_model].  Horizontal fusion stores the three matrices as one block
    and runs one product; it must return exactly these values, concatenated."""
    a = silu(c) if apply_silu else _f64(c)
    out = []
    for name in ("shift", "scale", "gate"):
        w, b = _f64(p[name + ".w"]), _f64(p[name + ".b"])
        y = np.empty((a.shape[0], w.shape[0]))
        for i in range(a.shape[0]):          # one matrix-vector product per conditioning vector and parameter
            y[i] = w @ a[i] + b
        out.append(y)
    return tuple(out)


def rel_err(got, want):
    """max|got-want| / rms(want): the comparison metric of every parity test."""
    want = np.asarray(want, dtype=np.float64)
    got = np.asarray(got, dtype=np.float64)
    rms = math.sqrt(float(np.mean(want * want)))
    return float(np.max(np.abs(got - want))) / (rms if rms > 0 else 1.0)


# ------------------------------------------------------------------ around the AdaLN projections of a transformer block
def row_norm(v, kind="none", eps=0.0, weight=None, bias=None):
    """Norm of the rows (last dimension): "none", "layer" (biased variance, two passes) or "rms", then weight and bias."""
    v = _f64(v)
    if kind == "none":
        return v
    mean = v.mean(-1, keepdims=True) if kind == "layer" else 0.0
    out = (v - mean) / np.sqrt(((v - mean) ** 2).mean(-1, keepdims=True) + eps)
    if weight is not None:
        out = out * _f64(weight)
    return out if bias is None else out + _f64(bias)


def gated_residual(x, h, post=(), gate=None, res_scale=1.0):
    """x + res_scale * gate * P(h); x, h [n,t,d], gate [n,d]."""
    b = row_norm(h, *post)
    return _f64(x) + res_scale * (b if gate is None else b * _f64(gate)[:, None])


def norm_modulate(x, pre=(), scale=None, shift=None):
    """N(x) * (1 + scale) + shift; scale, shift [n,d]."""
    y = row_norm(x, *pre)
    if scale is not None:
        y = y * (1.0 + _f64(scale)[:, None])
    return y if shift is None else y + _f64(shift)[:, None]


def rope_frequencies(axis_dims, base=10000.0, scaling="none", factor=1.0, trained_length=1.0, low_turns=1.0, high_turns=4.0):
    out = []
    for dim in axis_dims:
        for j in range(dim // 2):
            b = base * factor ** (dim / (dim - 2)) if scaling == "base" else base
            f = b ** (-2.0 * j / dim)
            if scaling == "linear":
                f /= factor
            if scaling == "ramp":
                w = min(max((trained_length * f / (2 * math.pi) - low_turns) / (high_turns - low_turns), 0.0), 1.0)
                f = f * (w + (1 - w) / factor)
            out.append(f)
    return np.array(out)


def rope(x, positions, freq, axis_dims, interleaved=False, inverse=False, magnitude=1.0):
    """x [n,t,heads,d], positions [n,t,axes]; pair after pair."""
    x = _f64(x)
    out, first, at = x.copy(), 0, 0
    for axis, dim in enumerate(axis_dims):
        for j in range(dim // 2):
            c0, c1 = (first + 2 * j, first + 2 * j + 1) if interleaved else (first + j, first + j + dim // 2)
            theta = np.asarray(positions)[:, :, axis].astype(np.float64)[:, :, None] * freq[at + j] * (-1.0 if inverse else 1.0)
            c, s = magnitude * np.cos(theta), magnitude * np.sin(theta)
            out[..., c0] = x[..., c0] * c - x[..., c1] * s
            out[..., c1] = x[..., c0] * s + x[..., c1] * c
        first, at = first + dim, at + dim // 2
    return out


def cross_attention(q, k, v, scale, key_lens=None, key_mask=None):
    """q [n,tq,hq,d], k, v [n,tk,hk,d] -> (o, a) with o = softmax over the valid keys v, a = the same weights times |v|; a query with
    no valid key has zeros."""
    q, k, v = _f64(q), _f64(k), _f64(v)
    n, tq, hq, d = q.shape
    tk, hk = k.shape[1:3]
    o, a = np.zeros((n, tq, hq, d)), np.zeros((n, tq, hq, d))
    for i in range(n):
        keep = np.arange(tk) < (tk if key_lens is None else key_lens[i])
        if key_mask is not None:
            keep = keep & (np.asarray(key_mask)[i] != 0)
        if not keep.any():
            continue
        for h in range(hq):
            kk, vv = k[i, keep, h // (hq // hk)], v[i, keep, h // (hq // hk)]
            s = q[i, :, h] @ kk.T * scale
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            o[i, :, h], a[i, :, h] = p @ vv, p @ np.abs(vv)
    return o, a
