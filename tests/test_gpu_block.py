"""The operators around the AdaLN projections of a transformer block on the GPU, against the oracle in 64 bits.

Tolerances are bounds, element by element: half a step of the stored type for every rounding to it, and for fp32 arithmetic
2^-24 of the magnitudes that go into an element times the roundings on its way."""
import math

import numpy as np
import pytest
import torch

from oracle import ref
from paper_2602_00608_amd import synth, wmdec
from tests import gpu_util as G

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}          # half a step, relative to the value
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}   # half a step of the smallest numbers


def rng(seed):
    return np.random.default_rng(synth.SEED_BASE + 7000 + seed)


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(G.TORCH[dtype]).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def assert_within(got, want, tol):
    got, want = np.asarray(got), np.asarray(want)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.abs(got - want)[bad].max()), float(np.broadcast_to(tol, got.shape)[bad].max()))


# ------------------------------------------------------------------ gated residual and norms
def norm_terms(v, kind, eps, w, u):
    """Sum of the magnitudes that an element of the norm is made of (its mean among them), for the bound of the fp32 arithmetic."""
    if kind == "none":
        return np.abs(v)
    mean = np.abs(v.mean(-1, keepdims=True)) if kind == "layer" else 0.0
    about = v - v.mean(-1, keepdims=True) if kind == "layer" else v
    rstd = 1 / np.sqrt((about ** 2).mean(-1, keepdims=True) + eps)
    # a mean off by 2^-24 of itself moves the element by mean * rstd; the sum of d squares, taken over lanes, is good to a few steps more
    return (np.abs(v) + 2 * mean) * rstd * (1.0 if w is None else np.abs(w)) + (0.0 if u is None else np.abs(u))


STEPS = 40   # roundings on the way of an element: two sums over up to 16384 values (64 in a lane or in order, ten joins), six products


def run_norm(xdt, adt, n, t, d, post, pre, residual=True, y=True, mod="three", seed=0, offset=0, mean=0.0, alias=False, res_scale=0.8):
    r = rng(seed)
    x = G.stored(r.standard_normal((n, t, d)) * 1.3 + mean, xdt)
    h = G.stored(r.standard_normal((n, t, d)) * 0.7 + 0.3 + mean, adt) if residual else None

    def spec(kind):
        if kind == "none":
            return ("none", 0.0, None, None)
        if kind in ("layer", "rms"):
            return (kind, 1e-6, (1 + 0.2 * r.standard_normal(d)).astype(np.float32), (0.1 * r.standard_normal(d)).astype(np.float32))
        return (kind[:-1], 1e-5, None, None)          # "layer-", "rms-": without weight and bias
    post, pre = spec(post) if residual else spec("none"), spec(pre) if y else spec("none")
    m = (0.4 * r.standard_normal((n, 3 * d))).astype(np.float32)
    md = G.dev_f32(m)
    shift, scale, gate = [m[:, i * d:(i + 1) * d] for i in range(3)] if mod == "three" else (None, None, None)
    views = [md[:, i * d:(i + 1) * d] for i in range(3)] if mod == "three" else (None, None, None)

    def shifted(a, dtype):
        big = torch.zeros(a.size + offset, dtype=G.TORCH[dtype], device="cuda")
        view = big[offset:].view(a.shape)
        view.copy_(dev(a, dtype))
        return view

    xd, hd = shifted(x, xdt), shifted(h, adt) if residual else None
    if alias:
        xo, yo, checks = (xd if residual else None), (hd if residual else xd) if y else None, []
    else:
        xo, c1 = G.canaried((n, t, d), G.TORCH[xdt]) if residual else (None, lambda: None)
        yo, c2 = G.canaried((n, t, d), G.TORCH[adt]) if y else (None, lambda: None)
        checks = [c1, c2]

    def on_device(s):
        return wmdec.Norm(s[0], s[1], *(None if v is None else G.dev_f32(v) for v in s[2:]))
    wmdec.residual_norm(xd, hd, on_device(post), views[2] if residual else None, res_scale if residual else 1.0, xo, on_device(pre),
                        views[1] if y else None, views[0] if y else None, yo)
    torch.cuda.synchronize()
    for c in checks:
        c()
    stream = x.astype(np.float64)
    if residual:
        want = ref.gated_residual(x, h, post, gate, res_scale)
        g = np.ones((n, d)) if gate is None else np.abs(gate)
        terms = np.abs(x) + abs(res_scale) * g[:, None] * norm_terms(h.astype(np.float64), *post)
        assert_within(host(xo), want, HALF[xdt] * np.abs(want) + TINY[xdt] + STEPS * U * terms)
        stream = host(xo)                             # the norm is of what is stored
    if y:
        want = ref.norm_modulate(stream, pre, scale, shift)
        terms = norm_terms(stream, *pre) * (1.0 if scale is None else 1 + np.abs(scale)[:, None]) + (0.0 if shift is None else np.abs(shift)[:, None])
        assert_within(host(yo), want, HALF[adt] * np.abs(want) + TINY[adt] + STEPS * U * terms)
    return (host(xo) if residual else None), (host(yo) if y else None)


@pytest.mark.parametrize("xdt, adt", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("f32", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("n, t, d", [(1, 1, 1920), (2, 7, 1920), (3, 5, 64), (1, 3, 1001), (2, 33, 8)])
def test_residual_norm_types(xdt, adt, n, t, d):
    run_norm(xdt, adt, n, t, d, "none", "layer", seed=1)
    run_norm(xdt, adt, n, t, d, "rms", "rms", seed=2)


@pytest.mark.parametrize("d", [1, 2, 7, 9, 63, 65, 72, 128, 136, 256, 257, 504, 512, 520, 768, 1024, 1152, 2040, 2048, 4095, 4096, 8192, 8200, 12345, 16384])
def test_residual_norm_widths(d):
    run_norm("bf16", "bf16", 2, 9, d, "layer", "rms", seed=3)
    run_norm("f32", "f32", 2, 2, d, "none", "layer", seed=4)


@pytest.mark.parametrize("post", ["none", "layer", "rms-"])
@pytest.mark.parametrize("pre", ["none", "layer-", "rms"])
@pytest.mark.parametrize("mod", ["three", None])
def test_residual_norm_parts(post, pre, mod):
    for d in (320, 1000):
        run_norm("f16", "f16", 2, 5, d, post, pre, mod=mod, seed=5)
        run_norm("f32", "bf16", 2, 5, d, post, "none", y=False, mod=mod, seed=6)
        run_norm("bf16", "bf16", 2, 5, d, "none", pre, residual=False, mod=mod, seed=7)


@pytest.mark.parametrize("xdt, adt", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("f32", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("d", [7, 40, 72, 320, 379, 1000, 1001, 1152, 1920, 4104, 8200])
def test_residual_norm_of_a_bare_post_norm(xdt, adt, d):
    """No weight, no bias, no gate: what a row's last lanes hold past its channels is no part of the next norm."""
    for post, pre in (("layer-", "layer"), ("layer-", "layer-"), ("layer-", "rms-"), ("rms-", "layer-")):
        for mean in (0.0, 5.0):
            for offset in (0, 1):
                run_norm(xdt, adt, 2, 5, d, post, pre, mod=None, mean=mean, offset=offset, seed=20)


def test_residual_norm_unaligned_in_place_and_far_from_zero():
    for offset in (1, 4, 8):
        run_norm("bf16", "bf16", 2, 5, 640, "layer", "layer", offset=offset, seed=8)
        run_norm("f32", "f16", 1, 5, 648, "rms", "layer", offset=offset, seed=8)
    for d in (64, 640, 1001, 1920, 9000):
        run_norm("bf16", "bf16", 2, 70, d, "rms", "layer", alias=True, seed=9)
        run_norm("f32", "f32", 2, 70, d, "none", "layer", residual=False, alias=True, seed=9)
    run_norm("f32", "f32", 2, 5, 1920, "layer", "layer", mean=300.0, seed=10)
    run_norm("f32", "f32", 1, 5, 1920, "none", "rms", res_scale=-1e4, seed=11)


def test_residual_norm_many_rows():
    for n, t, d in ((1, 5400, 1920), (3, 1801, 72), (1, 20000, 16), (2, 700, 4104)):
        run_norm("bf16", "bf16", n, t, d, "none", "layer", seed=12)


@pytest.mark.parametrize("d", [256, 257, 264, 379, 384, 504, 511, 512, 513])
def test_residual_norm_rows_of_a_whole_wavefront(d):
    """Up to 512 channels a row is a wavefront's and a workgroup has four of them: numbers of rows that are no multiple of that, one and several rounds of them."""
    for xdt, adt in (("bf16", "bf16"), ("f32", "f16")):
        for n, t in ((1, 1), (1, 3), (3, 5), (2, 2051), (1, 9001)):
            run_norm(xdt, adt, n, t, d, "layer-", "layer", seed=17)
        for offset in (0, 1):
            run_norm(xdt, adt, 2, 6, d, "rms", "layer-", mod=None, offset=offset, seed=18)
            run_norm(xdt, adt, 1, 7, d, "none", "rms", residual=False, offset=offset, seed=19)


def test_residual_norm_one_vector_for_all_samples_and_rows_alike():
    """gate, scale and shift expanded over the samples (stride 0); a row's bits depend neither on its place nor on the other rows."""
    r = rng(13)
    x, h = dev(r.standard_normal((1, 1, 1920)), "bf16"), dev(r.standard_normal((1, 1, 1920)), "bf16")
    m = G.dev_f32(0.3 * r.standard_normal((1, 1920)))
    spec = wmdec.Norm("layer", 1e-6)
    outs = []
    for n, t in ((1, 1), (3, 1), (1, 5), (2, 1999)):
        xo, y = torch.empty((n, t, 1920), dtype=torch.bfloat16, device="cuda"), torch.empty((n, t, 1920), dtype=torch.bfloat16, device="cuda")
        e = m.expand(n, 1920)
        wmdec.residual_norm(x.expand(n, t, 1920).contiguous(), h.expand(n, t, 1920).contiguous(), spec, e, 1.0, xo, spec, e, e, y)
        assert torch.equal(xo, xo[:1, :1].expand_as(xo)) and torch.equal(y, y[:1, :1].expand_as(y))
        outs.append((xo[0, 0], y[0, 0]))
    assert all(torch.equal(a, outs[0][0]) and torch.equal(b, outs[0][1]) for a, b in outs)


def test_residual_norm_rows_of_many_samples():
    """Samples that share their vectors, or have none, count as one; the bits are those of samples with equal vectors."""
    r = rng(14)
    x, h = dev(r.standard_normal((777, 1, 96)), "f16"), dev(r.standard_normal((777, 1, 96)), "f16")
    w, m = G.dev_f32(1 + 0.1 * r.standard_normal(96)), G.dev_f32(0.3 * r.standard_normal((1, 96)))
    spec = wmdec.Norm("rms", 1e-6, w)
    got = []
    for vectors in (m.expand(777, 96), m.expand(777, 96).contiguous()):
        xo, y = torch.empty_like(x), torch.empty_like(x)
        wmdec.residual_norm(x, h, spec, vectors, 0.5, xo, spec, vectors, vectors, y)
        got.append((xo, y))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    run_norm("f16", "f16", 777, 1, 96, "rms", "layer", seed=15)
    run_norm("f32", "bf16", 777, 3, 95, "layer", "rms", mod="none", seed=16)


def test_residual_norm_not_a_number_stays_in_its_row():
    x, h = torch.randn((1, 40, 1920), device="cuda"), torch.randn((1, 40, 1920), device="cuda")
    x[0, 7, 3], h[0, 9, 1919], x[0, 11, 0] = float("nan"), float("inf"), float("inf")
    x[0, 13] = 0.0
    h[0, 13] = 0.0
    xo, y = torch.empty_like(x), torch.empty_like(x)
    wmdec.residual_norm(x, h, None, None, 1.0, xo, wmdec.Norm("layer", 1e-6), None, None, y)
    rows = torch.isnan(y).all(-1)[0].nonzero().flatten().tolist()
    assert rows == [7, 9, 11] and not torch.isnan(y[0, [i for i in range(40) if i not in rows]]).any()
    assert not y[0, 13].any()


def test_residual_norm_past_32_bit_offsets():
    t, d = (1 << 21) + 5, 1032                         # 4.3 GB a tensor
    x = torch.zeros((1, t, d), dtype=torch.bfloat16, device="cuda")
    x[0, -3:] = torch.randn((3, d), device="cuda").bfloat16()
    y = torch.empty_like(x)
    wmdec.residual_norm(x, None, None, None, 1.0, None, wmdec.Norm("rms", 1e-6), None, None, y)
    want = ref.norm_modulate(host(x[:, -3:]), ("rms", 1e-6))
    assert_within(host(y[:, -3:]), want, (HALF["bf16"] + STEPS * U) * np.abs(want))
    assert not y[0, :3].any() and not y[0, t // 2].any()


# ------------------------------------------------------------------ rotary positions
def run_rope(dtype, n, t, hq, hk, d, dims, inter, inverse=False, magnitude=1.0, scaling="none", factor=1.0, place=lambda s: s, shared=False, in_place=False, far=1 << 17, seed=0):
    r = rng(100 + seed)
    sc = dict(base=10000.0, scaling=scaling, factor=factor, trained_length=2048.0, low_turns=1.0, high_turns=4.0)
    freq = torch.empty(sum(dims) // 2, dtype=torch.float64, device="cuda")
    wmdec.rope_frequencies(dims, freq, **sc)
    f = ref.rope_frequencies(dims, **sc)
    assert_within(freq.cpu().numpy(), f, 8e-16 * 64 * f)
    pos = r.integers(-far, far, (1 if shared else n, t, len(dims)))
    posd = torch.from_numpy(pos.astype(np.int32)).cuda()
    q, k = G.stored(r.standard_normal((n, t, hq, d)) * 3, dtype), G.stored(r.standard_normal((n, t, max(hk, 1), d)), dtype)
    qd, kd = place(dev(q, dtype)), place(dev(k, dtype)) if hk else None
    if in_place:
        qo, ko, checks = qd, kd, []
    else:
        qo, c1 = G.canaried((n, t, hq, d), G.TORCH[dtype])
        ko, c2 = G.canaried((n, t, hk, d), G.TORCH[dtype]) if hk else (None, lambda: None)
        checks = [c1, c2]
    wmdec.rope(qd, kd, posd[0] if shared else posd, freq, dims, qo, ko, interleaved=inter, inverse=inverse, magnitude=magnitude)
    torch.cuda.synchronize()
    for c in checks:
        c()
    mag = float(np.float32(magnitude))
    for x, o in ((q, qo), (k, ko))[:2 if hk else 1]:
        want = ref.rope(x, np.broadcast_to(pos, (n, t, len(dims))), f, dims, inter, inverse, mag)
        first, both = 0, np.abs(x).astype(np.float64)  # |u| + |v| of the pair that an element belongs to
        for dim in dims:
            part = np.abs(x[..., first:first + dim]).astype(np.float64)
            s = part[..., 0::2] + part[..., 1::2] if inter else part[..., :dim // 2] + part[..., dim // 2:]
            both[..., first:first + dim] = np.repeat(s, 2, -1) if inter else np.concatenate((s, s), -1)
            first += dim
        # sine and cosine: the angle reduced in 64 bits, then some four fp32 roundings; two products and their sum
        tol = HALF[dtype] * np.abs(want) + TINY[dtype] + 8 * U * abs(mag) * both
        assert_within(host(o), want, tol)
        assert np.array_equal(host(o)[..., sum(dims):], x[..., sum(dims):].astype(np.float64))
    return qo, ko


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("hq, hk, d, dims", [(30, 30, 64, (16, 24, 24)), (8, 2, 128, (96,)), (4, 4, 64, (64,)), (3, 1, 72, (72,)), (5, 0, 30, (14, 6)), (1, 1, 2, (2,)),
                                             (2, 2, 48, (8,)), (2, 1, 256, (128, 128)), (1, 1, 96, (32, 30, 2)), (2, 2, 33, (32,))])
def test_rope(dtype, inter, hq, hk, d, dims):
    for n, t in ((1, 1), (2, 37)):
        run_rope(dtype, n, t, hq, hk, d, dims, inter, seed=d)
    run_rope(dtype, 2, 5, hq, hk, d, dims, inter, inverse=True, magnitude=1.3, shared=True, seed=d + 1)


@pytest.mark.parametrize("scaling, factor", [("linear", 4.0), ("base", 8.0), ("ramp", 16.0)])
def test_rope_scaled(scaling, factor):
    run_rope("f32", 1, 65, 4, 2, 128, (128,), False, scaling=scaling, factor=factor, magnitude=1.2, seed=3)
    run_rope("bf16", 2, 9, 2, 2, 64, (32, 32), True, scaling=scaling, factor=factor, seed=4)


def test_rope_far_positions():
    """Positions over the whole range of int32: the angle (2^31 radians at most) is good to 2^-22 in 64 bits on both sides."""
    r = rng(150)
    x = r.standard_normal((1, 64, 2, 64)).astype(np.float32)
    pos = np.concatenate([r.integers(-2 ** 31, 2 ** 31, (1, 60, 1)), np.array([0, 1, -2 ** 31, 2 ** 31 - 1]).reshape(1, 4, 1)], 1)
    f = ref.rope_frequencies((64,))
    freq = torch.from_numpy(f).cuda()
    out = torch.empty((1, 64, 2, 64), device="cuda")
    wmdec.rope(dev(x, "f32"), None, torch.from_numpy(pos.astype(np.int32)).cuda(), freq, (64,), out, None)
    both = np.tile(np.abs(x[..., :32]) + np.abs(x[..., 32:]), 2)
    assert_within(host(out), ref.rope(x, pos, f, (64,)), (8 * U + 2.0 ** -21) * both)
    assert np.array_equal(host(out)[0, 60], x[0, 60].astype(np.float64))           # position 0 turns nothing


@pytest.mark.parametrize("inter", [False, True])
def test_rope_strided_and_in_place(inter):
    def in_qkv(s):                                     # a part of a fused projection
        n, t, h, d = s.shape
        big = torch.full((n, t, 3, h + 1, d), 7.0, dtype=s.dtype, device="cuda")
        view = big[:, :, 1, :h]
        view.copy_(s)
        return view

    def heads_first(s):
        return s.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)

    def odd_place(s):                                  # rows that are not 16-byte aligned
        n, t, h, d = s.shape
        big = torch.zeros((n, t, h, d + 3), dtype=s.dtype, device="cuda")
        big[..., 1:d + 1] = s
        return big[..., 1:d + 1]
    for place in (in_qkv, heads_first, odd_place):
        for in_place in (False, True):
            for dtype in ("bf16", "f32"):
                qo, _ = run_rope(dtype, 2, 19, 6, 2, 64, (32, 16), inter, place=place, in_place=in_place, seed=5)
                if in_place and place is in_qkv:
                    whole = qo.as_strided((2, 19, 3, 7, 64), (19 * 21 * 64, 21 * 64, 7 * 64, 64, 1), qo.storage_offset() - 7 * 64)
                    assert bool((whole[:, :, 0] == 7).all()) and bool((whole[:, :, 2] == 7).all()) and bool((whole[:, :, 1, 6] == 7).all())


def test_rope_inverse_is_the_gradient():
    r = rng(160)
    f = ref.rope_frequencies((24, 16))
    freq = torch.from_numpy(f).cuda()
    pos = torch.from_numpy(r.integers(0, 500, (2, 5, 2)).astype(np.int32)).cuda()
    x, g = r.standard_normal((2, 5, 3, 48)), r.standard_normal((2, 5, 3, 48)).astype(np.float32)
    for inter in (False, True):
        grad = torch.empty((2, 5, 3, 48), device="cuda")
        wmdec.rope(dev(g, "f32"), None, pos, freq, (24, 16), grad, None, interleaved=inter, inverse=True, magnitude=1.25)
        for i in (0, 5, 13, 24, 31, 39, 47):           # differences of sum(g * rope(x)) along a channel; it is linear, so they are exact
            step = np.zeros_like(x)
            step[..., i] = 1.0
            up, down = (ref.rope(x + s * step, pos.cpu().numpy(), f, (24, 16), inter, magnitude=1.25) for s in (0.5, -0.5))
            want = (g * (up - down)).sum(-1)
            assert_within(host(grad)[..., i], want, 16 * U * 1.25 * np.abs(g).sum(-1))


def test_rope_copied_channels_keep_their_bits():
    x = torch.randn((1, 3, 2, 64), device="cuda").bfloat16()
    x[..., 40], x[..., 41], x[..., 63] = float("nan"), float("inf"), -0.0
    x[0, 0, 0, 3] = float("inf")                       # and a pair that is not finite stays a pair
    freq = torch.empty(16, dtype=torch.float64, device="cuda")
    wmdec.rope_frequencies((32,), freq)
    out = torch.empty_like(x)
    for inter in (False, True):
        wmdec.rope(x, None, torch.arange(1, 4, dtype=torch.int32, device="cuda").view(3, 1), freq, (32,), out, None, interleaved=inter, magnitude=2.0)
        assert torch.equal(out[..., 32:].view(torch.int16), x[..., 32:].view(torch.int16))
        pair = [2, 3] if inter else [3, 19]
        finite = [i for i in range(32) if i not in pair]
        assert torch.isfinite(out[0, 0, 0, finite]).all() and torch.isfinite(out[0, 1:, :, :32]).all()


def test_rope_past_32_bit_offsets():
    t = (1 << 20) + 3                                  # 4.3 GB
    x = torch.zeros((1, t, 32, 64), dtype=torch.bfloat16, device="cuda")
    x[0, -2:] = torch.randn((2, 32, 64), device="cuda").bfloat16()
    pos = torch.arange(t, dtype=torch.int32, device="cuda").view(t, 1)
    f = ref.rope_frequencies((64,))
    want = ref.rope(host(x[:, -2:]), np.array([t - 2, t - 1]).reshape(1, 2, 1), f, (64,))
    both = np.tile(np.abs(host(x[:, -2:])[..., :32]) + np.abs(host(x[:, -2:])[..., 32:]), 2)
    wmdec.rope(x, None, pos, torch.from_numpy(f).cuda(), (64,), x, None)
    assert_within(host(x[:, -2:]), want, HALF["bf16"] * np.abs(want) + 8 * U * both)
    assert not x[0, :2].any()


def test_rope_far_turns_are_exact_to_fp32():
    """The pair (1, 0) comes back as (cos, sin) of theta = position * frequency in 64 bits.  The rest within an eighth of a turn (at most 0.79) is rounded
    once to fp32, 0.79 U; the last step of the polynomial rounds once, a step of at most 1, U / 2 below 1 counted as U; its terms before and those left out
    come to 0.31 U (r^3 / 6 at most 0.081 with four roundings, 2^-28.6 of 0.71); the products by 1 and 0 and their sum round nothing.  2.1 U."""
    r = rng(151)
    pos = np.concatenate([r.integers(2 ** 30, 2 ** 31, 20000), -r.integers(2 ** 30, 2 ** 31, 20000), np.array([2 ** 31 - 1, -2 ** 31, 0, 1])]).reshape(1, -1, 1)
    f = ref.rope_frequencies((64,))
    x = np.zeros((1, pos.size, 1, 64), np.float32)
    x[..., :32] = 1.0
    out = torch.empty(x.shape, device="cuda")
    wmdec.rope(dev(x, "f32"), None, torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(f).cuda(), (64,), out, None)
    assert_within(host(out), ref.rope(x, pos, f, (64,)), 2.1 * U)


# ------------------------------------------------------------------ attention to states of another length
def cross_tolerance(dtype, q, k, want, weighted, scale, tk, v):
    """weighted: the softmax weights times |v|.  Half a step for the output; half a step for every probability in 16 bits (and half of the
    smallest f16 number, beside a largest probability of at least one); fp32 scores that are off by d + 8 roundings of |q| |k| at most,
    which moves every weight by twice that; a sum of tk probabilities and exponentials good to a few steps."""
    d = q.shape[-1]
    size = float(np.sqrt((q ** 2).sum(-1)).max() * np.sqrt((k ** 2).sum(-1)).max()) * scale if k.size else 0.0
    fp32 = 2 * (d + 8) * U * size + (math.sqrt(tk) + 64) * 2 * U
    tol = HALF[dtype] * np.abs(want) + TINY[dtype] + fp32 * weighted
    if dtype != "f32":
        tol = tol + HALF[dtype] * weighted * 1.01
    if dtype == "f16":
        tol = tol + TINY["f16"] * float(np.abs(v).sum(1).max() if v.size else 0.0)
    return tol


def run_cross(dtype, n, tq, tk, hq, hk, d, lens=None, mask=None, place=lambda s: s, std=1.5, scale=None, seed=0, poison=True, kv_place=None):
    r = rng(200 + seed)
    q = G.stored(r.standard_normal((n, tq, hq, d)) * std, dtype)
    k, v = (G.stored(r.standard_normal((n, tk, hk, d)), dtype) for _ in range(2))
    scale = float(np.float32(1 / math.sqrt(d) if scale is None else scale))
    keep = np.ones((n, tk), bool)
    if lens is not None:
        keep &= np.arange(tk)[None] < np.asarray(lens)[:, None]
    if mask is not None:
        keep &= mask != 0
    kb, vb = k.copy(), v.copy()
    if poison:                                         # what invalid keys hold does not matter
        for b in (kb, vb):
            b[~keep] = np.array([np.nan, np.inf, -np.inf, 1e4], np.float32)[r.integers(0, 4, int((~keep).sum()))][:, None, None]
    qd, (kd, vd) = place(dev(q, dtype)), (map(kv_place or place, (dev(kb, dtype), dev(vb, dtype))))
    o, check = G.canaried((n, tq, hq, d), G.TORCH[dtype])
    need = wmdec.cross_attention_workspace_bytes(qd, kd)
    ws, wcheck = G.canaried((max(need // 4, 1),), torch.float32)
    wmdec.cross_attention(qd, kd, vd, o, scale, key_lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"),
                          key_mask=None if mask is None else torch.from_numpy(mask).cuda(), workspace=ws if need else None)
    torch.cuda.synchronize()
    check()
    wcheck()
    want, weighted = ref.cross_attention(q, np.where(keep[..., None, None], k, 0), np.where(keep[..., None, None], v, 0), scale, None, keep)
    assert_within(host(o), want, cross_tolerance(dtype, q, np.where(keep[..., None, None], k, 0), want, weighted, scale, tk, v))
    return o


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [8, 24, 32, 40, 64, 72, 96, 104, 128, 136, 160, 192, 200, 256])
def test_cross_head_sizes(dtype, d):
    run_cross(dtype, 2, 150, 77, 2, 1, d, lens=[77, 70], seed=d)
    run_cross(dtype, 2, 3, 301, 4, 2, d, lens=[301, 130], seed=d + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tq", [1, 2, 31, 33, 65, 129, 257, 300])
@pytest.mark.parametrize("tk", [1, 31, 32, 63, 64, 65, 127, 129, 257, 1000])
def test_cross_lengths(dtype, tq, tk):
    run_cross(dtype, 1, tq, tk, 2, 2, 64, seed=tq * 7 + tk)


@pytest.mark.parametrize("dtype, d", [("bf16", 64), ("f16", 128), ("f32", 64), ("bf16", 256), ("f32", 128)])
@pytest.mark.parametrize("tq", [1, 40, 300])
def test_cross_masks(dtype, d, tq):
    """Lengths of zero and one, beyond tk and negative; masks with holes, whole masked tiles, nothing left, a single key."""
    tk = 333
    run_cross(dtype, 5, tq, tk, 4, 2, d, lens=[0, 1, 333, 400, -3], seed=1)
    mask = rng(9).random((5, tk)) < 0.7
    mask[0] = False
    mask[1] = np.arange(tk) == tk - 1
    mask[2, 64:256] = False
    mask[3, :200] = False
    run_cross(dtype, 5, tq, tk, 4, 2, d, mask=mask, seed=2)
    run_cross(dtype, 5, tq, tk, 4, 2, d, lens=[333, 333, 60, 150, 299], mask=mask.astype(np.uint8) * 255, seed=3)


@pytest.mark.parametrize("tq", [1, 33])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_cross_masks_of_long_states(dtype, tq):
    """Many heads, so that a range of keys is as long as they are or half as long: its mask is read in parts, of which the second has nothing, or one key."""
    mask = rng(10).random((1, 5003)) < 0.5
    mask[:, 2048:4096] = False
    run_cross(dtype, 1, tq, 5003, 512, 512, 8, mask=mask, seed=4)
    mask[:, 4095] = True
    run_cross(dtype, 1, tq, 5003, 512, 512, 8, lens=[4999], mask=mask, seed=5)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_cross_masked_keys_might_as_well_not_be_there(dtype):
    """The same bits as without the masked keys, where all keys are one range."""
    for tq, d in ((1, 64), (200, 64), (4, 128), (40, 160), (90, 256)):
        q, k, v = (torch.randn(s, device="cuda").to(G.TORCH[dtype]) for s in ((2, tq, 4, d), (2, 127, 2, d), (2, 127, 2, d)))
        keep = torch.zeros(127, dtype=torch.bool, device="cuda")
        keep[torch.randperm(127, device="cuda")[:83]] = True
        outs = []
        for kk, vv, mask in ((k, v, keep.expand(2, 127).contiguous()), (k[:, keep].contiguous(), v[:, keep].contiguous(), None),
                             (k[:, keep].contiguous(), v[:, keep].contiguous(), torch.ones((2, 83), dtype=torch.bool, device="cuda"))):
            o = torch.empty_like(q)
            need = wmdec.cross_attention_workspace_bytes(q, kk)
            wmdec.cross_attention(q, kk, vv, o, 0.1, key_mask=mask, workspace=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
            outs.append(o)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_cross_masked_keys_far_apart():
    """8 MB from token to token: less than 256 of them are within reach of one address."""
    tk, step, d = 300, 1 << 22, 64
    big = torch.zeros(tk * step, dtype=torch.float16, device="cuda")
    k, v = (big[at:].as_strided((1, tk, 2, d), (tk * step, step, d, 1)) for at in (0, 4 * d))
    k.copy_(torch.randn((1, tk, 2, d), device="cuda"))
    v.copy_(torch.randn((1, tk, 2, d), device="cuda"))
    mask = torch.rand((1, tk), device="cuda") < 0.7
    for tq in (1, 64):
        q = torch.randn((1, tq, 2, d), device="cuda").half()
        o, near = torch.empty_like(q), torch.empty_like(q)
        need = wmdec.cross_attention_workspace_bytes(q, k)
        for kk, vv, out in ((k, v, o), (k.contiguous(), v.contiguous(), near)):
            wmdec.cross_attention(q, kk, vv, out, 0.1, key_mask=mask, workspace=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
        want, weighted = ref.cross_attention(host(q), host(k), host(v), float(np.float32(0.1)), None, mask.cpu().numpy())
        for out in (o, near):
            assert_within(host(out), want, cross_tolerance("f16", host(q), host(k), want, weighted, 0.1, tk, host(v)))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_cross_grouped_heads_and_long_states(dtype):
    for tq, hq, hk in ((1, 32, 8), (1, 7, 1), (5, 8, 1), (3, 40, 2), (2, 128, 1)):
        run_cross(dtype, 2, tq, 2500, hq, hk, 64, lens=[2500, 1111], seed=hq)
    run_cross(dtype, 1, 1, 20000, 4, 2, 128, seed=50)
    run_cross(dtype, 2, 70, 5000, 2, 2, 64, lens=[5000, 3], seed=51)


def test_cross_no_keys():
    for tq in (1, 200):
        q = torch.randn((2, tq, 4, 64), device="cuda").bfloat16()
        k = torch.empty((2, 0, 2, 64), dtype=torch.bfloat16, device="cuda")
        o = torch.full_like(q, 3.0)
        need = wmdec.cross_attention_workspace_bytes(q, k)
        wmdec.cross_attention(q, k, k, o, 0.1, workspace=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
        assert not o.any()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_cross_scores_of_any_size(dtype):
    """Scores that grow along the keys (the running maximum moves in every tile), fall, are tiny, huge, or alike."""
    for tq in (1, 150):
        r = rng(300)
        n, tk, h, d = 1, 700, 2, 64
        ramp = np.linspace(-1, 1, tk)
        for slope in (60.0, -60.0, 3000.0, 1e-4, 0.0):
            q = np.ones((n, tq, h, d))
            k = G.stored(np.broadcast_to((slope * ramp / d)[None, :, None, None], (n, tk, h, d)), dtype)
            v = G.stored(r.standard_normal((n, tk, h, d)), dtype)
            o = torch.empty((n, tq, h, d), dtype=G.TORCH[dtype], device="cuda")
            qd, kd, vd = dev(q, dtype), dev(k, dtype), dev(v, dtype)
            need = wmdec.cross_attention_workspace_bytes(qd, kd)
            wmdec.cross_attention(qd, kd, vd, o, 1.0, workspace=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
            want, weighted = ref.cross_attention(q, k, v, 1.0)
            assert_within(host(o), want, cross_tolerance(dtype, q, k, want, weighted, 1.0, tk, v))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tq, tk", [(1, 1), (1, 700), (150, 700), (300, 70)])
def test_cross_scores_past_24_bits(dtype, tq, tk):
    """Scores so large that fp32 holds no fraction of them.  Keys that are alike have the same score to the bit, those of the other sign are out of reach, so the
    output is the plain mean of the values with the higher score; rows with ordinary scores stand between.  (No bound of the scores' own error: those that count are
    alike.  What is left is the sum and quotient in fp32 and the roundings to dtype, as in cross_tolerance.)"""
    r = rng(310)
    h, d = 2, 64
    v = G.stored(r.standard_normal((1, tk, h, d)), dtype)
    sign = np.where(r.random((1, tk, 1, 1)) < 0.5, 1.0, -1.0) * np.ones((1, tk, h, d))
    for size, scale in ((7.68e10, 1.0), (7.68e10, 0.3), (3.1e9, 0.125), (3.1e9, 0.0884), (4.7e8, 0.7), (4.7e8, 1.0)) + (((1e30, 0.9), (1e36, 0.11)) if dtype != "f16" else ()):
        size, scale = math.sqrt(size / d), float(np.float32(scale))
        for signs in (sign, np.ones_like(sign), -np.ones_like(sign)):
            q, k = G.stored(np.full((1, tq, h, d), size), dtype), G.stored(size * signs, dtype)
            q[:, 1::3] /= np.float32(2.0) ** np.ceil(2 * np.log2(np.float32(size)) + 9)         # (a power of two; scores below 1, where they do not vanish)
            q = G.stored(q, dtype)
            qd, kd, vd = dev(q, dtype), dev(k, dtype), dev(v, dtype)
            o = torch.empty_like(qd)
            need = wmdec.cross_attention_workspace_bytes(qd, kd)
            wmdec.cross_attention(qd, kd, vd, o, scale, workspace=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
            want, weighted = ref.cross_attention(q, k, v, scale)
            tol = HALF[dtype] * np.abs(want) + TINY[dtype] + ((math.sqrt(tk) + 64) * 2 * U + (HALF[dtype] * 1.01 if dtype != "f32" else 0.0) + 2 * (d + 8) * U) * weighted
            if dtype == "f16":
                tol = tol + TINY["f16"] * float(np.abs(v).sum(1).max())
            assert_within(host(o), want, tol)


def test_cross_not_a_number_in_valid_places():
    for tq, dtype in ((1, "bf16"), (100, "bf16"), (1, "f32"), (100, "f32")):
        q, k, v = (torch.randn(s, device="cuda").to(G.TORCH[dtype]) for s in ((1, tq, 2, 64), (1, 90, 2, 64), (1, 90, 2, 64)))
        k[0, 80, 0, 5] = float("nan")
        v[0, 3, 1, 9] = float("inf")
        q[0, tq - 1, 1, 0] = float("nan")
        o = torch.zeros_like(q)
        need = wmdec.cross_attention_workspace_bytes(q, k)
        wmdec.cross_attention(q, k, v, o, 0.1, workspace=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
        assert torch.isnan(o[0, :, 0]).all() and torch.isnan(o[0, tq - 1, 1]).all()
        if tq > 1:
            assert torch.isinf(o[0, :tq - 1, 1, 9]).all() and torch.isfinite(o[0, :tq - 1, 1, :9]).all() and torch.isfinite(o[0, :tq - 1, 1, 10:]).all()


def test_cross_strides():
    def in_qkv(s):
        n, t, h, d = s.shape
        big = torch.full((n, t, 3, h, d), float("nan"), dtype=s.dtype, device="cuda")
        big[:, :, 2] = s
        return big[:, :, 2]

    def heads_first(s):
        return s.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)

    def padded_heads(s):
        big = torch.full(s.shape[:3] + (s.shape[3] + 8,), float("nan"), dtype=s.dtype, device="cuda")
        big[..., 8:] = s
        return big[..., 8:]

    def samples_last(s):
        return s.permute(1, 2, 0, 3).contiguous().permute(2, 0, 1, 3)
    for place in (in_qkv, heads_first, padded_heads, samples_last):
        for tq in (2, 140):
            for dtype, d in (("bf16", 64), ("f16", 72), ("f32", 40)):
                run_cross(dtype, 3, tq, 203, 4, 2, d, lens=[203, 100, 7], place=place, seed=17)
    # one sample's states for all, and an output in place of a part of a fused buffer
    q, k, v = (torch.randn(s, device="cuda").bfloat16() for s in ((3, 50, 2, 64), (1, 90, 2, 64), (1, 90, 2, 64)))
    wide = torch.full((3, 50, 3, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    wmdec.cross_attention(q, k.expand(3, -1, -1, -1), v.expand(3, -1, -1, -1), wide[:, :, 1], 0.125)
    want, weighted = ref.cross_attention(host(q), np.repeat(host(k), 3, 0), np.repeat(host(v), 3, 0), 0.125)
    assert_within(host(wide[:, :, 1]), want, cross_tolerance("bf16", host(q), host(k), want, weighted, 0.125, 90, host(v)))
    assert bool((wide[:, :, 0] == 5).all()) and bool((wide[:, :, 2] == 5).all())


def test_cross_past_32_bit_offsets():
    """k and v are every 4-million-th element on of a 9.6 GB buffer; the second sample starts past 2^32 bytes."""
    tk, stride = 600, 4 << 20
    big = torch.empty((2, tk, stride), dtype=torch.bfloat16, device="cuda")
    r = rng(400)
    q, k, v = (G.stored(r.standard_normal(s), "bf16") for s in ((2, 3, 2, 64), (2, tk, 2, 64), (2, tk, 2, 64)))
    kd, vd = (big[:, :, i * 128:(i + 1) * 128].view(2, tk, 2, 64) for i in range(2))
    kd.copy_(dev(k, "bf16"))
    vd.copy_(dev(v, "bf16"))
    for tq in (3, 1):
        qd = dev(q[:, :tq], "bf16")
        o = torch.empty_like(qd)
        need = wmdec.cross_attention_workspace_bytes(qd, kd)
        wmdec.cross_attention(qd, kd, vd, o, 0.125, workspace=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
        want, weighted = ref.cross_attention(q[:, :tq], k, v, 0.125)
        assert_within(host(o), want, cross_tolerance("bf16", q, k, want, weighted, 0.125, tk, v))


def test_cross_bits_of_a_sample_do_not_depend_on_the_batch():
    for dtype in ("bf16", "f32"):
        for tq, tk in ((1, 3000), (60, 700), (300, 200)):
            q, k, v = (torch.randn(s, device="cuda").to(G.TORCH[dtype]) for s in ((5, tq, 4, 64), (5, tk, 2, 64), (5, tk, 2, 64)))
            lens = torch.tensor([tk, 7, tk // 2, 0, tk - 1], dtype=torch.int32, device="cuda")

            def run(s):
                o = torch.empty_like(q[s])
                need = wmdec.cross_attention_workspace_bytes(q[s], k[s])
                ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")    # (NaN all over)
                wmdec.cross_attention(q[s], k[s], v[s], o, 0.125, key_lens=lens[s].contiguous(), workspace=ws)
                return o
            whole = run(slice(0, 5))
            assert torch.equal(whole, run(slice(0, 5)))
            for i in range(5):
                assert torch.equal(run(slice(i, i + 1))[0], whole[i])


@pytest.mark.parametrize("dtype, n, tq, tk, hq, hk, d", [("f16", 32, 1, 8192, 32, 8, 128), ("f32", 32, 1, 8192, 32, 8, 128), ("f16", 4, 700, 3000, 4, 4, 96), ("f32", 12, 9, 5000, 8, 2, 40)])
def test_cross_ranges_are_joined_alike_in_every_batch(dtype, n, tq, tk, hq, hk, d):
    """Many ranges of keys, and samples enough to make the join's launch another one."""
    q, k, v = (torch.randn(s, device="cuda").to(G.TORCH[dtype]) for s in ((n, tq, hq, d), (n, tk, hk, d), (n, tk, hk, d)))

    def run(s):
        o = torch.empty_like(q[s])
        need = wmdec.cross_attention_workspace_bytes(q[s], k[s])
        assert need
        wmdec.cross_attention(q[s], k[s], v[s], o, d ** -0.5, workspace=torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda"))
        return o
    whole = run(slice(0, n))
    for i in (0, 1, n // 2, n - 1):
        assert torch.equal(run(slice(i, i + 1))[0], whole[i]), i


def test_cross_more_rows_of_many_ranges_than_a_joining_launch_takes_at_once():
    """65 samples of 4 key heads and 32 rows each, 17 ranges of keys: 8320 rows with a workgroup each, in a launch of at most 8192."""
    q, k, v = (torch.randn(s, device="cuda").half() for s in ((65, 4, 32, 256), (1, 4400, 4, 256), (1, 4400, 4, 256)))
    k, v = k.expand(65, -1, -1, -1), v.expand(65, -1, -1, -1)

    def run(s):
        o = torch.empty_like(q[s])
        wmdec.cross_attention(q[s], k[s], v[s], o, 0.0625, workspace=torch.empty(wmdec.cross_attention_workspace_bytes(q[s], k[s]), dtype=torch.uint8, device="cuda"))
        return o
    whole = run(slice(0, 65))
    for i in (0, 31, 63, 64):
        assert torch.equal(run(slice(i, i + 1))[0], whole[i]), i
    want, weighted = ref.cross_attention(host(q[64:]), host(k[:1]), host(v[:1]), 0.0625)
    assert_within(host(whole[64:]), want, cross_tolerance("f16", host(q[64:]), host(k[:1]), want, weighted, 0.0625, 4400, host(v[:1])))


def test_workspace_too_small_is_refused():
    q, k = torch.zeros((1, 1, 32, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 32768, 8, 128), dtype=torch.bfloat16, device="cuda")
    need = wmdec.cross_attention_workspace_bytes(q, k)
    o = torch.full_like(q, 9.0)
    if need:
        for ws in (None, torch.zeros(need - 1, dtype=torch.uint8, device="cuda")):
            with pytest.raises(wmdec.WmdecError) as e:
                wmdec.cross_attention(q, k, k, o, 0.1, workspace=ws)
            assert e.value.status == wmdec.ERR_WORKSPACE
    torch.cuda.synchronize()
    assert bool((o == 9).all())


# ------------------------------------------------------------------ together
class Block:
    """One transformer block out of the library's operators: AdaLN projections, modulated norm, fused q/k/v projection, rotary positions in place,
    attention among the tokens, output projection, gated residual and next norm, attention to the conditioning, gated residual."""

    def __init__(self, n, gh, gw, tc, heads, d, dtype, seed):
        r = rng(500 + seed)
        self.n, self.t, self.tc, self.heads, self.d, self.c, self.dtype, self.g = n, gh * gw, tc, heads, d, heads * d, dtype, (gh, gw)
        c = self.c
        self.np = {"x": r.standard_normal((n, self.t, c)), "cond": r.standard_normal((n, tc, c)), "a": r.standard_normal((n, c)),
                   "w_ada": r.standard_normal((6 * c, c)) / math.sqrt(c) * 0.5, "b_ada": 0.05 * r.standard_normal(6 * c)}
        for name, rows in (("qkv", 3 * c), ("o", c), ("q2", c), ("kv2", 2 * c), ("o2", c)):
            self.np["w_" + name], self.np["b_" + name] = r.standard_normal((rows, c)) / math.sqrt(c), 0.05 * r.standard_normal(rows)
        for key in self.np:
            self.np[key] = G.stored(self.np[key], "f32" if key.startswith("b_") else dtype)
        self.np["rms"] = (1 + 0.1 * r.standard_normal(c)).astype(np.float32)
        self.lens = [tc - i for i in range(n)]
        ii = np.arange(self.t)
        self.pos = np.stack((ii // gw, ii % gw), -1)
        self.dims = (d // 2, d // 2)
        dt = G.TORCH[dtype]
        self.dev = {k: (G.dev_f32(v) if k.startswith("b_") or k == "rms" else dev(v, dtype)) for k, v in self.np.items()}
        self.packed = {name: G.pack(self.np["w_" + name][:, :, None, None], dtype) for name in ("qkv", "o", "q2", "kv2", "o2")}
        self.freq = torch.empty(d // 2, dtype=torch.float64, device="cuda")
        wmdec.rope_frequencies(self.dims, self.freq)
        self.posd, self.lensd = torch.from_numpy(self.pos.astype(np.int32)).cuda(), torch.tensor(self.lens, dtype=torch.int32, device="cuda")

        def buf(*s, t=dt):
            return torch.zeros(s, dtype=t, device="cuda")
        self.mod, self.y, self.x1, self.x2 = buf(n, 6 * c, t=torch.float32), buf(n, self.t, c), buf(n, self.t, c), buf(n, self.t, c)
        self.qkv, self.att, self.h, self.q2, self.kv2 = buf(n, self.t, 3, heads, d), buf(n, self.t, heads, d), buf(n, self.t, c), buf(n, self.t, heads, d), buf(n, tc, 2, heads, d)
        need = max(wmdec.cross_attention_workspace_bytes(self.qkv[:, :, 0], self.qkv[:, :, 1]), wmdec.cross_attention_workspace_bytes(self.q2, self.kv2[:, :, 0]))
        self.ws = torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda")

    def linear(self, x, name, y):
        tokens = x.shape[1]
        wmdec.gn_conv1x1(x.view(self.n, 1, tokens, -1), None, None, None, None, 1, False, self.packed[name], self.dev["b_" + name], None, y.view(self.n, 1, tokens, -1))

    def run(self):
        c, scale = self.c, 1 / math.sqrt(self.d)
        wmdec.adaln_fused_projection(self.dev["a"], self.dev["w_ada"], self.dev["b_ada"], self.mod)
        m = [self.mod[:, i * c:(i + 1) * c] for i in range(6)]
        layer, rms = wmdec.Norm("layer", 1e-6), wmdec.Norm("rms", 1e-6, self.dev["rms"])
        wmdec.residual_norm(self.dev["x"], None, None, None, 1.0, None, layer, m[1], m[0], self.y)
        self.linear(self.y, "qkv", self.qkv)
        q, k, v = (self.qkv[:, :, i] for i in range(3))
        wmdec.rope(q, k, self.posd, self.freq, self.dims, q, k, interleaved=True)
        wmdec.cross_attention(q, k, v, self.att, scale, workspace=self.ws)
        self.linear(self.att.view(self.n, self.t, c), "o", self.h)
        wmdec.residual_norm(self.dev["x"], self.h, None, m[2], 1.0, self.x1, layer, m[4], m[3], self.y)
        self.linear(self.y, "q2", self.q2)
        self.linear(self.dev["cond"], "kv2", self.kv2)
        wmdec.cross_attention(self.q2, self.kv2[:, :, 0], self.kv2[:, :, 1], self.att, scale, key_lens=self.lensd, workspace=self.ws)
        self.linear(self.att.view(self.n, self.t, c), "o2", self.h)
        wmdec.residual_norm(self.x1, self.h, rms, m[5], 0.5, self.x2, None, None, None, None)
        return self.x2

    def want(self):
        p, c, n = {k: v.astype(np.float64) for k, v in self.np.items()}, self.c, self.n
        mod = ref.silu(p["a"]) @ p["w_ada"].T + p["b_ada"]
        m = [mod[:, i * c:(i + 1) * c] for i in range(6)]
        scale = 1 / math.sqrt(self.d)

        def lin(x, name, *shape):
            return (x @ p["w_" + name].T + p["b_" + name]).reshape(shape)
        qkv = lin(ref.norm_modulate(p["x"], ("layer", 1e-6), m[1], m[0]), "qkv", n, self.t, 3, self.heads, self.d)
        pos = np.broadcast_to(self.pos, (n,) + self.pos.shape)
        f = ref.rope_frequencies(self.dims)
        q, k = (ref.rope(qkv[:, :, i], pos, f, self.dims, True) for i in range(2))
        h = lin(ref.cross_attention(q, k, qkv[:, :, 2], scale)[0].reshape(n, self.t, c), "o", n, self.t, c)
        x1 = ref.gated_residual(p["x"], h, (), m[2])
        q2 = lin(ref.norm_modulate(x1, ("layer", 1e-6), m[4], m[3]), "q2", n, self.t, self.heads, self.d)
        kv2 = lin(p["cond"], "kv2", n, self.tc, 2, self.heads, self.d)
        h = lin(ref.cross_attention(q2, kv2[:, :, 0], kv2[:, :, 1], scale, self.lens)[0].reshape(n, self.t, c), "o2", n, self.t, c)
        return ref.gated_residual(x1, h, ("rms", 1e-6, p["rms"]), m[5], 0.5)


@pytest.mark.parametrize("dtype, n, gh, gw, tc, heads, d", [("bf16", 2, 9, 15, 21, 6, 64), ("f16", 1, 6, 7, 77, 4, 128), ("f16", 3, 1, 1, 5, 2, 64)])
def test_transformer_block(dtype, n, gh, gw, tc, heads, d):
    """Some twenty roundings to 16 bits in a row: the bar of a whole layer, max|err| / rms <= 2e-2, that the decoder's operators have."""
    b = Block(n, gh, gw, tc, heads, d, dtype, 1)
    err = ref.rel_err(host(b.run()), b.want())
    assert err <= G.TOL[dtype], err


def test_transformer_block_captured_and_replayed():
    """A captured block replays to the eager bits, with eager work on the same workspace and other inputs in between; two graphs share it."""
    blocks = [Block(2, 5, 13, 2100, 4, 64, "bf16", s) for s in (2, 3)]
    blocks[1].ws = blocks[0].ws
    side = torch.cuda.Stream()
    eager = [b.run().clone() for b in blocks]
    torch.cuda.synchronize()
    graphs = []
    for b in blocks:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            b.run()
        graphs.append(g)
    first = blocks[0].dev["x"].clone()
    for i in range(4):
        for j, g in enumerate(graphs):
            blocks[j].x2.zero_()
            blocks[j].ws.fill_(0xFF)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(blocks[j].x2, eager[j]), (i, j)
        blocks[0].dev["x"].mul_(-0.5)
        graphs[0].replay()
        got = blocks[0].x2.clone()
        assert torch.equal(got, blocks[0].run()) and not torch.equal(got, eager[0])
        blocks[0].dev["x"].copy_(first)


def test_calls_follow_the_current_stream():
    """Work on a side stream while its inputs are still being made there; two streams with workspaces of their own."""
    side = [torch.cuda.Stream() for _ in range(2)]
    blocks = [Block(1, 8, 16, 300, 4, 64, "f16", 4 + i) for i in range(2)]
    torch.cuda.synchronize()
    want = [b.run().clone() for b in blocks]
    torch.cuda.synchronize()
    keep = [b.dev["x"].clone() for b in blocks]
    torch.cuda.synchronize()
    for _ in range(3):
        for b, s, x in zip(blocks, side, keep):
            with torch.cuda.stream(s):
                b.dev["x"].fill_(float("nan"))
                b.dev["x"].copy_(x)
                b.run()
        torch.cuda.synchronize()
        assert all(torch.equal(b.x2, w) for b, w in zip(blocks, want))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_cross_scores_half_a_step_beside_the_reference(dtype):
    """From 2^27 on fp32 holds scores in steps of 16, and a reference and eight more may be the next score: that one's probability is 2^16 unless the reference moves,
    which f16 does not hold.  Two keys alone have weight, with values of 1 and 2: an output lies between them."""
    for tq in (1, 40, 140):
        for low, high in ((8, 24), (16, 24), (32, 48)):
            q, k, v = (torch.zeros((1, t, 2, 64), dtype=G.TORCH[dtype], device="cuda") for t in (tq, 600, 600))
            q[..., 0], q[..., 32] = 22720.0, 1.0
            k[0, 5, :, 0] = k[0, 517, :, 0] = 4096.0
            k[0, 5, :, 32], k[0, 517, :, 32] = low, high
            v[:], v[0, 517] = 1.0, 2.0
            o = torch.empty_like(q)
            ws = torch.empty(max(16, wmdec.cross_attention_workspace_bytes(q, k)), dtype=torch.uint8, device="cuda")
            wmdec.cross_attention(q, k, v, o, 1.0, workspace=ws)
            assert bool(((o >= 1.0) & (o <= 2.0)).all()), (tq, low, high, o.flatten()[:4].tolist())
