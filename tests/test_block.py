"""The operators around the AdaLN projections of a transformer block: their oracle against brute force and identities, and what
the library and its binding refuse (no GPU needed)."""
import ctypes
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from oracle import ref
from paper_2602_00608_amd import asm_check, bench_ops, wmdec


# ------------------------------------------------------------------ oracle
def test_norm_oracle():
    r = np.random.default_rng(1)
    x, h = r.standard_normal((2, 3, 5)), r.standard_normal((2, 3, 5)) + 3.0
    w, u, g, c, b = r.standard_normal(5), r.standard_normal(5), r.standard_normal((2, 5)), r.standard_normal((2, 5)), r.standard_normal((2, 5))
    got = ref.gated_residual(x, h, ("layer", 1e-3, w, u), g, 0.5)
    y = ref.norm_modulate(x, ("rms", 1e-3, w, None), c, b)
    for n in range(2):
        for t in range(3):
            mean = sum(h[n, t]) / 5
            var = sum((v - mean) ** 2 for v in h[n, t]) / 5
            ms = sum(v * v for v in x[n, t]) / 5
            for i in range(5):
                assert abs(got[n, t, i] - (x[n, t, i] + 0.5 * g[n, i] * ((h[n, t, i] - mean) / math.sqrt(var + 1e-3) * w[i] + u[i]))) < 1e-12
                assert abs(y[n, t, i] - (x[n, t, i] / math.sqrt(ms + 1e-3) * w[i] * (1 + c[n, i]) + b[n, i])) < 1e-12
    z = ref.row_norm(h, "layer", 0.0)
    assert np.allclose(z.mean(-1), 0, atol=1e-14) and np.allclose((z * z).mean(-1), 1)
    assert np.array_equal(ref.gated_residual(x, h), x + h) and np.array_equal(ref.norm_modulate(x), x)


def test_rope_oracle():
    r = np.random.default_rng(2)
    x = r.standard_normal((1, 4, 2, 12))
    dims = (4, 6)
    f = ref.rope_frequencies(dims)
    assert np.allclose(f, [1, 1e-2, 1, 10000 ** (-1 / 3), 10000 ** (-2 / 3)])
    pos = r.integers(-50, 50, (1, 4, 2))
    for inter in (False, True):
        y = ref.rope(x, pos, f, dims, inter)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 10:], x[..., 10:])
        assert np.allclose(ref.rope(y, pos, f, dims, inter, inverse=True), x)
        # scores depend on differences of positions alone
        k = ref.rope(x[:, :1], pos[:, :1] + 7, f, dims, inter)
        k0, q0 = ref.rope(x[:, :1], pos[:, :1], f, dims, inter), ref.rope(x[:, 1:2], pos[:, 1:2], f, dims, inter)
        q = ref.rope(x[:, 1:2], pos[:, 1:2] + 7, f, dims, inter)
        assert np.allclose((q * k).sum(-1), (q0 * k0).sum(-1))
    a = ref.rope(x, pos, f, dims, True)
    c = x[0, 1, 0, 4] * math.cos(pos[0, 1, 1]) - x[0, 1, 0, 5] * math.sin(pos[0, 1, 1])      # first pair of the second axis: frequency 1
    assert abs(a[0, 1, 0, 4] - c) < 1e-12
    plain = ref.rope_frequencies((64,))
    assert np.allclose(ref.rope_frequencies((64,), scaling="linear", factor=4.0), plain / 4)
    scaled = ref.rope_frequencies((64,), scaling="base", factor=4.0)
    assert scaled[0] == 1 and abs(scaled[-1] * 4 - plain[-1]) < 1e-9        # the lowest frequency is stretched by the factor, the highest not at all
    ramp = ref.rope_frequencies((64,), scaling="ramp", factor=4.0, trained_length=2048, low_turns=1, high_turns=4)
    turns = 2048 * plain / (2 * math.pi)
    assert np.array_equal(ramp[turns >= 4], plain[turns >= 4]) and np.allclose(ramp[turns <= 1], plain[turns <= 1] / 4)


def test_cross_attention_oracle():
    r = np.random.default_rng(3)
    q, k, v = r.standard_normal((2, 3, 4, 5)), r.standard_normal((2, 6, 2, 5)), r.standard_normal((2, 6, 2, 5))
    mask = np.array([[1, 1, 0, 1, 1, 1], [0, 0, 1, 1, 1, 1]], dtype=bool)
    o, a = ref.cross_attention(q, k, v, 0.3, [4, 2], mask)
    assert not o[1].any() and not a[1].any()
    for t in range(3):
        for h in range(4):
            e = {j: math.exp(0.3 * sum(q[0, t, h, c] * k[0, j, h // 2, c] for c in range(5))) for j in (0, 1, 3)}
            for c in range(5):
                assert abs(o[0, t, h, c] - sum(e[j] * v[0, j, h // 2, c] for j in e) / sum(e.values())) < 1e-12
    assert np.allclose(ref.cross_attention(q, k, v, 1e-12)[0], np.repeat(v.mean(1), 2, 1)[:, None])
    assert (np.abs(ref.cross_attention(q, k, v, 1.0)[0]) <= ref.cross_attention(q, k, v, 1.0)[1] + 1e-15).all()


# ------------------------------------------------------------------ refusals of the C entry points
P = 0x10000
NORM = dict(x=P, x_dtype=1, h=2 * P, act_dtype=1, post=None, gate=3 * P, res_scale=1.0, x_out=4 * P, pre=None, scale=5 * P, shift=6 * P, mod_stride=192, y=7 * P,
            n=2, t=3, d=64, stream=None)


def _norm(**changes):
    return wmdec.lib().wmdec_residual_norm(*dict(NORM, **changes).values())


@pytest.mark.parametrize("status, changes", [
    (wmdec.ERR_INVALID_ARG, dict(x=None)), (wmdec.ERR_INVALID_ARG, dict(x_out=None)), (wmdec.ERR_INVALID_ARG, dict(x_dtype=3)),
    (wmdec.ERR_INVALID_ARG, dict(h=None)), (wmdec.ERR_INVALID_ARG, dict(h=None, x_out=None)), (wmdec.ERR_INVALID_ARG, dict(y=None)),
    (wmdec.ERR_INVALID_ARG, dict(h=None, x_out=None, gate=None, post=wmdec._CNorm(1, 1e-6, None, None))),
    (wmdec.ERR_INVALID_ARG, dict(y=None, scale=None, shift=None, pre=wmdec._CNorm(2, 1e-6, None, None))),
    (wmdec.ERR_INVALID_ARG, dict(h=None, x_out=None, gate=None, y=None, scale=None, shift=None)),
    (wmdec.ERR_UNSUPPORTED, dict(x_dtype=1, act_dtype=2)), (wmdec.ERR_UNSUPPORTED, dict(x_dtype=1, act_dtype=0)), (wmdec.ERR_UNSUPPORTED, dict(d=16385, mod_stride=0)),
    (wmdec.ERR_UNSUPPORTED, dict(n=65536, t=65536)),
    (wmdec.ERR_INVALID_ARG, dict(n=0)), (wmdec.ERR_INVALID_ARG, dict(t=-1)), (wmdec.ERR_INVALID_ARG, dict(d=0)), (wmdec.ERR_SHAPE, dict(mod_stride=63)),
    (wmdec.ERR_SHAPE, dict(mod_stride=-64)), (wmdec.ERR_INVALID_ARG, dict(res_scale=math.nan)), (wmdec.ERR_INVALID_ARG, dict(res_scale=math.inf)),
    (wmdec.ERR_INVALID_ARG, dict(x=P + 1)), (wmdec.ERR_INVALID_ARG, dict(gate=3 * P + 2)),
    (wmdec.ERR_INVALID_ARG, dict(x_out=2 * P)), (wmdec.ERR_INVALID_ARG, dict(y=4 * P)), (wmdec.ERR_INVALID_ARG, dict(y=P)), (wmdec.ERR_INVALID_ARG, dict(h=P)),
    (wmdec.ERR_INVALID_ARG, dict(h=None, x_out=None, gate=None, x_dtype=0, y=P)),
    (wmdec.ERR_INVALID_ARG, dict(pre=wmdec._CNorm(3, 1e-6, None, None))), (wmdec.ERR_INVALID_ARG, dict(pre=wmdec._CNorm(0, 0, P, None))),
    (wmdec.ERR_INVALID_ARG, dict(post=wmdec._CNorm(1, -1e-6, None, None))), (wmdec.ERR_INVALID_ARG, dict(post=wmdec._CNorm(1, math.nan, None, None))),
    (wmdec.ERR_INVALID_ARG, dict(post=wmdec._CNorm(1, 1e-6, P + 2, None))),
])
def test_residual_norm_refuses(status, changes):
    assert _norm(**changes) == status and "residual_norm" in wmdec.last_error()


S = wmdec._CStrides
ROPE = dict(q=P, qs=S(768, 256, 64), qo=2 * P, qos=S(768, 256, 64), hq=4, k=3 * P, ks=S(384, 128, 64), ko=4 * P, kos=S(384, 128, 64), hk=2, dtype=1, positions=5 * P,
            positions_stride=0, freq=6 * P, layout=wmdec._CRopeLayout(1, (ctypes.c_int * 3)(64, 0, 0), 0, 0, 1.0), n=1, t=3, d=64, stream=None)


def _layout(axes=1, dims=(64, 0, 0), magnitude=1.0):
    return wmdec._CRopeLayout(axes, (ctypes.c_int * 3)(*dims), 0, 0, magnitude)


@pytest.mark.parametrize("status, changes", [
    (wmdec.ERR_INVALID_ARG, dict(q=None)), (wmdec.ERR_INVALID_ARG, dict(qo=None)), (wmdec.ERR_INVALID_ARG, dict(qs=None)), (wmdec.ERR_INVALID_ARG, dict(ko=None)),
    (wmdec.ERR_INVALID_ARG, dict(positions=None)), (wmdec.ERR_INVALID_ARG, dict(freq=None)), (wmdec.ERR_INVALID_ARG, dict(freq=6 * P + 4)),
    (wmdec.ERR_INVALID_ARG, dict(dtype=5)), (wmdec.ERR_INVALID_ARG, dict(hq=0)), (wmdec.ERR_INVALID_ARG, dict(hk=-1)), (wmdec.ERR_INVALID_ARG, dict(n=0)),
    (wmdec.ERR_INVALID_ARG, dict(layout=_layout(0))), (wmdec.ERR_INVALID_ARG, dict(layout=_layout(4))), (wmdec.ERR_SHAPE, dict(layout=_layout(1, (63, 0, 0)))),
    (wmdec.ERR_SHAPE, dict(layout=_layout(2, (32, 0, 0)))), (wmdec.ERR_SHAPE, dict(layout=_layout(2, (32, 34, 0)))), (wmdec.ERR_INVALID_ARG, dict(layout=_layout(magnitude=math.inf))),
    (wmdec.ERR_UNSUPPORTED, dict(layout=_layout(1, (4098, 0, 0)), d=8192)), (wmdec.ERR_UNSUPPORTED, dict(d=16385)), (wmdec.ERR_UNSUPPORTED, dict(hq=16384)),
    (wmdec.ERR_INVALID_ARG, dict(qs=S(0, -256, 64))), (wmdec.ERR_INVALID_ARG, dict(qs=S(0, 1 << 60, 64))),
    (wmdec.ERR_INVALID_ARG, dict(qo=P, qos=S(0, 512, 64))), (wmdec.ERR_INVALID_ARG, dict(qo=4 * P)), (wmdec.ERR_INVALID_ARG, dict(qo=3 * P)), (wmdec.ERR_INVALID_ARG, dict(ko=P)),
    (wmdec.ERR_INVALID_ARG, dict(qos=S(0, 256, 0))), (wmdec.ERR_INVALID_ARG, dict(kos=S(0, 0, 64))),
    (wmdec.ERR_INVALID_ARG, dict(q=P + 1)), (wmdec.ERR_SHAPE, dict(n=2, positions_stride=2)), (wmdec.ERR_UNSUPPORTED, dict(n=65536, t=65536)),
])
def test_rope_refuses(status, changes):
    assert wmdec.lib().wmdec_rope(*dict(ROPE, **changes).values()) == status and "rope" in wmdec.last_error()


@pytest.mark.parametrize("status, dims, scaling", [
    (wmdec.ERR_INVALID_ARG, (), (0, 1e4)), (wmdec.ERR_SHAPE, (64, 3), (0, 1e4)), (wmdec.ERR_INVALID_ARG, (64,), (4, 1e4)), (wmdec.ERR_INVALID_ARG, (64,), (0, 1.0)),
    (wmdec.ERR_INVALID_ARG, (64,), (0, math.inf)), (wmdec.ERR_INVALID_ARG, (64,), (1, 1e4, 0.5)), (wmdec.ERR_SHAPE, (64, 2), (2, 1e4, 2.0)),
    (wmdec.ERR_INVALID_ARG, (64,), (3, 1e4, 2.0, 2048.0, 4.0, 4.0)), (wmdec.ERR_INVALID_ARG, (64,), (3, 1e4, 2.0, 0.0, 1.0, 4.0)),
])
def test_rope_frequencies_refuses(status, dims, scaling):
    dims = (ctypes.c_int * max(len(dims), 1))(*dims) if dims else None
    n = len(dims) if dims else 1
    assert wmdec.lib().wmdec_rope_frequencies(P, n, dims, ctypes.byref(wmdec._CRopeScaling(*scaling)), None) == status
    assert wmdec.lib().wmdec_rope_frequencies(P + 4, 1, (ctypes.c_int * 1)(64), ctypes.byref(wmdec._CRopeScaling(0, 1e4)), None) == wmdec.ERR_INVALID_ARG


CROSS = dict(q=P, qs=S(768, 256, 64), k=2 * P, ks=S(2560, 128, 64), v=3 * P, vs=S(2560, 128, 64), o=4 * P, os=S(768, 256, 64), dtype=1, scale=0.1, lens=None, mask=None,
             n=2, tq=3, tk=20, hq=4, hk=2, d=64, ws=5 * P, bytes=1 << 40, stream=None)


@pytest.mark.parametrize("status, changes", [
    (wmdec.ERR_INVALID_ARG, dict(q=None)), (wmdec.ERR_INVALID_ARG, dict(k=None)), (wmdec.ERR_INVALID_ARG, dict(v=None)), (wmdec.ERR_INVALID_ARG, dict(o=None)),
    (wmdec.ERR_INVALID_ARG, dict(os=None)), (wmdec.ERR_INVALID_ARG, dict(dtype=-1)), (wmdec.ERR_INVALID_ARG, dict(tq=0)), (wmdec.ERR_INVALID_ARG, dict(tk=-1)),
    (wmdec.ERR_SHAPE, dict(hq=5)), (wmdec.ERR_UNSUPPORTED, dict(d=60)), (wmdec.ERR_UNSUPPORTED, dict(d=264)), (wmdec.ERR_UNSUPPORTED, dict(dtype=0, d=66)),
    (wmdec.ERR_INVALID_ARG, dict(k=2 * P + 8)), (wmdec.ERR_INVALID_ARG, dict(ks=S(2560, 132, 64))), (wmdec.ERR_INVALID_ARG, dict(vs=S(2560, 128, 60))),
    (wmdec.ERR_INVALID_ARG, dict(qs=S(-768, 256, 64))), (wmdec.ERR_UNSUPPORTED, dict(ks=S(0, 1 << 23, 64))),
    (wmdec.ERR_INVALID_ARG, dict(scale=0.0)), (wmdec.ERR_INVALID_ARG, dict(scale=-1.0)), (wmdec.ERR_INVALID_ARG, dict(scale=math.inf)), (wmdec.ERR_INVALID_ARG, dict(scale=math.nan)),
    (wmdec.ERR_INVALID_ARG, dict(o=P)), (wmdec.ERR_INVALID_ARG, dict(o=3 * P)), (wmdec.ERR_INVALID_ARG, dict(os=S(768, 0, 64))), (wmdec.ERR_INVALID_ARG, dict(os=S(0, 256, 64))), (wmdec.ERR_INVALID_ARG, dict(lens=6 * P + 2)), (wmdec.ERR_UNSUPPORTED, dict(tk=(1 << 31) - 1)),
    (wmdec.ERR_UNSUPPORTED, dict(n=1 << 20, tq=1 << 20)),
])
def test_cross_attention_refuses(status, changes):
    assert wmdec.lib().wmdec_cross_attention(*dict(CROSS, **changes).values()) == status and "cross_attention" in wmdec.last_error()


def test_launches_of_too_many_threads_are_refused():
    """A launch has less than 2^32 threads: samples with vectors of their own, tokens with a workgroup each, rows, and rows whose ranges of keys are joined."""
    assert _norm(n=(1 << 22) + 1, t=1) == wmdec.ERR_UNSUPPORTED
    layout = wmdec._CRopeLayout(1, (ctypes.c_int * 3)(4096, 0, 0), 0, 0, 1.0)
    wide = S(0, 3 * 4096, 4096)
    assert wmdec.lib().wmdec_rope(*dict(ROPE, layout=layout, d=4096, t=1 << 24, hq=2, hk=1, qs=wide, qos=wide, ks=wide, kos=wide).values()) == wmdec.ERR_UNSUPPORTED
    for changes in (dict(n=1 << 23, tq=1, tk=20), dict(n=1 << 21, tq=1, tk=1 << 20, hq=1, hk=1), dict(n=1 << 20, tq=33, tk=4096, hq=1, hk=1)):
        assert wmdec.lib().wmdec_cross_attention(*dict(CROSS, **changes).values()) == wmdec.ERR_UNSUPPORTED, changes


def test_cross_attention_workspace_is_asked_for():
    size = wmdec.lib().wmdec_cross_attention_workspace_bytes
    need = size(wmdec.BF16, 1, 1, 32768, 32, 8, 128)
    assert need > 0
    big = dict(CROSS, n=1, tq=1, tk=32768, hq=32, hk=8, d=128, ks=S(0, 1024, 128), vs=S(0, 1024, 128), qs=S(0, 0, 128), os=S(0, 0, 128))
    for ws, have in ((None, 1 << 40), (5 * P, need - 1), (5 * P + 8, 1 << 40)):
        assert wmdec.lib().wmdec_cross_attention(*dict(big, ws=ws, bytes=have).values()) == wmdec.ERR_WORKSPACE
    assert size(wmdec.BF16, 7, 1, 32768, 32, 8, 128) == 7 * need and size(wmdec.BF16, 1, 5400, 512, 30, 30, 64) == 0
    for bad in ((7, 1, 1, 5, 4, 2, 64), (1, 1, 1, -1, 4, 2, 64), (1, 0, 1, 5, 4, 2, 64), (1, 1, 1, 5, 4, 3, 64), (1, 1, 1, 5, 4, 2, 512)):
        assert size(*bad) == 0


def test_cross_attention_refuses_a_scale_that_the_kernel_cannot_hold():
    """The kernel multiplies it by log2(e): from 2.36e38 on that is infinite, and a score of zero not a number."""
    for scale in (2.1e38, 2.4e38, 3.4e38, math.inf, math.nan, 0.0, -1e-30):
        assert wmdec.lib().wmdec_cross_attention(*dict(CROSS, scale=scale).values()) == wmdec.ERR_INVALID_ARG, scale
    assert wmdec.lib().wmdec_cross_attention(*dict(CROSS, scale=1.9e38, q=None).values()) == wmdec.ERR_INVALID_ARG and "null" in wmdec.last_error()


def test_cross_attention_workspace_of_what_is_refused_is_nothing():
    """Rows past 31 bits, keys past them, launches past 2^32 threads and widths that are no multiple of 16 bytes.  (In a process of its own: the size of 2^30 tokens of four
    heads once ended it by a division by zero.)"""
    cases = [(wmdec.BF16, 1, 1 << 30, 5000, 4, 1, 64), (wmdec.BF16, 1, 1 << 29, 5000, 4, 1, 64), (wmdec.F32, 2, (1 << 31) - 1, 5000, 64, 2, 128), (wmdec.F16, 1, 3, (1 << 31) - 1, 4, 2, 64),
             (wmdec.F16, 1 << 23, 1, 20, 4, 2, 64), (wmdec.BF16, 1 << 21, 1, 1 << 20, 1, 1, 64), (wmdec.BF16, 1, 1, 32768, 4, 2, 60), (wmdec.F32, 1, 1, 32768, 4, 2, 66)]
    code = "from paper_2602_00608_amd import wmdec; print([wmdec.lib().wmdec_cross_attention_workspace_bytes(*c) for c in %r])" % (cases,)
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert out.returncode == 0 and out.stdout.strip() == str([0] * len(cases)), (out.returncode, out.stdout, out.stderr[-500:])
    for c in cases:
        dtype, n, tq, tk, hq, hk, d = c
        assert wmdec.lib().wmdec_cross_attention(*dict(CROSS, dtype=dtype, n=n, tq=tq, tk=tk, hq=hq, hk=hk, d=d).values()) == wmdec.ERR_UNSUPPORTED, c
    assert wmdec.lib().wmdec_cross_attention_workspace_bytes(wmdec.F32, 1, 1, 32768, 4, 2, 60) > 0


# ------------------------------------------------------------------ refusals of the binding
def fake(*shape, dtype=torch.bfloat16, device="cuda:0"):
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device=device)


@pytest.fixture(autouse=True)
def current_device(monkeypatch):
    """Without a GPU the current device and its stream cannot be asked for; nothing here gets as far as a launch."""
    if not torch.cuda.is_available():
        monkeypatch.setattr(wmdec, "_device", lambda: 0)
        monkeypatch.setattr(wmdec, "_stream", lambda: 0)


def _call_norm(x=None, h=None, x_out=None, y=None, gate=None, scale=None, shift=None, pre=None):
    x = fake(2, 3, 8) if x is None else x
    wmdec.residual_norm(x, h, None, gate, 1.0, x_out, pre, scale, shift, fake(2, 3, 8) if y is None else y)


@pytest.mark.parametrize("call, error", [
    (lambda: _call_norm(x=torch.zeros(2, 3, 8)), AssertionError),                          # on the host
    (lambda: _call_norm(x=fake(2, 3, 8, device="cuda:1")), AssertionError),                # another device than the current one
    (lambda: _call_norm(y=fake(2, 3, 8, device="cuda:1")), AssertionError),
    (lambda: _call_norm(x=fake(2, 8)), ValueError), (lambda: _call_norm(y=fake(2, 4, 8)), ValueError), (lambda: _call_norm(x=fake(2, 8, 3).transpose(1, 2)), ValueError),
    (lambda: _call_norm(x=fake(2, 6, 8)[:, ::2]), AssertionError),                         # rows are dense
    (lambda: _call_norm(h=fake(2, 3, 8), x_out=fake(2, 3, 8, dtype=torch.float32)), ValueError),
    (lambda: _call_norm(h=fake(2, 3, 8, dtype=torch.float16), x_out=fake(2, 3, 8)), ValueError),
    (lambda: _call_norm(x=fake(2, 3, 8, dtype=torch.int32)), KeyError), (lambda: _call_norm(x=3), TypeError),
    (lambda: _call_norm(scale=fake(2, 8)), ValueError), (lambda: _call_norm(scale=fake(1, 8, dtype=torch.float32)), ValueError),
    (lambda: _call_norm(scale=fake(2, 24, dtype=torch.float32)[:, :8], shift=fake(2, 8, dtype=torch.float32)), ValueError),   # two strides
    (lambda: _call_norm(pre=wmdec.Norm("rms", 1e-6, fake(7, dtype=torch.float32))), ValueError), (lambda: _call_norm(pre=wmdec.Norm("batch")), KeyError),
    (lambda: _call_norm(pre=wmdec.Norm("rms", None)), TypeError),
])
def test_residual_norm_binding_refuses(call, error):
    with pytest.raises(error):
        call()


def _call_rope(q=None, k=None, positions=None, freq=None, dims=(8,), q_out=None, k_out=None, **more):
    wmdec.rope(fake(2, 3, 4, 8) if q is None else q, k, fake(2, 3, 1, dtype=torch.int32) if positions is None else positions,
               fake(4, dtype=torch.float64) if freq is None else freq, dims, fake(2, 3, 4, 8) if q_out is None else q_out, k_out, **more)


@pytest.mark.parametrize("call, error", [
    (lambda: _call_rope(q=fake(2, 3, 32)), ValueError), (lambda: _call_rope(q_out=fake(2, 3, 4, 16)), ValueError), (lambda: _call_rope(k=fake(2, 3, 2, 8)), TypeError),
    (lambda: _call_rope(k_out=fake(2, 3, 2, 8)), ValueError), (lambda: _call_rope(k=fake(2, 4, 2, 8), k_out=fake(2, 4, 2, 8)), ValueError),
    (lambda: _call_rope(k=fake(2, 3, 2, 8, dtype=torch.float16), k_out=fake(2, 3, 2, 8, dtype=torch.float16)), ValueError),
    (lambda: _call_rope(positions=fake(2, 3, 1, dtype=torch.int64)), ValueError), (lambda: _call_rope(positions=fake(2, 3, 2, dtype=torch.int32)), ValueError),
    (lambda: _call_rope(positions=fake(1, 3, 1, dtype=torch.int32)), ValueError), (lambda: _call_rope(positions=fake(3, dtype=torch.int32)), ValueError),
    (lambda: _call_rope(freq=fake(4, dtype=torch.float32)), ValueError), (lambda: _call_rope(freq=fake(3, dtype=torch.float64)), ValueError),
    (lambda: _call_rope(dims=()), ValueError), (lambda: _call_rope(dims=(2, 2, 2, 2)), ValueError), (lambda: _call_rope(dims=(8, 1)), ValueError),
    (lambda: _call_rope(q=fake(2, 3, 8, 4).transpose(2, 3)), ValueError), (lambda: _call_rope(q=fake(2, 3, 4, 8, device="cuda:1")), AssertionError),
    (lambda: _call_rope(magnitude="x"), TypeError),
    (lambda: wmdec.rope_frequencies((8,), fake(4, dtype=torch.float32)), ValueError), (lambda: wmdec.rope_frequencies((8,), fake(4, dtype=torch.float64), scaling="other"), KeyError),
    (lambda: wmdec.rope_frequencies((8,), fake(4, dtype=torch.float64, device="cuda:1")), AssertionError),
])
def test_rope_binding_refuses(call, error):
    with pytest.raises(error):
        call()


def _call_cross(q=None, k=None, v=None, o=None, **more):
    wmdec.cross_attention(fake(2, 3, 4, 8) if q is None else q, fake(2, 5, 2, 8) if k is None else k, fake(2, 5, 2, 8) if v is None else v,
                          fake(2, 3, 4, 8) if o is None else o, 1.0, **more)


@pytest.mark.parametrize("call, error", [
    (lambda: _call_cross(q=fake(2, 3, 32)), ValueError), (lambda: _call_cross(k=fake(2, 5, 2, 16)), ValueError), (lambda: _call_cross(v=fake(2, 6, 2, 8)), ValueError),
    (lambda: _call_cross(o=fake(2, 3, 2, 8)), ValueError), (lambda: _call_cross(k=fake(1, 5, 2, 8), v=fake(1, 5, 2, 8)), ValueError),
    (lambda: _call_cross(v=fake(2, 5, 2, 8, dtype=torch.float16)), ValueError), (lambda: _call_cross(key_lens=fake(2, dtype=torch.int64)), ValueError),
    (lambda: _call_cross(key_lens=fake(3, dtype=torch.int32)), ValueError), (lambda: _call_cross(key_mask=fake(2, 4, dtype=torch.bool)), ValueError),
    (lambda: _call_cross(key_mask=fake(2, 5, dtype=torch.float32)), ValueError), (lambda: _call_cross(key_mask=fake(2, 10, dtype=torch.bool)[:, ::2]), ValueError),
    (lambda: _call_cross(k=fake(2, 5, 2, 8, device="cuda:1")), AssertionError), (lambda: _call_cross(k=fake(2, 5, 8, 2).transpose(2, 3)), ValueError),
    (lambda: _call_cross(workspace=fake(4, 4, dtype=torch.uint8)), ValueError), (lambda: _call_cross(q=torch.zeros(2, 3, 4, 8)), AssertionError),
    (lambda: wmdec._ops().cross_attention(1, 2), TypeError), (lambda: wmdec._ops().bind_block(1), TypeError),
])
def test_cross_attention_binding_refuses(call, error):
    with pytest.raises(error):
        call()


# ------------------------------------------------------------------ compiled code
def test_other_uses_of_m0_are_found():
    load = ["s_add_u32 m0, s4, 0x400", "s_nop 0", "buffer_load_dwordx4 v2, s[8:11], s3 offen lds"]
    assert asm_check.check_m0(load) == []
    assert len(asm_check.check_m0(load + ["s_mov_b32 m0, s5"])) == 1 and len(asm_check.check_m0(load + ["v_readlane_b32 s3, v2, m0"])) == 1
    text = "\n".join(["_Z6kernel:"] + ["\t" + l for l in load + ["s_mov_b32 m0, -1", "s_endpgm"]] + [".Lfunc_end0:"])
    assert len(asm_check.check_source(text, m0="kernel")) == 1 and asm_check.check_source(text, m0="other") == []


# ------------------------------------------------------------------ timing
def test_a_cold_time_within_the_spread_of_what_is_subtracted_is_no_reading():
    alone = [450.0, 447.0, 452.0, 455.0, 449.0, 451.0, 446.0, 453.0]
    assert bench_ops.difference(alone, [v - 1.0 for v in alone]) is None and bench_ops.difference(alone, [v + 3.0 for v in alone]) is None
    assert bench_ops.difference(alone, [v + 40.0 for v in alone]) == 40.0
    assert bench_ops.figures(None, 1e9, "GB/s", 8000.0).split() == ["-", "us", "-", "GB/s", "(", "-)"]
    assert bench_ops.figures(100.0, 4e8, "GB/s", 8000.0).split() == ["100.0", "us", "4000.0", "GB/s", "(50.0%)"]
