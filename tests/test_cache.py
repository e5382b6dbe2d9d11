"""The cache of keys and values in four bits: its oracle against brute force, and what the library and its binding refuse (no GPU needed)."""
import math

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from oracle import ref
from paper_2602_00608_amd import wmdec


# ------------------------------------------------------------------ oracle
def test_held_oracle():
    """Block by block and value by value: no other of the sixteen values is nearer, and of two that are as near the one at the even place is taken."""
    r = np.random.default_rng(4)
    x = (r.standard_normal((7, 72)) * np.exp2(r.integers(-20, 20, (7, 1)))).astype(np.float32)
    x[0, :8] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]
    x[0, 8:32] = 0
    held = ref.cache_held(x, "f32")
    for row in range(7):
        for at in (0, 32, 64):
            part, got = x[row, at:at + 32].astype(float), held[row, at:at + 32]
            m = max(abs(v) for v in part)
            e = math.floor(math.log2(m)) - 2
            if m / 2.0 ** (e + 2) >= 1.75:
                e += 1
            values = [v * 2.0 ** e for v in (0, 0.5, 1, 1.5, 2, 3, 4, 6)]
            for v, g in zip(part, got):
                far = [abs(abs(v) - w) for w in values]
                best = [i for i in range(8) if far[i] == min(far)]
                assert abs(g) == values[next((i for i in best if i % 2 == 0), best[0])] and (g == 0 or (g > 0) == (v > 0))
    assert held[0, :8].tolist() == [4, 0, 1, 1, 2, 2, 4, 4]
    assert np.array_equal(ref.cache_held(held, "f32"), held)
    assert not ref.cache_held(np.zeros((2, 40)), "bf16").any()


def test_held_oracle_at_the_ends_of_the_types():
    big = np.zeros((1, 32), np.float32)
    big[0, :3] = [3.4028234e38, -3.4e38, 1e38]
    assert np.isfinite(ref.cache_held(big, "f32")).all() and ref.cache_held(big, "f32")[0, 0] == 6 * 2.0 ** 125
    half = np.zeros((1, 32), np.float32)
    half[0, :4] = [65504, -40000, 56000, 24576]
    assert ref.cache_held(half, "f16")[0, :4].tolist() == [49152, -32768, 49152, 24576] and ref.cache_held(half, "f32")[0, 0] == 65536
    tiny = np.zeros((1, 32), np.float32)
    tiny[0, :3] = [2.0 ** -126, -2.0 ** -128, 2.0 ** -130]
    assert ref.cache_held(tiny, "f32")[0, :3].tolist() == [2.0 ** -126, 0, 0]
    x = np.ones((2, 72), np.float32)
    x[0, 5], x[1, 70] = np.nan, np.inf
    held = ref.cache_held(x, "bf16")
    assert np.isnan(held[0, :32]).all() and np.isfinite(held[0, 32:]).all() and np.isnan(held[1, 64:]).all() and np.isfinite(held[1, :64]).all()


def test_seen_attention_oracle():
    r = np.random.default_rng(5)
    q, k, v = r.standard_normal((2, 6, 4, 8)), r.standard_normal((2, 9, 2, 8)), r.standard_normal((2, 9, 2, 8))
    mask = r.random((2, 9)) < 0.6
    mask[1] = False
    for got, want in zip(ref.seen_attention(q, k, v, 0.4, np.repeat(mask[:, None], 6, 1)), ref.cross_attention(q, k, v, 0.4, None, mask)):
        assert np.allclose(got, want, atol=1e-14) and not got[1].any()
    seen = np.broadcast_to(np.arange(9)[None] <= np.arange(-2, 4)[:, None], (2, 6, 9))
    o, a = ref.seen_attention(q, k, v, 0.4, seen)
    assert not o[:, :2].any() and np.allclose(o[:, 2], np.repeat(v[:, 0], 2, 1))
    for j in range(3, 6):
        assert np.allclose(o[:, j:j + 1], ref.cross_attention(q[:, j:j + 1], k, v, 0.4, [j - 1, j - 1])[0])


# ------------------------------------------------------------------ sizes
def test_page_bytes():
    size = wmdec.cache_page_bytes
    for page, heads, d in ((16, 8, 128), (1, 1, 8), (5400, 30, 64), (33, 3, 72), (65536, 8, 256)):
        blocks = -(-d // 32)
        least = page * heads * 2 * (16 * blocks + blocks)
        assert least <= size(page, heads, d) <= least * 1.07 + heads * 16 and size(page, heads, d) % 16 == 0
    assert size(256, 8, 128) == 256 * 8 * 2 * (64 + 4)
    for bad in ((0, 8, 64), (65537, 8, 64), (16, 0, 64), (16, 16385, 64), (16, 8, 0), (16, 8, 60), (16, 8, 264), (65536, 200, 256), (-1, 8, 64), (16, -8, 64)):
        assert size(*bad) == 0, bad


def test_attention_workspace_is_asked_for():
    size = wmdec.lib().wmdec_cache_attention_workspace_bytes
    need = size(wmdec.BF16, 1, 1, 32768, 32, 8, 128)
    assert need > 0 and size(wmdec.BF16, 7, 1, 32768, 32, 8, 128) == 7 * need
    assert size(wmdec.BF16, 1, 1, 77, 30, 30, 64) == 0 and size(wmdec.BF16, 1, 5400, 5400, 30, 30, 64) == 0
    for bad in ((7, 1, 1, 5, 4, 2, 64), (1, 1, 1, -1, 4, 2, 64), (1, 0, 1, 5, 4, 2, 64), (1, 1, 0, 5, 4, 2, 64), (1, 1, 1, 5, 4, 3, 64), (1, 1, 1, 5, 4, 2, 264), (1, 1, 1, 5, 4, 2, 60),
                (1, 1, 1 << 30, 50000, 4, 1, 64), (1, 1 << 23, 1, 20, 4, 2, 64), (1, 1 << 20, 1, 1 << 20, 1, 1, 64), (1, 1, 3, (1 << 31) - 1, 4, 2, 64), (1, 1, (1 << 31) - 1, 5, 64, 2, 64)):
        assert size(*bad) == 0, bad
    big = dict(ATTEND, n=1, tq=1, tk=32768, hq=8)
    for ws, have in ((None, 1 << 40), (7 * P, size(wmdec.BF16, 1, 1, 32768, 8, 2, 64) - 1), (7 * P + 8, 1 << 40)):
        assert _attend(**dict(big, ws=ws, bytes=have)) == wmdec.ERR_WORKSPACE and "workspace" in wmdec.last_error()


# ------------------------------------------------------------------ refusals of the C entry points
P = 0x10000
S = wmdec._CStrides


def _cache(data=P, pages=9, page_tokens=16, heads=2, d=64):
    return wmdec._CCache(data, pages, page_tokens, heads, d)


def _table(pages=2 * P, stride=8, count=8):
    return wmdec._CCacheTable(pages, stride, count)


TOKENS = dict(cache=_cache(), table=_table(), first=3 * P, counts=4 * P, k=5 * P, ks=S(2560, 128, 64), v=6 * P, vs=S(2560, 128, 64), dtype=1, n=2, t=20, stream=None)
ATTEND = dict(q=3 * P, qs=S(768, 256, 64), cache=_cache(), table=_table(), lens=4 * P, counts=5 * P, o=6 * P, os=S(768, 256, 64), dtype=1, scale=0.1, causal=0, n=2, tq=3, tk=100, hq=4,
              ws=7 * P, bytes=1 << 40, stream=None)


def _tokens(name, **changes):
    return getattr(wmdec.lib(), name)(*dict(TOKENS, **changes).values())


def _attend(**changes):
    return wmdec.lib().wmdec_cache_attention(*dict(ATTEND, **changes).values())


OF_THE_CACHE = [
    (wmdec.ERR_INVALID_ARG, dict(cache=None)), (wmdec.ERR_INVALID_ARG, dict(table=None)), (wmdec.ERR_INVALID_ARG, dict(cache=_cache(data=None))),
    (wmdec.ERR_INVALID_ARG, dict(table=_table(pages=None))), (wmdec.ERR_INVALID_ARG, dict(cache=_cache(pages=0))), (wmdec.ERR_INVALID_ARG, dict(cache=_cache(page_tokens=0))),
    (wmdec.ERR_INVALID_ARG, dict(cache=_cache(heads=-2))), (wmdec.ERR_INVALID_ARG, dict(cache=_cache(d=0))), (wmdec.ERR_INVALID_ARG, dict(table=_table(count=-1))),
    (wmdec.ERR_UNSUPPORTED, dict(cache=_cache(d=60))), (wmdec.ERR_UNSUPPORTED, dict(cache=_cache(d=264))), (wmdec.ERR_UNSUPPORTED, dict(cache=_cache(page_tokens=65537))),
    (wmdec.ERR_UNSUPPORTED, dict(cache=_cache(page_tokens=65536, heads=1000))), (wmdec.ERR_UNSUPPORTED, dict(table=_table(count=1 << 27, stride=1 << 27))),
    (wmdec.ERR_INVALID_ARG, dict(cache=_cache(data=P + 8))), (wmdec.ERR_INVALID_ARG, dict(table=_table(pages=2 * P + 2))),
    (wmdec.ERR_SHAPE, dict(table=_table(stride=7))), (wmdec.ERR_SHAPE, dict(table=_table(stride=-8))), (wmdec.ERR_SHAPE, dict(table=_table(stride=1 << 58))),
    (wmdec.ERR_INVALID_ARG, dict(dtype=3)), (wmdec.ERR_INVALID_ARG, dict(n=0)),
]


@pytest.mark.parametrize("status, changes", OF_THE_CACHE + [
    (wmdec.ERR_INVALID_ARG, dict(k=None, v=None)), (wmdec.ERR_INVALID_ARG, dict(t=0)), (wmdec.ERR_INVALID_ARG, dict(ks=None)), (wmdec.ERR_INVALID_ARG, dict(vs=None)),
    (wmdec.ERR_INVALID_ARG, dict(first=3 * P + 2)), (wmdec.ERR_INVALID_ARG, dict(counts=4 * P + 1)), (wmdec.ERR_INVALID_ARG, dict(k=5 * P + 8)),
    (wmdec.ERR_INVALID_ARG, dict(ks=S(2560, 132, 64))), (wmdec.ERR_INVALID_ARG, dict(vs=S(2560, 128, 60))), (wmdec.ERR_INVALID_ARG, dict(ks=S(-2560, 128, 64))),
    (wmdec.ERR_INVALID_ARG, dict(vs=S(1 << 59, 128, 64))), (wmdec.ERR_INVALID_ARG, dict(k=P)), (wmdec.ERR_INVALID_ARG, dict(v=P)),
    (wmdec.ERR_UNSUPPORTED, dict(t=1 << 30, n=64)), (wmdec.ERR_UNSUPPORTED, dict(n=1 << 30, t=1)),
])
@pytest.mark.parametrize("name", ["cache_write", "cache_read"])
def test_tokens_refused(name, status, changes):
    assert _tokens("wmdec_" + name, **changes) == status and name in wmdec.last_error()


@pytest.mark.parametrize("changes", [dict(v=5 * P), dict(ks=S(2560, 0, 64)), dict(vs=S(0, 128, 64)), dict(vs=S(2560, 128, 0))])
def test_read_refuses_outputs_that_overlap(changes):
    assert _tokens("wmdec_cache_read", **changes) == wmdec.ERR_INVALID_ARG and "overlap" in wmdec.last_error()


@pytest.mark.parametrize("status, changes", OF_THE_CACHE + [
    (wmdec.ERR_INVALID_ARG, dict(q=None)), (wmdec.ERR_INVALID_ARG, dict(o=None)), (wmdec.ERR_INVALID_ARG, dict(lens=None)), (wmdec.ERR_INVALID_ARG, dict(qs=None)),
    (wmdec.ERR_INVALID_ARG, dict(os=None)), (wmdec.ERR_INVALID_ARG, dict(tq=0)), (wmdec.ERR_INVALID_ARG, dict(tk=-1)), (wmdec.ERR_INVALID_ARG, dict(hq=0)), (wmdec.ERR_SHAPE, dict(hq=5)),
    (wmdec.ERR_INVALID_ARG, dict(q=3 * P + 8)), (wmdec.ERR_INVALID_ARG, dict(qs=S(768, 260, 64))), (wmdec.ERR_INVALID_ARG, dict(os=S(768, 256, 4))), (wmdec.ERR_INVALID_ARG, dict(qs=S(768, -256, 64))),
    (wmdec.ERR_INVALID_ARG, dict(os=S(0, 256, 64))), (wmdec.ERR_INVALID_ARG, dict(os=S(768, 0, 64))), (wmdec.ERR_INVALID_ARG, dict(os=S(768, 256, 0))),
    (wmdec.ERR_INVALID_ARG, dict(o=3 * P)), (wmdec.ERR_INVALID_ARG, dict(o=P)), (wmdec.ERR_INVALID_ARG, dict(q=P)), (wmdec.ERR_INVALID_ARG, dict(lens=4 * P + 2)), (wmdec.ERR_INVALID_ARG, dict(counts=5 * P + 1)),
    (wmdec.ERR_UNSUPPORTED, dict(n=1 << 20, tq=1 << 20)), (wmdec.ERR_UNSUPPORTED, dict(tk=(1 << 31) - 1)), (wmdec.ERR_UNSUPPORTED, dict(tq=1 << 30)), (wmdec.ERR_UNSUPPORTED, dict(n=1 << 23, tq=1)),
    *[(wmdec.ERR_INVALID_ARG, dict(scale=s)) for s in (0.0, -1.0, 2.1e38, math.inf, math.nan)],
])
def test_attention_refused(status, changes):
    assert _attend(**changes) == status and "cache_attention" in wmdec.last_error()


# ------------------------------------------------------------------ refusals of the binding
def fake(*shape, dtype=torch.bfloat16, device="cuda:0"):
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device=device)


def i32(*shape, **more):
    return fake(*shape, dtype=torch.int32, **more)


def held(pages=9, page=16, heads=2, d=64, data=None):
    return wmdec.Cache(fake(pages, wmdec.cache_page_bytes(page, heads, d), dtype=torch.uint8) if data is None else data, page, heads, d)


@pytest.fixture(autouse=True)
def current_device(monkeypatch):
    """Without a GPU the current device and its stream cannot be asked for; nothing here gets as far as a launch."""
    if not torch.cuda.is_available():
        monkeypatch.setattr(wmdec, "_device", lambda: 0)
        monkeypatch.setattr(wmdec, "_stream", lambda: 0)


def _write(k=None, v=None, cache=None, table=None, first=None, counts=None):
    wmdec.cache_write(fake(2, 3, 2, 64) if k is None else k, fake(2, 3, 2, 64) if v is None else v, held() if cache is None else cache, i32(2, 8) if table is None else table, first, counts)


@pytest.mark.parametrize("call, error", [
    (lambda: _write(k=torch.zeros(2, 3, 2, 64)), AssertionError), (lambda: _write(k=fake(2, 3, 2, 64, device="cuda:1")), AssertionError), (lambda: _write(k=fake(2, 3, 128)), ValueError),
    (lambda: _write(v=fake(2, 4, 2, 64)), ValueError), (lambda: _write(v=fake(2, 3, 2, 64, dtype=torch.float16)), ValueError), (lambda: _write(k=fake(2, 3, 4, 64), v=fake(2, 3, 4, 64)), ValueError),
    (lambda: _write(k=fake(2, 3, 2, 32), v=fake(2, 3, 2, 32)), ValueError), (lambda: _write(k=fake(2, 3, 64, 2).transpose(2, 3)), ValueError), (lambda: _write(k=i32(2, 3, 2, 64)), KeyError),
    (lambda: wmdec.cache_write(None, None, held(), i32(2, 8)), TypeError), (lambda: _write(cache=3), TypeError), (lambda: _write(cache=(1, 2, 3)), TypeError),
    (lambda: _write(cache=held(data=fake(9, 100, dtype=torch.uint8))), ValueError), (lambda: _write(cache=held(data=fake(9, wmdec.cache_page_bytes(16, 2, 64), dtype=torch.int8))), ValueError),
    (lambda: _write(cache=held(data=fake(18, wmdec.cache_page_bytes(16, 2, 64), dtype=torch.uint8)[::2])), AssertionError),
    (lambda: _write(cache=wmdec.Cache(fake(9, 64, dtype=torch.uint8), "x", 2, 64)), TypeError), (lambda: _write(table=fake(2, 8, dtype=torch.int64)), ValueError), (lambda: _write(table=i32(3, 8)), ValueError),
    (lambda: _write(table=i32(8)), ValueError), (lambda: _write(table=i32(2, 16)[:, ::2]), ValueError), (lambda: _write(table=i32(2, 8, device="cuda:1")), AssertionError),
    (lambda: _write(first=i32(3)), ValueError), (lambda: _write(first=fake(2, dtype=torch.int64)), ValueError), (lambda: _write(counts=i32(2, 1)), ValueError),
    (lambda: wmdec.cache_read(held(), i32(2, 8), fake(2, 3, 2, 64), fake(2, 3, 1, 64)), ValueError), (lambda: wmdec.cache_read(held(), i32(2, 8), None, None), TypeError),
    (lambda: wmdec._ops().cache_write(1, 2), TypeError), (lambda: wmdec._ops().bind_cache(1), TypeError),
])
def test_tokens_binding_refuses(call, error):
    with pytest.raises(error):
        call()


def _att(q=None, o=None, cache=None, table=None, lens=None, scale=1.0, tk=10, **more):
    wmdec.cache_attention(fake(2, 3, 4, 64) if q is None else q, held() if cache is None else cache, i32(2, 8) if table is None else table, i32(2) if lens is None else lens,
                          fake(2, 3, 4, 64) if o is None else o, scale, tk, **more)


@pytest.mark.parametrize("call, error", [
    (lambda: _att(q=fake(2, 3, 256)), ValueError), (lambda: _att(q=fake(2, 3, 4, 32), o=fake(2, 3, 4, 32)), ValueError), (lambda: _att(o=fake(2, 3, 2, 64)), ValueError),
    (lambda: _att(o=fake(2, 3, 4, 64, dtype=torch.float16)), ValueError), (lambda: _att(q=torch.zeros(2, 3, 4, 64)), AssertionError), (lambda: _att(lens=i32(3)), ValueError),
    (lambda: _att(lens=fake(2, dtype=torch.int64)), ValueError), (lambda: wmdec.cache_attention(fake(2, 3, 4, 64), held(), i32(2, 8), None, fake(2, 3, 4, 64), 1.0, 10), TypeError),
    (lambda: _att(counts=i32(1)), ValueError), (lambda: _att(scale="x"), TypeError), (lambda: _att(tk="x"), TypeError), (lambda: _att(tk=1.5), TypeError), (lambda: _att(tk=(1 << 32) + 5), ValueError), (lambda: _att(cache=held()._replace(heads=(1 << 32) + 2)), ValueError), (lambda: _att(causal=None), TypeError),
    (lambda: _att(workspace=fake(4, 4, dtype=torch.uint8)), ValueError), (lambda: _att(cache=None, table=i32(1, 8)), ValueError), (lambda: _att(q=fake(2, 3, 64, 4).transpose(2, 3)), ValueError),
    (lambda: wmdec._ops().cache_attention(1, 2), TypeError),
])
def test_attention_binding_refuses(call, error):
    with pytest.raises(error):
        call()


def test_library_refusals_come_through_the_binding():
    """Sizes that the library refuses reach it, and come back as its error.  (No tensor has an address here: only calls that need none get that far.)"""
    with pytest.raises(wmdec.WmdecError) as e:
        wmdec._check(_attend(cache=_cache(d=60)))
    assert e.value.status == wmdec.ERR_UNSUPPORTED and "multiple of 8" in str(e.value)


def test_launches_of_2_to_the_32_threads_are_refused():
    """Workgroups of eight wavefronts count twice."""
    wide = dict(cache=_cache(heads=1, d=8), table=_table(stride=0), qs=S(520, 8, 8), os=S(520, 8, 8), hq=1, tq=65)
    assert _attend(**dict(wide, n=1 << 23)) == wmdec.ERR_UNSUPPORTED and "too many" in wmdec.last_error()
    assert _attend(**dict(wide, cache=_cache(heads=1, d=128), qs=S(65 * 128, 128, 128), os=S(65 * 128, 128, 128), n=1 << 24)) == wmdec.ERR_UNSUPPORTED   # (four at this width)
    assert _attend(**dict(wide, dtype=0, n=1 << 22)) == wmdec.ERR_UNSUPPORTED                                                                    # (blocks of 16 rows)
    for heads, n in ((128, 1 << 16), (256, 1 << 15)):
        assert _attend(**dict(wide, cache=_cache(heads=heads, d=8), qs=S(65 * 8 * heads, 8 * heads, 8), os=S(65 * 8 * heads, 8 * heads, 8), hq=heads, n=n)) == wmdec.ERR_UNSUPPORTED


@pytest.mark.parametrize("name", ["cache_write", "cache_read"])
def test_tokens_of_2_to_the_32_threads_are_refused(name):
    """Workgroups are whole: one to three wavefronts less than 2^26 fill as many."""
    for heads, n, t in ((2731, 8191, 48), (62, 1082401, 1)):   # a head and sixteen tokens of fp32 each: 2^26 - 1, 2^26 - 2
        states = S(t * heads * 8, heads * 8, 8)
        assert _tokens("wmdec_" + name, cache=_cache(page_tokens=1, heads=heads, d=8), table=_table(stride=0), dtype=0, ks=states, vs=states, n=n, t=t) == wmdec.ERR_UNSUPPORTED
        assert "too many" in wmdec.last_error()
