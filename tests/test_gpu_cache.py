"""The cache of keys and values in four bits on the GPU, against the oracle in 64 bits.

What is held is defined to the bit, so writing and reading back are compared for equality.  The tolerance of attention is a bound, element by element:
half a step of the stored type for every rounding to it, and for fp32 arithmetic 2^-24 of the magnitudes that go into an element times the roundings on its way."""
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
MARK = 7.0                                                        # what lies where nothing is to be written


def rng(seed):
    return np.random.default_rng(synth.SEED_BASE + 9000 + seed)


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(G.TORCH[dtype]).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def new_cache(pages, page, hk, d, fill=255):
    """A cache inside a larger allocation; what it holds at first is of no consequence.  (256 bytes on both sides are checked by the second result.)"""
    size = pages * wmdec.cache_page_bytes(page, hk, d)
    big = torch.full((size + 512,), fill, dtype=torch.uint8, device="cuda")
    big[:256] = 77
    big[256 + size:] = 77

    def check():
        assert bool((big[:256] == 77).all()) and bool((big[256 + size:] == 77).all()), "out-of-bounds write"
    return wmdec.Cache(big[256:256 + size].view(pages, -1), page, hk, d), check


def tables(r, n, per, spare=2):
    """Pages of n samples, no two alike, in no order."""
    return r.permutation(n * per + spare)[:n * per].reshape(n, per), n * per + spare


def same_values(got, want):
    """Equal values, sign of zero included; not a number where it is wanted."""
    got, want = np.asarray(got), np.asarray(want)
    bad = ~((got == want) & (np.signbit(got) == np.signbit(want)) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())


# ------------------------------------------------------------------ writing and reading back
def run_store(dtype, n, t, hk, d, page, first=None, counts=None, place=lambda s: s, seed=0, values=None, out_dtype=None, spoil=0):
    """Writes, reads back and compares with the oracle; `spoil` table entries are no pages."""
    r = rng(seed)
    k, v = (G.stored(r.standard_normal((n, t, hk, d)) * np.exp2(r.integers(-6, 6, (n, t, hk, 1))), dtype) if values is None else G.stored(values, dtype) for _ in range(2))
    f = np.zeros(n, int) if first is None else np.asarray(first)
    c = np.full(n, t) if counts is None else np.asarray(counts)
    per = max(1, -(-int((f + t).max()) // page))
    table, pages = tables(r, n, per)
    for _ in range(spoil):
        table[r.integers(n), r.integers(per)] = r.choice([-1, pages, 2 ** 31 - 1, -2 ** 31])
    cache, check = new_cache(pages, page, hk, d)
    before = cache.data.clone()
    ft, ct = None if first is None else ints(first), None if counts is None else ints(counts)
    wmdec.cache_write(place(dev(k, dtype)), place(dev(v, dtype)), cache, ints(table), ft, ct)
    used = np.zeros(pages, bool)
    for b in range(n):
        for i in range(min(max(c[b], 0), t)):
            p = f[b] + i
            if 0 <= p < per * page and 0 <= table[b, p // page] < pages:
                used[table[b, p // page]] = True
    assert torch.equal(cache.data[torch.from_numpy(~used).cuda()], before[torch.from_numpy(~used).cuda()])     # pages that no token lies in
    out = out_dtype or dtype
    ko, vo = (torch.full((n, t, hk, d), MARK, dtype=G.TORCH[out], device="cuda") for _ in range(2))
    kp, vp = place(ko), place(vo)
    wmdec.cache_read(cache, ints(table), kp, vp, ft, ct)
    torch.cuda.synchronize()
    check()
    for x, o in ((k, kp), (v, vp)):
        want = ref.cache_held(x, dtype)
        for b in range(n):
            for i in range(t):
                p = f[b] + i
                if i >= c[b]:
                    want[b, i] = MARK
                elif not (0 <= p < per * page and 0 <= table[b, p // page] < pages):
                    want[b, i] = 0.0
        with np.errstate(over="ignore"):
            same_values(host(o), want if out == dtype else torch.from_numpy(want).to(G.TORCH[out]).double().numpy())
    return cache, table, k, v


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [8, 16, 32, 40, 64, 72, 96, 104, 128, 136, 160, 192, 200, 224, 232, 256])
def test_store_head_sizes(dtype, d):
    run_store(dtype, 2, 37, 3, d, 16, seed=d)
    run_store(dtype, 1, 1, 1, d, 1, seed=d)


@pytest.mark.parametrize("page", [1, 2, 7, 16, 33, 64, 100, 256, 5400, 65536])
@pytest.mark.parametrize("t", [1, 5, 130])
def test_store_pages(page, t):
    run_store("bf16", 2, t, 2, 64, page, seed=page)
    run_store("f32", 2, t, 1, 72, page, first=[3, 5407], seed=page + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_ragged(dtype):
    run_store(dtype, 4, 50, 2, 96, 16, first=[0, 17, 300, 1], counts=[50, 0, 31, 1], seed=1)
    run_store(dtype, 4, 50, 2, 40, 16, first=[5, 0, 2, 9], counts=[60, -3, 50, 49], seed=2)         # counts past both ends
    run_store(dtype, 3, 40, 2, 64, 8, first=[-5, -40, -2 ** 31], seed=3)                          # positions below zero are dropped
    run_store(dtype, 3, 70, 2, 64, 8, spoil=6, seed=4)                                            # entries that are no pages


def test_store_past_the_table():
    """Positions from the row's end on, up to those past 31 bits, are dropped, and read as zeros."""
    for first in (60, 64, 1000, 2 ** 31 - 1):
        cache, check = new_cache(3, 32, 2, 64)
        k = torch.randn((1, 8, 2, 64), device="cuda").bfloat16()
        before = cache.data.clone()
        table = ints([[0, 2]])
        wmdec.cache_write(k, k, cache, table, ints([first]))
        out = torch.full_like(k, MARK)
        wmdec.cache_read(cache, table, out, None, ints([first]))
        inside = max(0, min(8, 64 - first))
        same_values(host(out[:, :inside]), ref.cache_held(host(k[:, :inside]), "bf16"))
        assert not out[:, inside:].any()
        assert torch.equal(cache.data[1], before[1]) and (inside or torch.equal(cache.data, before))
        check()
    none, check = new_cache(1, 16, 1, 32)
    x = torch.randn((2, 3, 1, 32), device="cuda")
    wmdec.cache_write(x, x, none, torch.empty((2, 0), dtype=torch.int32, device="cuda"))     # rows without pages
    assert bool((none.data == 255).all())
    wmdec.cache_read(none, torch.empty((2, 0), dtype=torch.int32, device="cuda"), x, None)
    assert not x.any()


def every(dtype):
    """Numbers whose rounding is next to a border, and those at the ends of the type."""
    steps = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 0.5, 1, 1.5, 2, 3, 4, 6])
    eps = {"f32": 2.0 ** -23, "bf16": 2.0 ** -7, "f16": 2.0 ** -10}[dtype]
    near = np.concatenate([steps, steps * (1 + eps), steps * (1 - eps / 2), [0.0, 2.0 ** -12, 3 * 2.0 ** -9]])
    tops = np.array([4.0, 6.0, 7.0 * (1 - eps / 2), 7.0, 7.0 * (1 + eps), 8.0 * (1 - eps / 2)])
    big = {"f32": 127, "bf16": 127, "f16": 15}[dtype]
    small = {"f32": -140, "bf16": -130, "f16": -24}[dtype]
    rows = []
    for e in list(range(small, small + 12)) + [-8, 0, 5] + list(range(big - 6, big - 1)):
        for top in tops:
            for at in range(0, near.size, 31):
                part = near[at:at + 31]
                rows.append(np.ldexp(np.concatenate([[top], part, np.zeros(31 - part.size)]), e))
    x = np.array(rows)
    x = np.clip(x, 0, {"f32": 3.4028234e38, "bf16": 3.3895e38, "f16": 65504.0}[dtype])
    return x * np.where(np.arange(x.size).reshape(x.shape) % 2, 1.0, -1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_store_rounds_as_defined(dtype):
    x = every(dtype)
    run_store(dtype, 1, x.shape[0], 1, 32, 64, values=x[None, :, None])
    assert np.isfinite(ref.cache_held(G.stored(x, dtype), dtype)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_store_not_finite_stays_in_its_block(dtype):
    x = rng(5).standard_normal((1, 6, 2, 72))
    x[0, 1, 0, 3], x[0, 2, 1, 40], x[0, 3, 0, 71], x[0, 4, 1, 0] = np.nan, np.inf, -np.inf, np.nan
    run_store(dtype, 1, 6, 2, 72, 4, values=x)


def test_read_in_another_type():
    """What bf16 and fp32 wrote, rounded to f16 (past its range: infinite), and what any wrote in the wider types."""
    x = rng(6).standard_normal((1, 40, 2, 64)) * np.exp2(rng(7).integers(-30, 22, (1, 40, 2, 1)))
    for dtype, out in (("bf16", "f16"), ("f32", "f16"), ("f16", "f32"), ("f32", "bf16"), ("f16", "bf16"), ("bf16", "f32")):
        run_store(dtype, 1, 40, 2, 64, 16, values=x, out_dtype=out)


def test_store_strided():
    def in_qkv(s):
        n, t, h, d = s.shape
        big = torch.full((n, t, 3, h + 1, d), MARK, dtype=s.dtype, device="cuda")
        big[:, :, 1, :h].copy_(s)
        return big[:, :, 1, :h]

    def heads_first(s):
        return s.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    for place in (in_qkv, heads_first):
        for dtype in ("bf16", "f32"):
            run_store(dtype, 3, 21, 5, 64, 16, counts=[21, 4, 0], place=place, seed=8)
            run_store(dtype, 3, 21, 5, 40, 16, counts=[21, 4, 0], place=place, seed=8)


def test_store_one_of_both_and_pages_shared():
    r = rng(9)
    k, v = (dev(r.standard_normal((1, 20, 2, 64)), "bf16") for _ in range(2))
    cache, check = new_cache(3, 8, 2, 64)
    table = ints([[2, 0, 1]])
    wmdec.cache_write(k, v, cache, table)
    both = cache.data.clone()
    wmdec.cache_write(None, v, cache, table)
    wmdec.cache_write(k, None, cache, table)
    assert torch.equal(cache.data, both)
    out = torch.empty((3, 20, 2, 64), dtype=torch.bfloat16, device="cuda")
    wmdec.cache_read(cache, table.expand(3, 3), None, out)                     # the same pages for three samples
    same_values(host(out), np.repeat(ref.cache_held(host(v), "bf16"), 3, 0))
    moved = wmdec.Cache(cache.data[[1, 2, 0]].contiguous(), 8, 2, 64)          # pages are moved as a whole
    again = torch.empty_like(k)
    wmdec.cache_read(moved, ints([[1, 2, 0]]), again, None)
    same_values(host(again), ref.cache_held(host(k), "bf16"))
    check()


def test_store_is_stable():
    """What is held is held as itself: storing what was read back changes nothing."""
    cache, table, k, v = run_store("bf16", 2, 33, 2, 72, 16, seed=10)
    ko, vo = (torch.empty((2, 33, 2, 72), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    wmdec.cache_read(cache, ints(table), ko, vo)
    kk = ko.clone()
    wmdec.cache_write(ko, vo, cache, ints(table))
    wmdec.cache_read(cache, ints(table), ko, None)
    assert torch.equal(ko, kk)


def test_store_past_32_bit_offsets():
    page, hk, d = 65536, 8, 256                                       # 136 MiB a page: 40 of them are 5.7 GB
    cache = wmdec.Cache(torch.empty((40, wmdec.cache_page_bytes(page, hk, d)), dtype=torch.uint8, device="cuda"), page, hk, d)
    assert cache.data.numel() > 1 << 32
    k, v = (torch.randn((1, 700, hk, d), device="cuda").bfloat16() for _ in range(2))
    table, first = ints([[0, 39]]), ints([65536 - 300])
    wmdec.cache_write(k, v, cache, table, first)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    wmdec.cache_read(cache, table, ko, vo, first)
    same_values(host(ko), ref.cache_held(host(k), "bf16"))
    same_values(host(vo), ref.cache_held(host(v), "bf16"))


# ------------------------------------------------------------------ attention
def tolerance(dtype, q, k, want, weighted, scale, tk, v):
    """weighted: the softmax weights times |v|.  Half a step for the output; half a step for every probability in 16 bits (and half of the smallest f16
    number, beside a largest probability of at least one); fp32 scores that are off by 3 d + 8 roundings of |q| |k| at most (three products a channel in fp32),
    which moves every weight by twice that; a sum of tk probabilities and exponentials good to a few steps.  And a probability below 2^-126, beside a
    largest one of at least one, may be taken as zero, as may its products with a value: an element loses at most 2^-126 times the sum of |v| for either."""
    d = q.shape[-1]
    size = float(np.sqrt((q ** 2).sum(-1)).max() * np.sqrt((k ** 2).sum(-1)).max()) * scale if k.size else 0.0
    fp32 = 2 * ((3 if dtype == "f32" else 1) * d + 8) * U * size + (math.sqrt(tk) + 64) * 2 * U
    tol = HALF[dtype] * np.abs(want) + TINY[dtype] + fp32 * weighted
    if dtype != "f32":
        tol = tol + HALF[dtype] * weighted * 1.01
    tol = tol + 2 * 2.0 ** -126 * float(np.abs(v).sum(1).max() if v.size else 0.0)
    if dtype == "f16":
        tol = tol + TINY["f16"] * float(np.abs(v).sum(1).max() if v.size else 0.0)
    return tol


def run_attend(dtype, n, tq, tk, hq, hk, d, page, lens=None, counts=None, causal=False, place=lambda s: s, std=1.5, seed=0, spoil=0, source=None, bound=None, scale=None):
    """tk: tokens in the cache; bound: what the call is told."""
    r = rng(500 + seed)
    source = source or dtype
    lens = [tk] * n if lens is None else lens
    q = G.stored(r.standard_normal((n, tq, hq, d)) * std, dtype)
    k, v = (G.stored(r.standard_normal((n, tk, hk, d)), source) for _ in range(2))
    scale = float(np.float32(1 / math.sqrt(d) if scale is None else scale))
    per = max(1, -(-tk // page))
    table, pages = tables(r, n, per)
    for _ in range(spoil):
        table[r.integers(n), r.integers(per)] = r.choice([-1, pages, 2 ** 31 - 1, -2 ** 31])
    cache, ccheck = new_cache(pages, page, hk, d)
    if tk:
        wmdec.cache_write(dev(k, source), dev(v, source), cache, ints(table), None, ints(np.clip(lens, 0, tk)))
    there = np.arange(tk)[None] < np.clip(lens, 0, tk)[:, None]
    there &= np.array([[0 <= table[b, j // page] < pages for j in range(tk)] for b in range(n)], bool).reshape(n, tk)
    kh, vh = (np.where(there[..., None, None], ref.cache_held(x, source), 0.0) for x in (k, v))
    big = torch.full((n, tq, hq, d), MARK, dtype=G.TORCH[dtype], device="cuda")
    o, qd, told = place(big), place(dev(q, dtype)), tk if bound is None else bound
    need = wmdec.cache_attention_workspace_bytes(qd, cache, told)
    ws, wcheck = G.canaried((max(need // 4, 1),), torch.float32)
    wmdec.cache_attention(qd, cache, ints(table), ints(lens), o, scale, told, causal=causal, counts=None if counts is None else ints(counts), workspace=ws if need else None)
    torch.cuda.synchronize()
    ccheck()
    wcheck()
    got = host(o)
    c = np.full(n, tq) if counts is None else np.clip(counts, 0, tq)
    for b in range(n):
        length = int(np.clip(lens[b], 0, tk))
        assert (got[b, c[b]:] == MARK).all()
        if c[b] == 0 or tk == 0:
            assert not got[b, :c[b]].any()
            continue
        seen = np.broadcast_to(there[b], (c[b], tk))
        if causal:
            seen = seen & (np.arange(tk)[None] <= length - c[b] + np.arange(c[b])[:, None])
        rows = slice(0, c[b])
        want, weighted = ref.seen_attention(q[b:b + 1, rows], kh[b:b + 1], vh[b:b + 1], scale, seen[None])
        tol = tolerance(dtype, q[b:b + 1], kh[b:b + 1], want, weighted, scale, tk, vh[b:b + 1])
        bad = ~(np.abs(got[b:b + 1, rows] - want) <= tol)
        assert not bad.any(), (b, int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.abs(got[b:b + 1, rows] - want)[bad].max()), float(np.broadcast_to(tol, want.shape)[bad].max()))
    return o


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [8, 24, 32, 40, 64, 72, 96, 104, 128, 136, 160, 192, 200, 224, 256])
def test_attend_head_sizes(dtype, d):
    run_attend(dtype, 2, 3, 301, 4, 2, d, 64, lens=[301, 130], seed=d)
    run_attend(dtype, 2, 150, 77, 2, 1, d, 16, lens=[77, 70], seed=d + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tq", [1, 2, 15, 17, 33, 65, 129, 257])
@pytest.mark.parametrize("tk", [1, 31, 33, 64, 127, 129, 257, 1000])
def test_attend_lengths(dtype, tq, tk):
    run_attend(dtype, 1, tq, tk, 2, 2, 64, 48, seed=tq + tk)


@pytest.mark.parametrize("group", [1, 2, 3, 4, 7, 8, 16, 33])
def test_attend_groups(group):
    for tq in (1, 2, 40):
        run_attend("bf16", 2, tq, 200, 2 * group, 2, 64, 32, lens=[200, 37], seed=group)


@pytest.mark.parametrize("page", [1, 3, 16, 31, 32, 50, 64, 100, 128, 1000, 5400])
def test_attend_pages(page):
    """Pages that end inside a tile, and entries that are no pages."""
    for tq in (1, 70):
        run_attend("bf16", 2, tq, 900, 4, 2, 64, page, lens=[900, 333], seed=page)
        run_attend("f32", 2, tq, 300, 4, 2, 72, page, spoil=3, seed=page + 1)
        run_attend("f16", 1, tq, 2500, 4, 2, 128, page, spoil=4, causal=tq > 1, seed=page + 2)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_attend_causal(dtype):
    for tq, tk in ((1, 50), (5, 5), (16, 100), (33, 33), (70, 300), (130, 130), (200, 1500)):
        run_attend(dtype, 1, tq, tk, 4, 2, 64, 32, causal=True, seed=tq)
    run_attend(dtype, 4, 60, 400, 6, 2, 96, 32, lens=[400, 60, 17, 0], counts=[60, 60, 17, 0], causal=True, seed=1)
    run_attend(dtype, 3, 40, 100, 3, 3, 40, 8, lens=[10, 39, 100], causal=True, seed=2)               # more queries than tokens: the first see none
    run_attend(dtype, 3, 140, 100, 3, 1, 64, 8, lens=[10, 0, 100], causal=True, seed=3)
    run_attend(dtype, 3, 3, 5000, 4, 1, 128, 64, lens=[5000, 700, 2], counts=[3, 1, 2], causal=True, seed=4)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [24, 64, 72, 128, 160, 192, 224, 256])
def test_attend_blocks_for_all_compute_units(dtype, d):
    """More than 256 blocks of 128 rows: pages that hold less than a tile and more, keys that end inside a tile, pages that are none, causal."""
    run_attend(dtype, 1, 1000, 150, 33, 33, d, 16, seed=d)
    run_attend(dtype, 1, 300, 333, 88, 88, d, 100, spoil=1, lens=[331], seed=d + 1)
    run_attend(dtype, 1, 150, 200, 130, 130, d, 64, causal=True, spoil=1, seed=d + 2)


def test_attend_nothing_to_see():
    for tq in (1, 40, 200):
        for causal in (False, True):
            o = run_attend("bf16", 3, tq, 700, 2, 1, 64, 32, lens=[0, 700, -5], causal=causal, seed=3)
            assert not o[0].any() and not o[2].any()
    o = run_attend("f32", 2, 2, 0, 2, 2, 64, 32, lens=[0, 4], seed=4)
    assert not o.any()
    run_attend("f16", 2, 3, 40, 2, 2, 64, 32, lens=[1000, 2 ** 31 - 1], seed=5)                        # clamped to what is there


def test_attend_counts_of_a_padded_batch():
    for tq in (4, 33, 150):
        run_attend("bf16", 4, tq, 600, 4, 2, 64, 32, lens=[600, 40, 599, 1], counts=[0, tq, 2, tq - 1], seed=6)
        run_attend("bf16", 4, tq, 600, 4, 2, 64, 32, lens=[600, 40, 599, 1], counts=[-1, tq + 5, 2, 1], seed=7)


def test_attend_long():
    run_attend("bf16", 1, 1, 20000, 4, 1, 128, 256, seed=8)
    run_attend("f32", 2, 2, 9000, 4, 2, 64, 100, lens=[9000, 4097], seed=9)
    run_attend("f16", 1, 100, 6000, 2, 1, 64, 100, seed=10)
    run_attend("bf16", 1, 1, 700, 4, 2, 64, 16, lens=[700], bound=100000, seed=11)                     # a bound far above, past the table
    run_attend("bf16", 1, 150, 700, 4, 2, 64, 16, lens=[700], bound=60000, causal=True, seed=12)


def test_attend_strided():
    def in_qkv(s):
        n, t, h, d = s.shape
        big = torch.full((n, t, h + 2, d), MARK, dtype=s.dtype, device="cuda")
        big[:, :, 1:h + 1].copy_(s)
        return big[:, :, 1:h + 1]

    def heads_first(s):
        return s.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    for place in (in_qkv, heads_first):
        for tq in (2, 140):
            run_attend("bf16", 2, tq, 300, 6, 2, 72, 32, counts=[tq, tq - 1], place=place, seed=13)
            run_attend("f32", 2, tq, 900, 6, 2, 64, 32, lens=[900, 3], place=place, seed=13)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_attend_large_scores(dtype):
    """Scores of some thousands: one key has all the weight."""
    for tq in (2, 100):
        run_attend(dtype, 1, tq, 200, 2, 2, 64, 32, std=300.0, seed=14)


def test_attend_largest_probability_is_one():
    """Scores past 2^24 of the reference's steps: the key that wins gets its value to the bit."""
    r = rng(15)
    for dtype in ("bf16", "f32"):
        for tq in (1, 140):
            k = np.zeros((1, 64, 1, 64))
            k[0, :, 0, 0] = np.arange(64) % 2 * 4.0 + 2.0
            k[0, 37, 0, 0] = 6144.0
            v = np.zeros((1, 64, 1, 64))
            v[0, :, 0, 5] = r.permutation(64) % 7
            cache, check = new_cache(4, 16, 1, 64)
            wmdec.cache_write(dev(k, dtype), dev(v, dtype), cache, ints([[3, 1, 0, 2]]))
            q = torch.zeros((1, tq, 1, 64), dtype=G.TORCH[dtype], device="cuda")
            q[..., 0] = 23000.0
            o = torch.empty_like(q)
            wmdec.cache_attention(q, cache, ints([[3, 1, 0, 2]]), ints([64]), o, 1.37, 64)
            assert bool((o[..., 5] == float(ref.cache_held(v, dtype)[0, 37, 0, 5])).all())


def test_attend_not_finite_stays_where_it_is_seen():
    """A block that is not a number reaches the rows that see it, and no others; what lies past a sample's tokens does not matter."""
    for tq, heads, d in ((4, 2, 64), (150, 2, 64), (150, 200, 64), (150, 2, 128), (150, 2, 256), (150, 200, 256)):
        k, v = (torch.randn((2, 200, heads, d), device="cuda") for _ in range(2))
        v[0, 190, 1, 40] = float("inf")
        k[1, 199, 0, 3] = float("nan")
        cache, check = new_cache(26, 16, heads, d)
        table = ints(np.arange(26).reshape(2, 13))
        wmdec.cache_write(k.bfloat16(), v.bfloat16(), cache, table)
        q = torch.randn((2, tq, 2 * heads, d), device="cuda").bfloat16()
        for rows in (2 * heads, heads):                  # two query heads a key head, and one
            o = torch.empty_like(q[:, :, :rows])
            wmdec.cache_attention(q[:, :, :rows], cache, table, ints([191, 199]), o, 0.125, 200, causal=True)
            bad = torch.isnan(o)
            want = torch.zeros_like(bad)
            want[0, -1, rows // heads:2 * rows // heads, 32:64] = True   # the last query alone sees token 190
            assert torch.equal(bad, want)


def test_attend_bits_do_not_depend_on_the_batch():
    r = rng(16)
    for dtype, tq, tk, hq, hk, d in (("bf16", 1, 3000, 8, 2, 128), ("f32", 3, 2000, 4, 2, 64), ("f16", 150, 2500, 4, 2, 64), ("bf16", 20, 900, 4, 1, 96)):
        k, v, q = (dev(r.standard_normal((3, t, h, d)), dtype) for t, h in ((tk, hk), (tk, hk), (tq, hq)))
        per = -(-tk // 64)
        cache, _ = new_cache(3 * per, 64, hk, d)
        table = ints(r.permutation(3 * per).reshape(3, per))
        wmdec.cache_write(k, v, cache, table)
        outs = []
        for samples in ([0, 1, 2], [1], [2, 1]):
            lens = ints([tk, tk - 411, 77])[samples]
            qs, o = q[samples].contiguous(), torch.empty((len(samples), tq, hq, d), dtype=q.dtype, device="cuda")
            ws = torch.empty(max(16, wmdec.cache_attention_workspace_bytes(qs, cache, tk)), dtype=torch.uint8, device="cuda")
            wmdec.cache_attention(qs, cache, table[samples].contiguous(), lens, o, 0.1, tk, workspace=ws)
            outs.append(o[samples.index(1)])
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_attend_equals_attention_to_what_is_read_back():
    """The same softmax over the states that cache_read gives, in f16 from a cache that bf16 wrote too."""
    for dtype, source in (("bf16", "bf16"), ("f16", "bf16"), ("f16", "f16"), ("f32", "bf16")):
        for tq in (3, 140):
            run_attend(dtype, 2, tq, 260, 4, 2, 64, 32, lens=[260, 100], source=source, seed=17)


def test_attend_past_32_bit_offsets():
    page, hk, d = 65536, 8, 256
    cache = wmdec.Cache(torch.empty((40, wmdec.cache_page_bytes(page, hk, d)), dtype=torch.uint8, device="cuda"), page, hk, d)
    k, v = (torch.randn((1, 300, hk, d), device="cuda").bfloat16() for _ in range(2))
    table = ints([[39]])
    wmdec.cache_write(k, v, cache, table)
    for tq in (1, 130):
        q = torch.randn((1, tq, hk, d), device="cuda").bfloat16()
        o = torch.empty_like(q)
        wmdec.cache_attention(q, cache, table, ints([300]), o, 0.0625, 300)
        kh, vh = (ref.cache_held(host(x), "bf16") for x in (k, v))
        want, weighted = ref.cross_attention(host(q), kh, vh, 0.0625)
        assert (np.abs(host(o) - want) <= tolerance("bf16", host(q), kh, want, weighted, 0.0625, 300, vh)).all()


# ------------------------------------------------------------------ together, as they are used
def test_a_stream_of_frames():
    """A block's part of a stream that is made frame by frame: rotary positions, the frame's keys and values into the page of the oldest frame, attention to
    the frames that are there.  The order of a table's pages does not matter to attention, so the oldest page is simply written over."""
    r = rng(30)
    tokens, hq, hk, d, window, n = 45, 6, 2, 64, 3, 2
    freq = torch.empty(32, dtype=torch.float64, device="cuda")
    wmdec.rope_frequencies((16, 24, 24), freq)
    f = ref.rope_frequencies((16, 24, 24))
    cache, check = new_cache(n * window, tokens, hk, d)
    table = ints(r.permutation(n * window).reshape(n, window))
    seen = []
    for frame in range(6):
        place = np.stack([np.full(tokens, frame), np.arange(tokens) // 9, np.arange(tokens) % 9], -1)
        x = G.stored(r.standard_normal((n, tokens, hq + 2 * hk, d)), "bf16")
        xd = dev(x, "bf16")
        q, k, v = xd[:, :, :hq], xd[:, :, hq:hq + hk], xd[:, :, hq + hk:]
        wmdec.rope(q, k, ints(place), freq, (16, 24, 24), q, k)
        first = ints([frame % window * tokens] * n)
        wmdec.cache_write(k, v, cache, table, first)
        lens = min(frame + 1, window) * tokens
        o = torch.empty((n, tokens, hq, d), dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(max(16, wmdec.cache_attention_workspace_bytes(q, cache, window * tokens)), dtype=torch.uint8, device="cuda")
        wmdec.cache_attention(q, cache, table, ints([lens] * n), o, 0.125, window * tokens, workspace=ws)
        turned = ref.rope(x[:, :, hq:hq + hk], place[None].repeat(n, 0), f, (16, 24, 24))
        assert (np.abs(host(k) - turned) <= HALF["bf16"] * np.abs(turned) + 2.0 ** -18).all()
        seen = (seen + [(host(k), x[:, :, hq + hk:])])[-window:]
        kh, vh = (ref.cache_held(np.concatenate([s[i] for s in seen], 1), "bf16") for i in (0, 1))
        want, weighted = ref.cross_attention(host(q), kh, vh, 0.125)
        assert (np.abs(host(o) - want) <= tolerance("bf16", host(q), kh, want, weighted, 0.125, lens, vh)).all()
        # the same states, read back and attended to as dense ones
        ko, vo = (torch.empty((n, lens, hk, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        wmdec.cache_read(cache, table, ko, vo)
        dense = torch.empty_like(o)
        ws = torch.empty(max(16, wmdec.cross_attention_workspace_bytes(q, ko)), dtype=torch.uint8, device="cuda")
        wmdec.cross_attention(q, ko, vo, dense, 0.125, workspace=ws)
        assert (np.abs(host(dense) - want) <= tolerance("bf16", host(q), kh, want, weighted, 0.125, lens, vh)).all()
    check()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_prompt_and_then_token_by_token(dtype):
    """A padded batch of prompts in two stretches, and then a token of every sequence at a time."""
    r = rng(31)
    n, hq, hk, d, page = 3, 4, 2, 96, 24
    lengths = np.array([130, 64, 7])
    total = lengths + 5
    q, k, v = (G.stored(r.standard_normal((n, 135, h, d)), dtype) for h in (hq, hk, hk))
    per = -(-135 // page)
    cache, check = new_cache(n * per + 1, page, hk, d)
    table = ints(r.permutation(n * per + 1)[:n * per].reshape(n, per))
    kh, vh = ref.cache_held(k, dtype), ref.cache_held(v, dtype)
    steps = [(np.zeros(n, int), np.minimum(lengths, 60)), (np.minimum(lengths, 60), lengths - np.minimum(lengths, 60))] + [(lengths + i, np.ones(n, int)) for i in range(5)]
    for first, count in steps:
        t = int(count.max())
        part = [torch.full((n, t, h, d), float("nan"), device="cuda").to(G.TORCH[dtype]) for h in (hq, hk, hk)]     # what pads the batch does not matter
        for b in range(n):
            for x, y in zip(part, (q, k, v)):
                x[b, :count[b]] = dev(y[b, first[b]:first[b] + count[b]], dtype)
        wmdec.cache_write(part[1], part[2], cache, table, ints(first), ints(count))
        o = torch.full((n, t, hq, d), MARK, device="cuda").to(G.TORCH[dtype])
        ws = torch.empty(max(16, wmdec.cache_attention_workspace_bytes(part[0], cache, 135)), dtype=torch.uint8, device="cuda")
        wmdec.cache_attention(part[0], cache, table, ints(first + count), o, 0.1, 135, causal=True, counts=ints(count), workspace=ws)
        got = host(o)
        for b in range(n):
            assert (got[b, count[b]:] == MARK).all()
            for i in range(count[b]):
                see = first[b] + i + 1
                at = slice(first[b] + i, first[b] + i + 1)
                want, weighted = ref.cross_attention(q[b:b + 1, at], kh[b:b + 1, :see], vh[b:b + 1, :see], float(np.float32(0.1)))
                assert (np.abs(got[b:b + 1, i:i + 1] - want) <= tolerance(dtype, q[b:b + 1, at], kh[b:b + 1, :see], want, weighted, 0.1, see, vh[b:b + 1, :see])).all(), (b, i)
    assert (first + count == total).all()
    check()


def test_graphs_are_replayed():
    """A token's step captured: what it reads and writes is on the device, positions and lengths among it.  Two graphs share a workspace; every replay is compared with
    an eager step on a cache of its own, with eager work and synchronisation in between."""
    r = rng(32)
    n, hq, hk, d, page, most = 2, 8, 2, 128, 64, 20000
    per = -(-most // page)
    table = ints(r.permutation(n * per).reshape(n, per))
    start = [dev(r.standard_normal((n, 2500, hk, d)), "bf16") for _ in range(2)]
    caches = [new_cache(n * per, page, hk, d)[0] for _ in range(2)]
    for c in caches:
        wmdec.cache_write(*start, c, table)
    q, k, v = (torch.zeros((n, 1, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hk, hk))
    first, lens = ints([2500, 1300]), ints([2501, 1301])
    o, wide, qw, ow = torch.empty_like(q), [torch.empty((n, 1, hk, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)], torch.zeros((n, 90, hq, d), dtype=torch.bfloat16, device="cuda"), None
    ow = torch.empty_like(qw)
    ws = torch.empty(max(wmdec.cache_attention_workspace_bytes(x, caches[0], most) for x in (q, qw)), dtype=torch.uint8, device="cuda")
    assert min(wmdec.cache_attention_workspace_bytes(x, caches[0], most) for x in (q, qw)) > 0

    def token(c, out, back):
        wmdec.cache_write(k, v, c, table, first)
        wmdec.cache_attention(q, c, table, lens, out, 0.09, most, workspace=ws)
        wmdec.cache_read(c, table, back[0], back[1], first)

    def many(c, out):
        wmdec.cache_attention(qw, c, table, lens, out, 0.09, most, causal=True, workspace=ws)
    token(caches[0], o, wide)
    many(caches[0], ow)
    torch.cuda.synchronize()
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        token(caches[0], o, wide)
    with torch.cuda.graph(two):
        many(caches[0], ow)
    for i in range(5):
        for x in (q, k, v, qw):
            x.copy_(dev(r.standard_normal(tuple(x.shape)), "bf16"))
        one.replay()
        if i % 2:
            two.replay()
        eager, eb, em = torch.empty_like(o), [torch.empty_like(x) for x in wide], torch.empty_like(ow)
        token(caches[1], eager, eb)
        many(caches[1], em)
        if not i % 2:
            two.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, eager) and torch.equal(ow, em) and all(torch.equal(a, b) for a, b in zip(wide, eb))
        assert torch.isfinite(o).all() and torch.isfinite(ow).all()
        first += 1
        lens += 1


def test_calls_on_streams_of_their_own():
    """Calls on two streams at once, each with a cache, a workspace and outputs of its own, give what they give one after the other."""
    r = rng(33)
    jobs = []
    for i, (dtype, tq) in enumerate((("bf16", 1), ("f16", 100))):
        k, v, q = (dev(r.standard_normal((2, t, h, 64)), dtype) for t, h in ((3000, 2), (3000, 2), (tq, 8)))
        cache, _ = new_cache(2 * 47, 64, 2, 64)
        table = ints(r.permutation(94).reshape(2, 47))
        o = [torch.empty_like(q) for _ in range(6)]
        ws = torch.empty(max(16, wmdec.cache_attention_workspace_bytes(q, cache, 3000)), dtype=torch.uint8, device="cuda")
        back = [torch.empty_like(k) for _ in range(2)]
        jobs.append((k, v, q, cache, table, o, ws, back))
    lens = ints([3000, 1700])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for i in range(5):
        for s, (k, v, q, cache, table, o, ws, back) in zip(streams, jobs):
            with torch.cuda.stream(s):
                wmdec.cache_write(k, v, cache, table)
                wmdec.cache_attention(q, cache, table, lens, o[i], 0.125, 3000, workspace=ws)
                wmdec.cache_read(cache, table, *back)
    torch.cuda.synchronize()
    for k, v, q, cache, table, o, ws, back in jobs:
        wmdec.cache_attention(q, cache, table, lens, o[5], 0.125, 3000, workspace=ws)
        torch.cuda.synchronize()
        assert all(torch.equal(x, o[5]) for x in o[:5])
        same_values(host(back[0]), ref.cache_held(host(k), {torch.bfloat16: "bf16", torch.float16: "f16"}[k.dtype]))


def test_attend_samples_that_share_pages():
    """A prefix that all samples have in common is held once: rows of the table with the same pages, and one row for all."""
    r = rng(34)
    k, v = (dev(r.standard_normal((1, 200, 2, 64)), "bf16") for _ in range(2))
    cache, check = new_cache(7, 32, 2, 64)
    row = ints([[4, 0, 6, 1, 2, 3, 5]])
    wmdec.cache_write(k, v, cache, row)
    for tq in (1, 80):
        q = dev(r.standard_normal((3, tq, 4, 64)), "bf16")
        o, again = torch.empty_like(q), torch.empty_like(q)
        lens = ints([200, 33, 150])
        wmdec.cache_attention(q, cache, row.expand(3, 7), lens, o, 0.125, 200)
        wmdec.cache_attention(q, cache, row.repeat(3, 1), lens, again, 0.125, 200)
        assert torch.equal(o, again)
        kh, vh = (ref.cache_held(host(x), "bf16").repeat(3, 0) for x in (k, v))
        want, weighted = ref.cross_attention(host(q), kh, vh, 0.125, [200, 33, 150])
        assert (np.abs(host(o) - want) <= tolerance("bf16", host(q), kh, want, weighted, 0.125, 200, vh)).all()
    check()


# ------------------------------------------------------------------ values that the type of the call does not hold
def attend_what_is_held(dtype, q, kh, vh, scale, lens, causal, source, k, v, page):
    """Writes k and v as `source`, attends in `dtype`, and compares with the oracle on kh, vh.  An infinite value makes its channel infinite for the queries that see its
    key (not a number, where they see both signs), and is nothing to the others; what is finite is compared as ever."""
    n, tq, hq, d = q.shape
    tk, hk = k.shape[1:3]
    per = -(-tk // page)
    table, pages = tables(rng(600), n, per)
    cache, check = new_cache(pages, page, hk, d)
    wmdec.cache_write(dev(k, source), dev(v, source), cache, ints(table), None, ints(lens))
    qd = dev(q, dtype)
    o = torch.full_like(qd, MARK)
    need = wmdec.cache_attention_workspace_bytes(qd, cache, tk)
    wmdec.cache_attention(qd, cache, ints(table), ints(lens), o, scale, tk, causal=causal, workspace=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
    got = host(o)
    check()
    group = hq // hk
    for b in range(n):
        seen = np.broadcast_to(np.arange(tk)[None] < lens[b], (tq, tk))
        if causal:
            seen = seen & (np.arange(tk)[None] <= lens[b] - tq + np.arange(tq)[:, None])
        finite = np.where(np.isfinite(vh[b:b + 1]), vh[b:b + 1], 0.0)
        want, weighted = ref.seen_attention(q[b:b + 1], kh[b:b + 1], finite, scale, seen[None])
        tol = tolerance(dtype, q[b:b + 1], kh[b:b + 1, :lens[b]], want, weighted, scale, tk, finite)
        at = np.flatnonzero(~np.isfinite(vh[b]).all((1, 2)))
        up, down, none = ((seen[:, at, None, None] & x[None, at]).any(1).repeat(group, 1) for x in (vh[b] == np.inf, vh[b] == -np.inf, np.isnan(vh[b])))
        special = np.where(none | (up & down), np.nan, np.where(up, np.inf, np.where(down, -np.inf, 0.0)))
        ordinary = special == 0.0
        assert ordinary.any() and not ordinary.all()
        g = got[b]
        bad = np.where(ordinary, ~(np.abs(np.where(ordinary, g, 0.0) - want[0]) <= tol[0]), ~((g == special) | (np.isnan(g) & np.isnan(special))))
        assert not bad.any(), (b, int(bad.sum()), np.argwhere(bad)[:4].tolist(), g[bad][:4].tolist(), want[0][bad][:4].tolist(), special[bad][:4].tolist())


@pytest.mark.parametrize("source", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("tq, tk, hq, hk, d, page", [
    (4, 90, 2, 2, 40, 16), (5, 100, 8, 2, 64, 33), (3, 2000, 4, 2, 128, 64), (6, 500, 2, 2, 160, 33), (3, 1300, 2, 2, 256, 100), (16, 70, 4, 2, 96, 16), (9, 40, 2, 2, 32, 7),
    (150, 200, 2, 2, 40, 16), (150, 330, 4, 2, 64, 100), (100, 4000, 2, 2, 128, 100), (140, 150, 2, 2, 160, 16), (130, 260, 2, 2, 224, 64), (70, 300, 2, 2, 256, 31),
    (300, 200, 88, 88, 64, 64), (300, 150, 90, 90, 96, 16), (150, 180, 130, 130, 192, 32), (260, 330, 90, 90, 256, 100)])
def test_attend_values_past_f16(source, causal, tq, tk, hq, hk, d, page):
    """f16 over what another type wrote: values past 65504 are infinite, as cache_read gives them, and reach the queries that see them alone."""
    r = rng(700 + d + tk)
    q = G.stored(r.standard_normal((2, tq, hq, d)) * 1.5, "f16")
    k, v = (r.standard_normal((2, tk, hk, d)) for _ in range(2))
    last, blocks = min(tq, tk), (d + 31) // 32
    # blocks whose largest is infinite in f16, and all or some of whose others are not: of a token that all queries see in the first head, of some that the last ones see in the second
    for b in range(2):
        v[b, 1, 0, 32 * (blocks - 1):] *= 2.0 ** 15
        for i, power in enumerate((14, 15, 16, 17, 40)):
            v[b, tk - 1 - (i * (last - 1)) // 5 - 3 * b, 1, 32 * (i % blocks):32 * (i % blocks) + 32] *= 2.0 ** power
    k, v = G.stored(k, source), G.stored(v, source)
    kh, vh = ref.cache_held(k, source), ref.cache_held(v, source)
    with np.errstate(over="ignore"):
        vh = vh.astype(np.float16).astype(np.float64)
    attend_what_is_held("f16", q, kh, vh, float(np.float32(1 / math.sqrt(d))), [tk, tk - 3], causal, source, k, v, page)


def test_attend_values_past_f16_whatever_their_weight():
    """An infinite value counts where its probability is nothing in f16, before and behind larger ones, and where no query of a tile has a score before it."""
    for tq, tk, slope in ((1, 300, 40), (4, 3000, 40), (120, 300, 40), (1, 300, -40), (4, 3000, -40), (120, 300, -40)):
        q, k, v = np.zeros((1, tq, 2, 64)), np.zeros((1, tk, 2, 64)), np.ones((1, tk, 2, 64))
        q[..., 0] = 1.0
        k[0, :, :, 0] = np.linspace(-slope, slope, tk)[:, None]
        v[0, 3, 0, 5], v[0, tk - tq, 1, 40], v[0, tk // 2, 1, 41] = 1e6, -1e30, 3e5
        v[0, :, 0, 7] = np.arange(tk) % 5
        k, v = G.stored(k, "bf16"), G.stored(v, "bf16")
        with np.errstate(over="ignore"):
            kh, vh = ref.cache_held(k, "bf16"), ref.cache_held(v, "bf16").astype(np.float16).astype(np.float64)
        for causal in (False, True):
            attend_what_is_held("f16", q, kh, vh, 1.0, [tk], causal, "bf16", k, v, 32)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_attend_scores_half_a_step_beside_the_reference(dtype):
    """From 2^27 on fp32 holds scores in steps of 16, and a reference and eight more may be the next score: that one's probability is 2^16 unless the reference moves,
    which f16 does not hold.  Two keys alone have weight, with values of 1 and 2: an output lies between them."""
    for tq in (1, 5, 140):
        for low, high in ((8, 24), (16, 24), (32, 48)):
            k, v = np.zeros((1, 200, 2, 64)), np.ones((1, 200, 2, 64))
            k[0, (5, 133), :, 0] = 4096.0
            k[0, 5, :, 32], k[0, 133, :, 32] = low, high
            v[0, 133] = 2.0
            cache, check = new_cache(13, 16, 2, 64)
            table = ints([list(range(13))])
            wmdec.cache_write(dev(k, dtype), dev(v, dtype), cache, table)
            q = torch.zeros((1, tq, 2, 64), dtype=G.TORCH[dtype], device="cuda")
            q[..., 0], q[..., 32] = 22720.0, 1.0
            o = torch.empty_like(q)
            wmdec.cache_attention(q, cache, table, ints([200]), o, 1.0, 200)
            assert bool(((o >= 1.0) & (o <= 2.0)).all()), (tq, low, high, o.flatten()[:4].tolist())
            check()


def test_attend_queries_at_the_end_of_fp32():
    """fp32 queries go into the products in pieces; those next to the largest number, and infinite ones, are in order too."""
    top = 3.4028234e38
    for tq in (1, 40):
        q = np.zeros((1, tq, 1, 64))
        q[..., 0] = np.array([top, -top, 3.39e38, 3.3961776e38, 3.3961775e38])[np.arange(tq) % 5][None, :, None]
        q = G.stored(q, "f32")
        k = np.zeros((1, 50, 1, 64))
        k[0, :, 0, 0] = 2.0 ** -125 * np.array([0.5, 1, 1.5, 2, 3, 4, -2, 0])[np.arange(50) % 8]
        v = rng(41).standard_normal((1, 50, 1, 64))
        cache, check = new_cache(4, 16, 1, 64)
        table = ints([[1, 3, 0, 2]])
        wmdec.cache_write(dev(k, "f32"), dev(v, "f32"), cache, table)
        qd = dev(q, "f32")
        o = torch.full_like(qd, MARK)
        wmdec.cache_attention(qd, cache, table, ints([50]), o, 1.0, 50)
        kh, vh = ref.cache_held(k, "f32"), ref.cache_held(G.stored(v, "f32"), "f32")
        want, weighted = ref.cross_attention(q, kh, vh, 1.0)
        # (the tolerance of test_attend_*, whose bound on the scores, sums of 64 |q| |k|, is of their magnitude here)
        with np.errstate(over="ignore"):
            size = float(np.abs(q[0, :, 0, :1] * kh[0, :, 0, 0][None]).max())
        fp32 = 2 * (3 * 64 + 8) * U * size + (math.sqrt(50) + 64) * 2 * U
        assert (np.abs(host(o) - want) <= U * np.abs(want) + fp32 * weighted + 2.0 ** -126).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_attend_scores_of_minus_infinity(dtype):
    """A query whose scores are all -inf gets zeros; the others are not touched by it."""
    for tq in (2, 80):
        q = rng(42).standard_normal((1, tq, 1, 64))
        k, v = rng(43).standard_normal((1, 60, 1, 64)), rng(44).standard_normal((1, 60, 1, 64))
        k[..., 0] = 1.0 + np.abs(k).max()
        q[0, 0, 0, 0] = -np.inf
        cache, check = new_cache(4, 16, 1, 64)
        table = ints([[1, 3, 0, 2]])
        wmdec.cache_write(dev(k, dtype), dev(v, dtype), cache, table)
        qd = dev(q, dtype)
        o = torch.full_like(qd, MARK)
        wmdec.cache_attention(qd, cache, table, ints([60]), o, 0.125, 60)
        assert not o[0, 0].any()
        kh, vh = (ref.cache_held(G.stored(x, dtype), dtype) for x in (k, v))
        rest = G.stored(q[:, 1:], dtype)
        want, weighted = ref.cross_attention(rest, kh, vh, 0.125)
        assert (np.abs(host(o[:, 1:]) - want) <= tolerance(dtype, rest, kh, want, weighted, 0.125, 60, vh)).all()


def test_attend_as_many_samples_as_a_launch_takes():
    n = (1 << 23) - 1
    k, v = (torch.randn((1, 3, 1, 8), device="cuda").bfloat16() for _ in range(2))
    cache, check = new_cache(1, 16, 1, 8)
    wmdec.cache_write(k, v, cache, ints([[0]]))
    q = torch.randn((1, 65, 1, 8), device="cuda").bfloat16()
    o = torch.full((n, 65, 1, 8), MARK, dtype=torch.bfloat16, device="cuda")
    wmdec.cache_attention(q.expand(n, 65, 1, 8), cache, ints([[0]]).expand(n, 1), torch.full((n,), 3, dtype=torch.int32, device="cuda"), o, 0.3, 3)
    kh, vh = (ref.cache_held(host(x), "bf16") for x in (k, v))
    want, weighted = ref.cross_attention(host(q), kh, vh, 0.3)
    assert (np.abs(host(o[:1]) - want) <= tolerance("bf16", host(q), kh, want, weighted, 0.3, 3, vh)).all()
    for at in range(0, n, 1 << 20):
        assert bool((o[at:at + (1 << 20)] == o[:1]).all())
    check()


def test_store_as_many_tokens_as_a_launch_takes():
    """2^26 - 4 wavefronts."""
    n, heads = 4097, 16380
    assert n * heads == (1 << 26) - 4
    k = torch.randn((n, 1, heads, 8), device="cuda")
    cache, check = new_cache(n, 1, heads, 8)
    table = torch.arange(n, dtype=torch.int32, device="cuda").flip(0).contiguous()[:, None]
    wmdec.cache_write(k, None, cache, table)
    out = torch.full_like(k, MARK)
    wmdec.cache_read(cache, table, out, None)
    for at in (0, 1, 2047, n - 1):
        same_values(host(out[at]), ref.cache_held(host(k[at]), "f32"))
    assert bool((out.abs() <= 8).all()) and not bool((out == MARK).any())
    check()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [40, 72, 160, 256])
@pytest.mark.parametrize("page", [16, 33])
@pytest.mark.parametrize("tq, tk, hq, hk", [(4, 90, 2, 2), (3, 1400, 4, 2), (150, 200, 2, 2), (100, 4000, 2, 2), (300, 150, 88, 88)])
def test_attend_not_a_number_by_block(dtype, d, page, tq, tk, hq, hk):
    """Blocks of values that are not a number, the last of a head among them, in tiles that some of a block's rows see, whose sums are joined from ranges or not."""
    r = rng(800 + d)
    q = G.stored(r.standard_normal((2, tq, hq, d)) * 1.5, dtype)
    k, v = (G.stored(r.standard_normal((2, tk, hk, d)), dtype) for _ in range(2))
    blocks, last = (d + 31) // 32, min(tq, tk)
    for b in range(2):
        v[b, tk - 1 - 3 * b, 0, 32 * (blocks - 1) + 7] = np.nan
        v[b, tk - 1 - last // 2, 1, 32 * (blocks // 2) + 1] = np.inf
        v[b, tk - last, 1, 32 * (blocks // 3)] = -np.inf
    kh, vh = ref.cache_held(k, dtype), ref.cache_held(v, dtype)
    for causal in (True, False):
        attend_what_is_held(dtype, q, kh, vh, float(np.float32(1 / math.sqrt(d))), [tk, tk - 3], causal, dtype, k, v, page)


def test_attend_keys_that_are_not_a_number():
    """A key that is not a number makes every channel of the queries that see it so, and is nothing to the others."""
    for dtype, tq, tk, d, page in (("bf16", 4, 90, 160, 16), ("f16", 5, 1400, 72, 33), ("f32", 4, 700, 256, 16), ("bf16", 150, 200, 160, 33), ("f16", 100, 4000, 64, 100)):
        q, k, v = (torch.randn((1, t, 2, d), device="cuda").to(G.TORCH[dtype]) for t in (tq, tk, tk))
        bad = tk - 1 - tq // 2
        k[0, bad, 1, d - 1] = float("nan")
        per = -(-tk // page)
        cache, check = new_cache(per, page, 2, d)
        table = ints(rng(45).permutation(per)[None])
        wmdec.cache_write(k, v, cache, table)
        o = torch.empty_like(q)
        ws = torch.empty(max(16, wmdec.cache_attention_workspace_bytes(q, cache, tk)), dtype=torch.uint8, device="cuda")
        wmdec.cache_attention(q, cache, table, ints([tk]), o, 0.1, tk, causal=True, workspace=ws)
        want = torch.zeros_like(o, dtype=torch.bool)
        want[0, tq - 1 - tq // 2:, 1] = True
        assert torch.equal(torch.isnan(o), want)
        check()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_attend_scales_of_any_size(dtype):
    """Scales at both ends of what is taken, with queries that bring the scores back to their size, or not."""
    for tq in (2, 90):
        for scale, size in ((1e-45, 1.0), (1e-39, 1.0), (2.0 ** -10, 2.0 ** 10)) + (((2e38, 2.0 ** -126), (1e38, 2.0 ** -121)) if dtype != "f16" else ((2.0 ** 24, 2.0 ** -24), (2.0 ** 20, 2.0 ** -18))):
            r = rng(900 + tq)
            q = G.stored(r.standard_normal((1, tq, 2, 64)) * size, dtype)
            k, v = (G.stored(r.standard_normal((1, 150, 2, 64)), dtype) for _ in range(2))
            cache, check = new_cache(10, 16, 2, 64)
            table = ints([list(range(10))])
            wmdec.cache_write(dev(k, dtype), dev(v, dtype), cache, table)
            qd = dev(q, dtype)
            o = torch.full_like(qd, MARK)
            scale = float(np.float32(scale))
            wmdec.cache_attention(qd, cache, table, ints([150]), o, scale, 150, causal=True)
            kh, vh = (ref.cache_held(x, dtype) for x in (k, v))
            seen = (np.arange(150)[None] <= 150 - tq + np.arange(tq)[:, None])[None]
            want, weighted = ref.seen_attention(q, kh, vh, scale, seen)
            tol = tolerance(dtype, q, kh, want, weighted, scale, 150, vh)
            if dtype == "f32":   # the last of a query's three pieces is a bf16 number, in steps of 2^-133: an element is off by half of one, a score by that times |k|, and a weight by a factor of twice that score's exponential
                tol = tol + math.expm1(2 * 2.0 ** -134 * float(np.abs(kh).sum(-1).max()) * scale) * weighted
            bad = ~(np.abs(host(o) - want) <= tol)
            assert not bad.any(), (tq, scale, size, int(bad.sum()), np.abs(host(o) - want)[bad].max())
