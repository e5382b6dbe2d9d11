"""A cache of keys and values in four bits, as cases to be timed: states stored and handed back as they are stored, a stretch of
the cache read back, and attention to what it holds.

The format: 32 channels of a head of a token (the last block of a head may be shorter) share a power of two 2^e, and a value is a sign and one of
0, 0.5, 1, 1.5, 2, 3, 4, 6 times that.  e is floor(log2(largest magnitude)) - 2, and one more where the largest magnitude is 1.75 times its power
of two or above, kept within -125 .. 125 (.. 13 where the source is f16).  Nearest values, ties to the even place of the list, 6 for what is above.
A sequence's tokens lie in pages of a pool, in the order that its row of a page table gives.

Sizes: 5400 tokens are the 60x90 latent of a 480x720 frame, 30 heads of 64 channels are the width of 1920 that the block's other operators are
timed at; the others are generic.  Where `own` is false every operator runs in its plain form, in 32-bit torch operations, rounded
once at the end, on codes and exponents that stand in plain tensors; where it is true through the library's entry points.
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 32
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # one token of a stream that advances token by token; latency
        _store("store_1_30x64_bf16", "bf16", 1, 1, 30, 64, 256, 300, False),
        # a token of each of many streams in the middle of their sequences
        _store("store_64x1_8x128_f16", "f16", 64, 1, 8, 128, 16, 700, True),
        # a frame and its twin, a page each, behind the frame before
        _store("store_2x5400_30x64_bf16", "bf16", 2, 5400, 30, 64, 5400, 5400, False),
        # a sensitive layer in fp32, a padded batch of prompts, heads that end inside a block, pages of an odd size
        _store("store_5x1001_6x72_f32", "f32", 5, 1001, 6, 72, 100, 37, True),
        # long states handed on in 16 bits
        _read("read_1x32768_8x128_bf16", "bf16", 1, 32768, 8, 128, 256, 0, False),
        # stretches of different lengths from the middle of three sequences
        _read("read_3x777_10x96_f32", "f32", 3, 777, 10, 96, 48, 61, True),
        # one token against a short sequence; latency
        _attend("attend_1x77_30x64_bf16", "bf16", 2, 1, 77, 30, 30, 64, 64, False, False),
        # a token of each of 16 streams, grouped heads
        _attend("attend_16x1x4096_32_8x128_f16", "f16", 16, 1, 4096, 32, 8, 128, 64, False, False),
        # one token of four streams of different lengths: the most bytes
        _attend("attend_4x1x65536_32_8x128_bf16", "bf16", 4, 1, 65536, 32, 8, 128, 256, True, False),
        # a few tokens at a time in fp32, causal, heads of an odd multiple of eight
        _attend("attend_3x5x2000_8_2x72_f32", "f32", 3, 5, 2000, 8, 2, 72, 33, True, True),
        # a stretch of a prompt behind what is there of it, padded and causal
        _attend("attend_3x700x3500_16_4x128_bf16", "bf16", 3, 700, 3500, 16, 4, 128, 100, True, True),
        # the tokens of a frame against that frame and the one before it: the most arithmetic
        _attend("attend_5400x10800_30x64_f16", "f16", 1, 5400, 10800, 30, 30, 64, 5400, False, False),
    ]


def _store(name, dtype, n, t, hk, d, page, before, ragged):
    """before: tokens that a sequence has already, at most; ragged: sequences have earlier tokens of their own number, and of more than one new token too."""
    return {"name": name, "op": "store", "dtype": dtype, "n": n, "t": t, "hk": hk, "d": d, "page": page, "before": before, "ragged": ragged}


def _read(name, dtype, n, t, hk, d, page, before, ragged):
    return dict(_store(name, dtype, n, t, hk, d, page, before, ragged), op="read")


def _attend(name, dtype, n, tq, tk, hq, hk, d, page, ragged, causal):
    """ragged: sequences have lengths of their own (with three or more one has none); causal: a sequence's queries are its last tokens."""
    return {"name": name, "op": "attend", "dtype": dtype, "n": n, "tq": tq, "tk": tk, "hq": hq, "hk": hk, "d": d, "page": page, "ragged": ragged, "causal": causal}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, of no more work than the largest listed one of its operator."""
    op = rng.choice(["store", "read", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f16", "f32"])
    hk, d = rng.choice([1, 2, 5, 8, 10, 30]), rng.choice([8, 32, 64, 64, 72, 96, 128, 128, 160, 256])
    n, page = rng.choice([1, 1, 2, 3, 4, 16]), rng.choice([1, 16, 33, 64, 100, 256, 1024, 5400])
    if op != "attend":
        t = max(1, min(_log(rng, 1, 32768), 32768 * 8 * 128 * 2 // (n * hk * _blocks(d) * BLOCK * SIZE[dtype])))
        return _without_name((_store if op == "store" else _read)("", dtype, n, t, hk, d, page, _log(rng, 1, 6000) - 1, rng.random() < 0.5))
    group = rng.choice([1, 1, 2, 4, 7, 16])
    tq, tk = (rng.choice([1, 1, 1, 2, 5]) if rng.random() < 0.6 else _log(rng, 8, 8000)), _log(rng, 1, 131072)
    # keys are cut to the reading of the longest listed sequences, queries to as many elements, both to the arithmetic of a frame and two
    tk = min(tk, 65536 * 4 * 8 * 128 // (n * hk * _blocks(d) * BLOCK))
    tq = max(1, min(tq, 32768 * 8 * 128 * 2 // (n * hk * group * d * SIZE[dtype])))
    tk = max(1, min(tk, 5400 * 10800 * 30 * 64 // (n * tq * hk * group * max(d, 64) * (4 if dtype == "f32" else 1))))
    return _without_name(_attend("", dtype, n, tq, tk, hk * group, hk, d, page, rng.random() < 0.5, rng.random() < 0.4))


def _without_name(case):
    del case["name"]
    return case


def _blocks(d):
    return (d + BLOCK - 1) // BLOCK


# ---------------------------------------------------------------- inputs
class _Draw:
    """Tensors from one seeded generator on the GPU, in the order they are asked for."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, shape, dtype="f32", std=1.0):
        return torch.randn(shape, generator=self.g, device="cuda").mul_(std).to(TORCH[dtype])

    def order(self, count):
        return torch.randperm(count, generator=self.g, device="cuda")


def _spread(case, most):
    """Numbers up to `most`, one a sequence, in ascending order."""
    n = case["n"]
    if not case["ragged"]:
        return [most] * n
    return [most * i // (n - 1) for i in range(n)] if n >= 3 else [most * (i + 1) // n for i in range(n)]


def _numbers(values, order):
    return torch.tensor(values, dtype=torch.int32, device="cuda")[order].contiguous()


def _states(r, case, t):
    """Keys and values of t tokens as halves of a projection's rows; keys have a few channels far larger than the others."""
    n, hk, d = case["n"], case["hk"], case["d"]
    kv = r.normal((n, t, 2, hk, d), case["dtype"])
    kv[:, :, 0] *= (1.0 + 7.0 * (r.normal((hk, d)) > 2.0)).to(kv.dtype)
    return kv


def prepare(case, seed):
    r = _Draw(seed)
    s = {"case": case}
    n, hk, d, page = (case[k] for k in ("n", "hk", "d", "page"))
    attend = case["op"] == "attend"
    order, other = r.order(n), r.order(n)
    if attend:
        new, have = case["tk"], _spread(case, case["tk"])
        s["lens"] = _numbers(have, order)
        # the queries of a padded batch: as many as there are tokens, where they are the last ones
        s["counts"] = torch.clamp(s["lens"], max=case["tq"]) if case["ragged"] and case["causal"] else None
        first = torch.zeros(n, dtype=torch.int32, device="cuda")
        stored = s["lens"]
    else:
        new = case["t"]
        s["counts"] = _numbers(_spread(case, new), order) if case["ragged"] and new > 1 else None
        first = s["first"] = _numbers(_spread(case, case["before"]), other)
        stored = s["counts"]
    most = new if attend else new + case["before"]
    per = (most + page - 1) // page
    pool = n * per + 3
    s["table"] = r.order(pool)[:n * per].to(torch.int32).reshape(n, per).contiguous()
    s["kv"] = _states(r, case, new)
    if own:
        from paper_2602_00608_amd import wmdec
        s["cache"] = wmdec.Cache(torch.empty((pool, wmdec.cache_page_bytes(page, hk, d)), dtype=torch.uint8, device="cuda"), page, hk, d)
        if case["op"] != "store":
            wmdec.cache_write(s["kv"][:, :, 0], s["kv"][:, :, 1], s["cache"], s["table"], first, stored)
    else:
        s["codes"] = torch.zeros((2, pool * page, hk, _blocks(d) * BLOCK // 2), dtype=torch.uint8, device="cuda")
        s["exponents"] = torch.zeros((2, pool * page, hk, _blocks(d)), dtype=torch.int8, device="cuda")
        if case["op"] != "store":
            _plain_write(s, first, stored)
    if case["op"] != "store":
        s["kv"] = None
    if attend:
        s["q"] = r.normal((n, case["tq"], case["hq"], d), case["dtype"])
        s["scale"] = 1.0 / math.sqrt(d)
        s["o"] = torch.zeros_like(s["q"])
        if own:
            s["ws"] = torch.empty(max(wmdec.cache_attention_workspace_bytes(s["q"], s["cache"], case["tk"]), 16), dtype=torch.uint8, device="cuda")
    else:
        s["out"] = [torch.zeros((n, new, hk, d), dtype=TORCH[case["dtype"]], device="cuda") for _ in range(2)]
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    if own:
        return {"store": _own_store, "read": _own_read, "attend": _own_attend}[state["case"]["op"]](state)
    return {"store": _plain_store, "read": _plain_read, "attend": _plain_attend}[state["case"]["op"]](state)


def _own_store(s):
    from paper_2602_00608_amd import wmdec
    wmdec.cache_write(s["kv"][:, :, 0], s["kv"][:, :, 1], s["cache"], s["table"], s["first"], s["counts"])
    wmdec.cache_read(s["cache"], s["table"], s["out"][0], s["out"][1], s["first"], s["counts"])
    return s["out"]


def _own_read(s):
    from paper_2602_00608_amd import wmdec
    wmdec.cache_read(s["cache"], s["table"], s["out"][0], s["out"][1], s["first"], s["counts"])
    return s["out"]


def _own_attend(s):
    from paper_2602_00608_amd import wmdec
    wmdec.cache_attention(s["q"], s["cache"], s["table"], s["lens"], s["o"], s["scale"], s["case"]["tk"], causal=s["case"]["causal"], counts=s["counts"], workspace=s["ws"])
    return s["o"]


def _places(s, first, t):
    """[n, t]: rows of the pool that t tokens from first on have."""
    page = s["case"]["page"]
    at = first[:, None].long() + torch.arange(t, device="cuda")
    at = at.clamp(max=s["table"].shape[1] * page - 1)   # (past a sequence's end: not used)
    return torch.gather(s["table"].long(), 1, at // page) * page + at % page


def _power(e):
    """2^e to the bit, -126 <= e <= 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _plain_quantise(x, highest):
    """x [..., channels] -> codes, two a byte, and exponents of its blocks."""
    d = x.shape[-1]
    x = torch.nn.functional.pad(x.float(), (0, _blocks(d) * BLOCK - d)).unflatten(-1, (_blocks(d), BLOCK))
    fraction, power = torch.frexp(x.abs().amax(-1))                     # a fraction of 0.5 .. 1
    e = (power - 3 + (fraction >= 0.875).int()).clamp(-125, highest)
    scaled = x * _power(-e)[..., None]
    a = scaled.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0) + 8 * (scaled < 0)
    code = code.flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), e.to(torch.int8)


def _plain_values(codes, e, d):
    """Codes and exponents -> float32 [..., d]."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), device="cuda")
    return (table[c].unflatten(-1, (-1, BLOCK)) * _power(e)[..., None]).flatten(-2)[..., :d]


def _plain_write(s, first, counts):
    n, t = s["kv"].shape[:2]
    places = _places(s, first, t)
    if counts is not None:
        there = torch.arange(t, device="cuda")[None] < counts[:, None]
        places = places[there]
    for i in range(2):
        x = s["kv"][:, :, i] if counts is None else s["kv"][:, :, i][there]
        s["codes"][i, places], s["exponents"][i, places] = _plain_quantise(x, 13 if s["case"]["dtype"] == "f16" else 125)


def _plain_store(s):
    _plain_write(s, s["first"], s["counts"])
    return _plain_read(s)


def _plain_read(s):
    n, t, _, d = s["out"][0].shape
    places = _places(s, s["first"], t)
    out = []
    for i in range(2):
        v = _plain_values(s["codes"][i, places], s["exponents"][i, places], d)
        if s["counts"] is not None:
            v = v * (torch.arange(t, device="cuda")[None] < s["counts"][:, None])[:, :, None, None]
        out.append(v.to(s["out"][i].dtype))
    return out


def _plain_attend(s):
    c = s["case"]
    n, tq, tk, hk, d, group = c["n"], c["tq"], c["tk"], c["hk"], c["d"], c["hq"] // c["hk"]
    places = _places(s, torch.zeros_like(s["lens"]), tk)
    key = torch.arange(tk, device="cuda")
    there = key[None] < s["lens"][:, None]
    k, v = (_plain_values(s["codes"][i, places], s["exponents"][i, places], d).masked_fill(~there[:, :, None, None], 0.0) for i in (0, 1))
    counts = s["counts"] if s["counts"] is not None else torch.full_like(s["lens"], tq)
    row = torch.arange(tq, device="cuda")
    last = s["lens"][:, None] - (counts[:, None] - row[None] if c["causal"] else 0 * row[None])   # [n, tq]: keys up to it, or below it
    ok = (key[None, None] <= last[:, :, None]) & there[:, None] if c["causal"] else there[:, None].expand(n, tq, tk)
    ok = ok & (row[None] < counts[:, None])[:, :, None]
    q = s["q"].float().reshape(n, tq, hk, group, d).permute(0, 2, 1, 3, 4).reshape(n, hk, tq * group, d).contiguous()
    score = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * s["scale"]
    score = score.view(n, hk, tq, group, tk).masked_fill_(~ok[:, None, :, None, :], float("-inf")).view(n, hk, tq * group, tk)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v.permute(0, 2, 1, 3).contiguous()) / torch.where(total == 0, torch.ones_like(total), total)
    return o.view(n, hk, tq, group, d).permute(0, 2, 1, 3, 4).reshape(n, tq, hk * group, d).to(s["q"].dtype)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    held = case["hk"] * _blocks(case["d"]) * (BLOCK // 2 + 1) * 2          # bytes of a token's keys and values in the cache
    if case["op"] != "attend":
        tokens = sum(_spread(case, case["t"])) if case["t"] > 1 else case["n"]
        dense = tokens * case["hk"] * case["d"] * 2 * SIZE[case["dtype"]]
        return {"bytes": tokens * held + dense * (2 if case["op"] == "store" else 1), "flops": tokens * case["hk"] * case["d"] * (8 if case["op"] == "store" else 2)}
    tq, rows, pairs = case["tq"], 0, 0
    lens = _spread(case, case["tk"])
    for length in lens:
        count = min(length, tq) if case["ragged"] and case["causal"] else tq
        rows += count
        pairs += sum(max(0, length - count + i + 1) for i in range(count)) if case["causal"] else count * length
    return {"bytes": sum(lens) * held + 2 * rows * case["hq"] * case["d"] * SIZE[case["dtype"]], "flops": 4 * pairs * case["hq"] * case["d"]}


# ---------------------------------------------------------------- from the definitions, in 64 bits
def exact(case, seed):
    """The states are drawn again; where their tokens lie does not matter to what comes out."""
    r = _Draw(seed)
    n, hk, d, page = (case[k] for k in ("n", "hk", "d", "page"))
    attend = case["op"] == "attend"
    order = r.order(n).tolist()
    r.order(n)
    new = case["tk"] if attend else case["t"]
    most = new if attend else new + case["before"]
    ascending = _spread(case, new)
    count = [ascending[i] if attend or new > 1 else new for i in order]
    r.order(n * ((most + page - 1) // page) + 3)
    kv = _states(r, case, new)
    if not attend:
        out = [torch.zeros((n, new, hk, d), dtype=torch.float64, device="cuda") for _ in range(2)]
        for b in range(n):
            for i in range(2):
                out[i][b, :count[b]] = _exact_held(kv[b, :count[b], i], case["dtype"])
        return out
    q = r.normal((n, case["tq"], case["hq"], d), case["dtype"]).double()
    out, group = torch.zeros_like(q), case["hq"] // hk
    for b in range(n):
        length = count[b]
        queries = min(length, case["tq"]) if case["ragged"] and case["causal"] else case["tq"]
        if length == 0 or queries == 0:
            continue
        for h in range(hk):
            k, v = (_exact_held(kv[b, :length, i, h], case["dtype"]) for i in (0, 1))
            for g in range(h * group, (h + 1) * group):
                score = (q[b, :queries, g] @ k.t()) / math.sqrt(d)
                if case["causal"]:
                    place = torch.arange(length - queries, length, device="cuda")
                    score[torch.arange(length, device="cuda")[None, :] > place[:, None]] = -math.inf
                seen = score.max(-1, keepdim=True).values > -math.inf
                weight = torch.exp(score - torch.where(seen, score.max(-1, keepdim=True).values, 0.0))
                out[b, :queries, g] = (weight @ v) / torch.where(seen, weight.sum(-1, keepdim=True), 1.0)
    return out


def _exact_power(e):
    return ((e + 1023) << 52).view(torch.float64)


def _exact_held(x, dtype):
    """What the cache holds of x [..., channels], from the definition: the nearest of the sixteen values, block by block."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    grid = torch.tensor(VALUES, dtype=torch.float64, device=x.device)
    for at in range(0, x.shape[-1], BLOCK):
        part = x[..., at:at + BLOCK].double()
        largest = part.abs().max(-1, keepdim=True).values
        power = torch.floor(torch.log2(torch.clamp(largest, min=2.0 ** -140))).long()
        power = torch.where(_exact_power(power) > largest, power - 1, power)             # (a logarithm that was rounded up, or down, to a whole number)
        power = torch.where(_exact_power(power + 1) <= largest, power + 1, power)
        power = torch.where(largest >= 1.75 * _exact_power(power), power + 1, power)
        unit = _exact_power(torch.clamp(power - 2, -125, 13 if dtype == "f16" else 125))
        a = part.abs() / unit
        below = torch.searchsorted(grid, a.contiguous(), right=True) - 1                # the last value that is not above
        above = torch.clamp(below + 1, max=7)
        down, up = a - grid[below], grid[above] - a
        place = torch.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)
        out[..., at:at + BLOCK] = torch.copysign(grid[place], part) * unit
    return out
