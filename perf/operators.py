"""The operators of a transformer block that stand around its AdaLN projections, as cases to be timed: the gated residual
with the norms before and after it, rotary positions, and attention to states of another length.

Sizes: 5400 tokens are the 60x90 latent of a 480x720 frame, 1920 = 30 heads of 64 channels is the width that the AdaLN
projections are tested and timed at; the others are generic.  Where `own` is false every operator runs in its plain form, in
32-bit torch operations (angles in 64 bits), rounded once at the end; where it is true through the library's entry points.
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def listed():
    return [
        # one token of a stream that advances token by token: shift and scale in front of a block; latency
        _norm("norm_1_1920_bf16", "bf16", "bf16", 1, 1, 1920, "none", "layer", False, True, True),
        # between the attention and the MLP of a block, one frame and its unconditional twin
        _norm("norm_2x5400_1920_bf16", "bf16", "bf16", 2, 5400, 1920, "none", "layer", True, True, True),
        # a block with norms on both sides over a residual stream in fp32, four frames: the most bytes
        _norm("norm_4x5400_1152_f32_f16", "f32", "f16", 4, 5400, 1152, "rms", "rms", True, True, True),
        # the last residual of a stack of an odd width on a padded prompt
        _norm("norm_3x77_1001_f16", "f16", "f16", 3, 77, 1001, "layer", "none", True, False, False),
        # one token
        _rope("rope_1_30x64_bf16", "bf16", 1, 1, 30, 30, 64, 64, 1, True, "none", 1.0),
        # the tokens of a frame and its twin, placed by frame, row and column
        _rope("rope_2x5400_30x64_3axes_bf16", "bf16", 2, 5400, 30, 30, 64, 64, 3, True, "none", 1.0),
        # a long stretch of context past the trained length, grouped heads, three quarters of the head rotated
        _rope("rope_16385_32_8x128_half_f16", "f16", 1, 16385, 32, 8, 128, 96, 1, False, "ramp", 8.0),
        # one token against a short conditioning
        _cross("cross_1x77_30x64_bf16", "bf16", 2, 1, 77, 30, 30, 64, False, False),
        # one token of four streams against long states of different lengths, grouped heads
        _cross("cross_1x32768_32_8x128_bf16", "bf16", 4, 1, 32768, 32, 8, 128, True, False),
        # the tokens of a frame and its twin against conditioning of two lengths
        _cross("cross_5400x512_30x64_bf16", "bf16", 2, 5400, 512, 30, 30, 64, True, False),
        # a frame against the frame before it: the most arithmetic
        _cross("cross_5400x5400_30x64_f16", "f16", 1, 5400, 5400, 30, 30, 64, False, False),
        # a sensitive layer in fp32, a head of an odd multiple of eight, padding anywhere and a sample with nothing to see
        _cross("cross_333x301_8x72_f32", "f32", 3, 333, 301, 8, 8, 72, True, True),
    ]


def _norm(name, x, act, n, t, d, post, pre, residual, y, mod):
    """post, pre: the norms of the block's result and of the residual; residual: there is a block's result; y: the normalised
    residual is wanted; mod: gate, shift and scale are there."""
    return {"name": name, "op": "norm", "x": x, "act": act, "n": n, "t": t, "d": d, "post": post, "pre": pre, "residual": residual, "y": y, "mod": mod}


def _rope(name, dtype, n, t, hq, hk, d, rot, axes, interleaved, scaling, factor):
    return {"name": name, "op": "rope", "dtype": dtype, "n": n, "t": t, "hq": hq, "hk": hk, "d": d, "rot": rot, "axes": axes, "interleaved": interleaved,
            "scaling": scaling, "factor": factor}


def _cross(name, dtype, n, tq, tk, hq, hk, d, ragged, masked):
    """ragged: samples have key counts of their own (with three samples or more one has none); masked: a fifth of the keys is masked."""
    return {"name": name, "op": "cross", "dtype": dtype, "n": n, "tq": tq, "tk": tk, "hq": hq, "hk": hk, "d": d, "ragged": ragged, "masked": masked}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, of no more work than the largest listed one of its operator."""
    op = rng.choice(["norm", "rope", "cross", "cross"])
    if op == "norm":
        x, act = rng.choice([("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("f32", "bf16"), ("f32", "f16")])
        n, d = rng.choice([1, 1, 2, 3, 4]), rng.choice([8, 2, 1]) * _log(rng, 32, 512)
        t = min(_log(rng, 1, 21600), 4 * 5400 * 1152 * 12 // (n * d * (2 * SIZE[x] + 2 * SIZE[act])))
        residual = rng.random() < 0.75
        y = not residual or rng.random() < 0.8
        return _without_name(_norm("", x, act, n, max(t, 1), d, rng.choice(["none", "layer", "rms"]) if residual else "none",
                                   rng.choice(["layer", "rms"]) if y else "none", residual, y, rng.random() < 0.8))
    if op == "rope":
        hk, group = rng.choice([1, 2, 5, 8, 30]), rng.choice([1, 1, 2, 4])
        d = rng.choice([32, 64, 64, 72, 96, 128, 128, 256])
        rot = rng.choice([d, d, d // 8 * 4, 8])
        axes = rng.choice([1, 1, 2, 3]) if rot >= 24 else 1
        n = rng.choice([1, 1, 2, 3])
        dtype = rng.choice(["bf16", "f16", "f32"])
        t = min(_log(rng, 1, 20000), 16384 * 40 * 128 * 2 // (n * hk * (group + 1) * d * SIZE[dtype]))
        scaling = rng.choice(["none", "linear", "base", "ramp"]) if axes == 1 else "none"
        return _without_name(_rope("", dtype, n, max(t, 1), hk * group, hk, d, rot, axes, rng.random() < 0.5, scaling,
                                   round(rng.uniform(1.5, 32.0), 2) if scaling != "none" else 1.0))
    dtype = rng.choice(["bf16", "bf16", "f16", "f16", "f32"])
    hk, group = rng.choice([1, 2, 8, 10, 30]), rng.choice([1, 1, 2, 4, 7])
    d = rng.choice([32, 64, 64, 72, 96, 128, 128, 160, 256])
    n = rng.choice([1, 1, 2, 3, 4])
    tq, tk = (rng.choice([1, 1, 2, 5]) if rng.random() < 0.4 else _log(rng, 8, 8000)), _log(rng, 1, 32768)
    # queries and keys are cut to the reading of the longest listed states, keys to the arithmetic (a twelfth of it in fp32) of two frames as well
    states = 32768 * 8 * 128 * 2 * 2 // (n * hk * d * SIZE[dtype])
    tq = max(1, min(tq, states // group))
    tk = min(tk, states, 5400 * 5400 * 30 * 64 // (n * tq * hk * group * d * (12 if dtype == "f32" else 1)))
    return _without_name(_cross("", dtype, n, tq, max(tk, 1), hk * group, hk, d, rng.random() < 0.5, rng.random() < 0.3))


def _without_name(case):
    del case["name"]
    return case


# ---------------------------------------------------------------- inputs
class _Draw:
    """Tensors from one seeded generator on the GPU, in the order they are asked for."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, shape, dtype="f32", std=1.0, mean=0.0):
        return torch.randn(shape, generator=self.g, device="cuda").mul_(std).add_(mean).to(TORCH[dtype])

    def below(self, high, shape):
        return torch.randint(0, high, shape, generator=self.g, device="cuda", dtype=torch.int32)


def prepare(case, seed):
    return {"norm": _prepare_norm, "rope": _prepare_rope, "cross": _prepare_cross}[case["op"]](case, _Draw(seed))


def _prepare_norm(case, r):
    n, t, d = case["n"], case["t"], case["d"]
    s = {"case": case}
    # a residual stream has a few channels far larger than the others
    s["x"] = (r.normal((n, t, d)) * (1.0 + 20.0 * (r.normal((d,)) > 2.5))).to(TORCH[case["x"]])
    s["h"] = r.normal((n, t, d), case["act"], 0.7) if case["residual"] else None
    for which in ("post", "pre"):
        kind = case[which]
        s[which] = (kind, EPS, r.normal((d,), std=0.2, mean=1.0) if kind != "none" else None, r.normal((d,), std=0.1) if kind == "layer" else None)
    # shift, scale and gate as the AdaLN projections leave them: thirds of one row a sample
    s["mod"] = r.normal((n, 3 * d), std=0.3) if case["mod"] else None
    s["res_scale"] = 0.9
    s["x_out"] = torch.empty_like(s["x"]) if case["residual"] else None
    s["y"] = torch.empty((n, t, d), dtype=TORCH[case["act"]], device="cuda") if case["y"] else None
    return s


def _axis_dims(rot, axes):
    """Channels of the axes: even parts, what is left over at the first."""
    part = rot // axes // 2 * 2
    return [rot - part * (axes - 1)] + [part] * (axes - 1)


BASE, TRAINED, LOW, HIGH = 10000.0, 2048, 1.0, 4.0


def _prepare_rope(case, r):
    n, t, hq, hk, d, axes = (case[k] for k in ("n", "t", "hq", "hk", "d", "axes"))
    s = {"case": case, "dims": _axis_dims(case["rot"], axes)}
    s["q"], s["k"] = r.normal((n, t, hq, d), case["dtype"]), r.normal((n, t, hk, d), case["dtype"])
    if axes == 1:      # consecutive tokens, from anywhere in a long context
        s["positions"] = (r.below(1 << 17, (n, 1)) + torch.arange(t, device="cuda", dtype=torch.int32)).reshape(n, t, 1).contiguous()
    else:              # frame, row, column of a latent 90 wide
        i = torch.arange(t, device="cuda", dtype=torch.int32)
        place = [r.below(1000, (1,)).expand(t), i // 90, i % 90][-axes:]
        s["positions"] = torch.stack(place, -1).expand(n, t, axes).contiguous()
    s["freq"] = torch.empty(case["rot"] // 2, dtype=torch.float64, device="cuda")
    if own:
        from paper_2602_00608_amd import wmdec
        wmdec.rope_frequencies(s["dims"], s["freq"], base=BASE, scaling=case["scaling"], factor=case["factor"], trained_length=TRAINED, low_turns=LOW, high_turns=HIGH)
    else:
        at = 0
        for dim in s["dims"]:
            j = torch.arange(dim // 2, device="cuda", dtype=torch.float64)
            base = BASE * case["factor"] ** (dim / (dim - 2)) if case["scaling"] == "base" else BASE
            f = torch.exp(-2.0 * j / dim * math.log(base))
            if case["scaling"] == "linear":
                f = f / case["factor"]
            if case["scaling"] == "ramp":
                w = ((TRAINED * f / (2.0 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
                f = f * (w + (1.0 - w) / case["factor"])
            s["freq"][at:at + dim // 2] = f
            at += dim // 2
    s["magnitude"] = 1.0 + 0.1 * math.log(case["factor"]) if case["scaling"] == "ramp" else 1.0
    s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    return s


def _lengths(case):
    """Keys that the samples have, in ascending order."""
    n, tk = case["n"], case["tk"]
    if not case["ragged"]:
        return [tk] * n
    return [tk * i // (n - 1) for i in range(n)] if n >= 3 else [tk * (i + 1) // n for i in range(n)]


def _prepare_cross(case, r):
    n, tq, tk, hq, hk, d = (case[k] for k in ("n", "tq", "tk", "hq", "hk", "d"))
    dt = case["dtype"]
    s = {"case": case}
    s["q"] = r.normal((n, tq, hq, d), dt, 1.5)
    # keys and values as one projection of the states leaves them: halves of a row
    s["kv"] = r.normal((n, tk, 2, hk, d), dt)
    lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    s["lens"] = lens[torch.randperm(n, generator=r.g, device="cuda")].contiguous() if case["ragged"] else None
    s["mask"] = (torch.rand((n, tk), generator=r.g, device="cuda") < 0.8).contiguous() if case["masked"] else None
    s["scale"] = 1.0 / math.sqrt(d)
    s["o"] = torch.empty_like(s["q"])
    if own:
        from paper_2602_00608_amd import wmdec
        s["ws"] = torch.empty(max(wmdec.cross_attention_workspace_bytes(s["q"], s["kv"][:, :, 0]), 16), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    if own:
        return {"norm": _own_norm, "rope": _own_rope, "cross": _own_cross}[state["case"]["op"]](state)
    return {"norm": _plain_norm, "rope": _plain_rope, "cross": _plain_cross}[state["case"]["op"]](state)


def _thirds(s):
    d = s["case"]["d"]
    m = s["mod"]
    return (None, None, None) if m is None else (m[:, :d], m[:, d:2 * d], m[:, 2 * d:])


def _own_norm(s):
    from paper_2602_00608_amd import wmdec
    shift, scale, gate = _thirds(s)
    residual = s["h"] is not None
    wmdec.residual_norm(s["x"], s["h"], wmdec.Norm(*s["post"]), gate if residual else None, s["res_scale"] if residual else 1.0, s["x_out"],
                        wmdec.Norm(*s["pre"]), scale if s["y"] is not None else None, shift if s["y"] is not None else None, s["y"])
    return [o for o in (s["x_out"], s["y"]) if o is not None]


def _own_rope(s):
    from paper_2602_00608_amd import wmdec
    wmdec.rope(s["q"], s["k"], s["positions"], s["freq"], s["dims"], s["q_out"], s["k_out"], interleaved=s["case"]["interleaved"], magnitude=s["magnitude"])
    return [s["q_out"], s["k_out"]]


def _own_cross(s):
    from paper_2602_00608_amd import wmdec
    wmdec.cross_attention(s["q"], s["kv"][:, :, 0], s["kv"][:, :, 1], s["o"], s["scale"], key_lens=s["lens"], key_mask=s["mask"], workspace=s["ws"])
    return s["o"]


def _norm_of(v, spec):
    kind, eps, w, u = spec
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps)
    if w is not None:
        v = v * w
    return v if u is None else v + u


def _plain_norm(s):
    shift, scale, gate = _thirds(s)
    out, x = [], s["x"]
    if s["h"] is not None:
        b = _norm_of(s["h"].float(), s["post"])
        if gate is not None:
            b = b * gate[:, None, :]
        x = (x.float() + s["res_scale"] * b).to(x.dtype)     # what the stream holds is what is normalised
        out.append(x)
    if s["y"] is not None:
        y = _norm_of(x.float(), s["pre"])
        if scale is not None:
            y = y * (1.0 + scale[:, None, :]) + shift[:, None, :]
        out.append(y.to(s["y"].dtype))
    return out


def _plain_rope(s):
    axis = torch.repeat_interleave(torch.arange(len(s["dims"]), device="cuda"), torch.tensor([v // 2 for v in s["dims"]], device="cuda"))
    angle = s["positions"].double()[:, :, axis] * s["freq"]
    cos, sin = (torch.cos(angle) * s["magnitude"]).float()[:, :, None], (torch.sin(angle) * s["magnitude"]).float()[:, :, None]
    out = []
    for v in (s["q"], s["k"]):
        v32 = v.float()
        o, at = v32.clone(), 0
        for dim in s["dims"]:
            part = slice(at, at + dim)
            if s["case"]["interleaved"]:
                first, second = v32[..., part][..., 0::2], v32[..., part][..., 1::2]
            else:
                first, second = v32[..., part][..., :dim // 2], v32[..., part][..., dim // 2:]
            c, n = cos[..., at // 2:(at + dim) // 2], sin[..., at // 2:(at + dim) // 2]
            a, b = first * c - second * n, first * n + second * c
            o[..., part] = torch.stack((a, b), -1).flatten(-2) if s["case"]["interleaved"] else torch.cat((a, b), -1)
            at += dim
        out.append(o.to(v.dtype))
    return out


def _valid(s):
    """[n, tk]: the keys that count."""
    c = s["case"]
    ok = torch.ones((c["n"], c["tk"]), dtype=torch.bool, device="cuda")
    if s["lens"] is not None:
        ok = ok & (torch.arange(c["tk"], device="cuda")[None] < s["lens"][:, None])
    return ok if s["mask"] is None else ok & s["mask"]


def _plain_cross(s):
    c = s["case"]
    group, ok = c["hq"] // c["hk"], _valid(s)
    q = s["q"].float().permute(0, 2, 1, 3).contiguous()
    k, v = (s["kv"][:, :, i].float().masked_fill(~ok[:, :, None, None], 0.0).repeat_interleave(group, 2) for i in (0, 1))
    score = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * s["scale"]
    if s["lens"] is not None or s["mask"] is not None:
        score.masked_fill_(~ok[:, None, None, :], float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(torch.isinf(top) & (top < 0), torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v.permute(0, 2, 1, 3).contiguous()) / torch.where(total == 0, torch.ones_like(total), total)
    return o.permute(0, 2, 1, 3).to(s["q"].dtype).contiguous()


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "norm":
        e = case["n"] * case["t"] * case["d"]
        passes = e * SIZE[case["x"]] * (2 if case["residual"] else 1) + e * SIZE[case["act"]] * (int(case["residual"]) + int(case["y"]))
        vectors = case["n"] * case["d"] * 4 * ((int(case["residual"]) + 2 * int(case["y"])) if case["mod"] else 0)
        return {"bytes": passes + vectors, "flops": e * (4 * int(case["residual"]) + 7 * int(case["y"]) + (6 if case["post"] != "none" else 0))}
    if case["op"] == "rope":
        e = case["n"] * case["t"] * (case["hq"] + case["hk"])
        return {"bytes": 2 * e * case["d"] * SIZE[case["dtype"]] + case["n"] * case["t"] * case["axes"] * 4 + case["rot"] * 4, "flops": 3 * e * case["rot"]}
    keys = sum(_lengths(case)) * (0.8 if case["masked"] else 1.0)
    q = case["n"] * case["tq"] * case["hq"] * case["d"]
    return {"bytes": int((2 * q + 2 * keys * case["hk"] * case["d"]) * SIZE[case["dtype"]]), "flops": int(4 * case["tq"] * keys * case["hq"] * case["d"])}


# ---------------------------------------------------------------- from the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "rope": _exact_rope, "cross": _exact_cross}[case["op"]](s)


def _exact_norm(s):
    d = s["case"]["d"]

    def normalise(v, spec):
        kind, eps, w, u = spec
        if kind == "none":
            return v
        mean = v.sum(-1) / d if kind == "layer" else torch.zeros_like(v[..., 0])
        variance = ((v - mean[..., None]) ** 2).sum(-1) / d
        out = (v - mean[..., None]) * ((variance + eps) ** -0.5)[..., None] * w.double()
        return out + u.double() if u is not None else out

    mod = s["mod"].double() if s["mod"] is not None else torch.zeros((s["case"]["n"], 3 * d), dtype=torch.float64, device="cuda")
    gate = mod[:, 2 * d:] if s["mod"] is not None else torch.ones_like(mod[:, :d])
    results, stream = [], s["x"].double()
    if s["h"] is not None:
        stream = stream + s["res_scale"] * gate[:, None] * normalise(s["h"].double(), s["post"])
        results.append(stream)
        stream = stream.to(s["x"].dtype).double()
    if s["y"] is not None:
        results.append(normalise(stream, s["pre"]) * (mod[:, None, d:2 * d] + 1.0) + mod[:, None, :d])
    return results


def _exact_rope(s):
    c = s["case"]
    results = [s["q"].double(), s["k"].double()]
    done = 0
    for axis, dim in enumerate(s["dims"]):
        for j in range(dim // 2):
            base = BASE * c["factor"] ** (dim / (dim - 2)) if c["scaling"] == "base" else BASE
            f = base ** (-2.0 * j / dim)
            if c["scaling"] == "linear":
                f /= c["factor"]
            elif c["scaling"] == "ramp":
                share = min(max((TRAINED * f / (2.0 * math.pi) - LOW) / (HIGH - LOW), 0.0), 1.0)
                f = share * f + (1.0 - share) * f / c["factor"]
            theta = (s["positions"][..., axis].double() * f)[..., None]
            i0, i1 = (done + 2 * j, done + 2 * j + 1) if c["interleaved"] else (done + j, done + j + dim // 2)
            for v in results:
                a, b = v[..., i0].clone(), v[..., i1].clone()
                v[..., i0] = s["magnitude"] * (torch.cos(theta) * a - torch.sin(theta) * b)
                v[..., i1] = s["magnitude"] * (torch.sin(theta) * a + torch.cos(theta) * b)
        done += dim
    return results


def _exact_cross(s):
    c = s["case"]
    out = torch.zeros((c["n"], c["tq"], c["hq"], c["d"]), dtype=torch.float64, device="cuda")
    for i in range(c["n"]):
        count = int(s["lens"][i]) if s["lens"] is not None else c["tk"]
        keep = torch.arange(count, device="cuda")
        if s["mask"] is not None:
            keep = keep[s["mask"][i, :count]]
        if keep.numel() == 0:
            continue
        for h in range(c["hq"]):
            k, v = (s["kv"][i, :, j, h // (c["hq"] // c["hk"])].double()[keep] for j in (0, 1))
            score = s["q"][i, :, h].double() @ k.t() * s["scale"]
            weight = torch.exp(score - score.max(-1, keepdim=True).values)
            out[i, :, h] = (weight @ v) / weight.sum(-1, keepdim=True)
    return out
