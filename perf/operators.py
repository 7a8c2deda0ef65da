"""Rows in 8 bits, as timed cases: the residual's addition with a root-mean-square norm in front of an 8-bit product, rows made
into 8-bit codes with a scale each, the product of 8-bit integers with a scale for each row and each channel, and a run of
them together.

A row's codes are whole numbers from -127 to 127 that stand for code * scale; they lie in rows of whole 128-byte lines.  Codes
that an operator gives are returned as the values they stand for, in bf16 as a layer behind them would read them.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6


def listed():
    return [
        # one row through the norm: a single token or a single region's features, where launches and latency are all there is
        {"name": "norm-1x2048", "kind": "norm", "rows": 1, "k": 2048, "type": "bf16", "residual": True},
        # 32 frames' regions between the two wide layers of the box head
        {"name": "norm-9600x1024", "kind": "norm", "rows": 9600, "k": 1024, "type": "bf16", "residual": True},
        # a long batch of wide rows
        {"name": "norm-8192x8192", "kind": "norm", "rows": 8192, "k": 8192, "type": "bf16", "residual": True},
        # single precision, odd everywhere: rows that start on odd addresses; no residual
        {"name": "norm-odd-fp32", "kind": "norm", "rows": 1237, "k": 2047, "type": "fp32", "residual": False},
        # one frame's region features in front of the first wide layer (300 regions of 7 x 7 x 256)
        {"name": "quantize-300x12544", "kind": "quantize", "rows": 300, "k": 12544, "type": "bf16"},
        # 32 frames' region features
        {"name": "quantize-9600x12544", "kind": "quantize", "rows": 9600, "k": 12544, "type": "bf16"},
        # one row through a square layer: the weights are all there is to read
        {"name": "linear-1x4096x4096", "kind": "linear", "rows": 1, "k": 4096, "n": 4096, "type": "bf16", "relu": False, "residual": False},
        # the first wide layer of the box head for one frame and for 32
        {"name": "linear-300x12544x1024", "kind": "linear", "rows": 300, "k": 12544, "n": 1024, "type": "bf16", "relu": True, "residual": False},
        {"name": "linear-9600x12544x1024", "kind": "linear", "rows": 9600, "k": 12544, "n": 1024, "type": "bf16", "relu": True, "residual": False},
        # class and box predictors of 20 classes behind 8 full-HD frames: few, odd channels, results in fp32
        {"name": "linear-8000x1024x100-fp32", "kind": "linear", "rows": 8000, "k": 1024, "n": 100, "type": "fp32", "relu": False, "residual": False},
        # the largest product
        {"name": "linear-8192x8192x8192", "kind": "linear", "rows": 8192, "k": 8192, "n": 8192, "type": "bf16", "relu": False, "residual": True},
        # all together: norm, product, ReLU, codes again, product back onto the residual
        {"name": "block-4096x1024x4096", "kind": "block", "rows": 4096, "k": 1024, "n": 4096, "type": "bf16"},
    ]


def _between(rng, low, high):
    """A whole number from low to high, spread over its logarithm."""
    return min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    kind = rng.choices(["norm", "quantize", "linear", "block"], [4, 3, 6, 2])[0]
    type_ = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if kind in ("norm", "quantize"):
        k = _between(rng, 16, 12544 if kind == "quantize" else 8192)
        rows = _between(rng, 1, min(16384, (1 << 26 if kind == "norm" else 9600 * 12544) // (k * (1 if type_ == "bf16" else 2))))
        case = {"kind": kind, "rows": rows, "k": k, "type": type_}
        return dict(case, residual=rng.random() < 0.7) if kind == "norm" else case
    if kind == "block":
        k = _between(rng, 64, 1024)
        return {"kind": kind, "rows": _between(rng, 1, 4096), "k": k, "n": _between(rng, k, 4 * k), "type": "bf16"}
    k, n = _between(rng, 16, 12544), _between(rng, 8, 8192)
    if rng.random() < 0.5:   # layers are mostly round
        k, n = -(-k // 64) * 64, -(-n // 64) * 64
    rows = _between(rng, 1, min(16384, 8192 ** 3 // (k * n)))
    return {"kind": kind, "rows": rows, "k": k, "n": n, "type": type_, "relu": rng.random() < 0.5, "residual": rng.random() < 0.3}


def _pitch(k):
    return -(-k // 128) * 128


def _codes(rng, rows, k):
    """Codes as normal values give them (the largest of a row near four deviations), rows and scales like a quantised batch's."""
    codes = torch.zeros((rows, _pitch(k)), dtype=torch.int8, device="cuda")
    codes[:, :k] = (torch.randn((rows, k), generator=rng, device="cuda", dtype=torch.bfloat16) * 32).round_().clamp_(-127, 127)
    scales = torch.empty(rows, device="cuda").uniform_(0.5, 2.0, generator=rng) * (4 / 127)
    return codes, scales


def _rows(rng, rows, k, type_, bump=True):
    """Activations: normal, rows of different size, a few columns that stand out."""
    x = torch.randn((rows, k), generator=rng, device="cuda", dtype=TYPES[type_])
    x *= torch.empty((rows, 1), device="cuda").uniform_(0.5, 2.0, generator=rng).to(x.dtype)
    if bump and k >= 64:
        x[:, torch.randint(k, (k // 64,), generator=rng, device="cuda")] *= 3
    return x


def _weights(rng, n, k):
    codes, scales = _codes(rng, n, k)
    return {"codes": codes[:, :k].contiguous(), "scales": scales * (32 / 4) / math.sqrt(k) / 8, "bias": 0.1 * torch.randn(n, generator=rng, device="cuda")}


def _layer(w):
    import paper_2102_08481_amd as thia
    return thia.thia_linear_i8_load_codes(w["codes"], w["scales"], w["bias"])


def prepare(case, seed):
    rng = torch.Generator(device="cuda")
    rng.manual_seed(seed)
    kind, rows, k = case["kind"], case["rows"], case["k"]
    s = {"case": case}
    if kind == "linear":
        s["codes"], s["scales"] = _codes(rng, rows, k)
        s["w"] = _weights(rng, case["n"], k)
        s["residual"] = _rows(rng, rows, case["n"], case["type"], False) if case["residual"] else None
    else:
        s["x"] = _rows(rng, rows, k, case["type"])
    if kind == "block":
        s["w1"], s["w2"] = _weights(rng, case["n"], k), _weights(rng, k, case["n"])
    if kind in ("norm", "block"):
        s["residual"] = _rows(rng, rows, k, case["type"]) if case.get("residual", True) else None
        s["gain"] = torch.empty(k, device="cuda").uniform_(0.5, 1.5, generator=rng)
    if own:   # the layers that a program keeps
        for name in ("w", "w1", "w2"):
            if name in s:
                s["layer_" + name] = _layer(s[name])
    return s


# ---------------------------------------------------------------- the plain forms
def _quantize(y):
    """fp32 rows -> (codes, scales); a row of zeros has scale 0."""
    scale = y.abs().amax(1, keepdim=True) / 127
    codes = torch.round(y / torch.where(scale > 0, scale, torch.ones_like(scale))).clamp(-127, 127)
    return codes, scale


def _norm(x, residual, gain):
    h = x.float()
    if residual is not None:
        h = h + residual.float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * gain
    return (h.to(x.dtype) if residual is not None else None,) + _quantize(y)


def _linear(codes, scale, w, relu, residual, dtype):
    # sums of products of codes stay below 2^24 in all but absurd cases, where fp32 holds every whole number
    out = (codes.float() @ w["codes"].float().T) * scale * w["scales"] + w["bias"]
    if residual is not None:
        out = out + residual.float()
    return (torch.clamp(out, min=0) if relu else out).to(dtype)


def _values(codes, scales):
    """What codes stand for, in bf16: one product of whole numbers and fp32 scales, rounded once."""
    return torch.mul(codes, scales.unsqueeze(1), out=torch.empty(codes.shape, dtype=torch.bfloat16, device=codes.device))


def run(s):
    c = s["case"]
    kind, k = c["kind"], c["k"]
    if own:
        import paper_2102_08481_amd as thia
        if kind == "norm":
            codes, scales, total = thia.thia_rms_norm_i8(s["x"], s["gain"], EPS, s["residual"])
            return {"values": _values(codes[:, :k], scales), "scales": scales, "sum": total}
        if kind == "quantize":
            codes, scales = thia.thia_quantize_rows(s["x"])
            return {"values": _values(codes[:, :k], scales), "scales": scales}
        if kind == "linear":
            return {"out": thia.thia_linear_i8_run(s["layer_w"], s["codes"], s["scales"], relu=c["relu"], residual=s["residual"], out_f32=c["type"] == "fp32")}
        codes, scales, total = thia.thia_rms_norm_i8(s["x"], s["gain"], EPS, s["residual"])
        u = thia.thia_linear_i8_run(s["layer_w1"], codes, scales, relu=True)
        codes, scales = thia.thia_quantize_rows(u)
        return {"out": thia.thia_linear_i8_run(s["layer_w2"], codes, scales, residual=total), "sum": total}
    if kind == "norm":
        total, codes, scale = _norm(s["x"], s["residual"], s["gain"])
        return {"values": (codes * scale).bfloat16(), "scales": scale[:, 0], "sum": total}
    if kind == "quantize":
        codes, scale = _quantize(s["x"].float())
        return {"values": (codes * scale).bfloat16(), "scales": scale[:, 0]}
    if kind == "linear":
        return {"out": _linear(s["codes"][:, :k], s["scales"][:, None], s["w"], c["relu"], s["residual"], TYPES[c["type"]])}
    total, codes, scale = _norm(s["x"], s["residual"], s["gain"])
    u = _linear(codes, scale, s["w1"], True, None, torch.bfloat16)
    codes, scale = _quantize(u.float())
    return {"out": _linear(codes, scale, s["w2"], False, total, torch.bfloat16), "sum": total}


# ---------------------------------------------------------------- work
def work(case):
    rows, k, size = case["rows"], case["k"], 2 if case["type"] == "bf16" else 4
    if case["kind"] == "quantize":
        return {"bytes": rows * (k * (size + 1) + 4), "flops": 3 * rows * k}
    norm = rows * (k * (size * (3 if case.get("residual", True) else 1) + 1) + 4) + 4 * k
    if case["kind"] == "norm":
        return {"bytes": norm, "flops": 6 * rows * k}
    n = case["n"]
    if case["kind"] == "linear":
        return {"bytes": rows * (k + 4) + n * (k + 8) + rows * n * size * (2 if case["residual"] else 1), "flops": 2 * rows * k * n}
    # the block: both inputs once, both weights, the sum and the result
    return {"bytes": rows * k * 2 * 4 + 2 * n * k + 4 * (2 * n + 3 * k), "flops": 4 * rows * k * n}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    kind, k = case["kind"], case["k"]

    def to_codes(v):
        step = v.abs().max(dim=1).values / 127.0
        held = torch.zeros_like(v)
        some = step > 0
        held[some] = torch.round(v[some] / step[some].unsqueeze(1))
        return held, step

    def product(q, step, w, onto=None):
        r = torch.matmul(q, w["codes"].double().t().contiguous()) * torch.outer(step, w["scales"].double()) + w["bias"].double().unsqueeze(0)
        return r if onto is None else r + onto.double()

    if kind == "linear":
        r = product(s["codes"][:, :k].double(), s["scales"].double(), s["w"], s["residual"])
        return {"out": r.relu() if case["relu"] else r}
    v, total = s["x"].double(), None
    if kind != "quantize":
        if s["residual"] is not None:
            v = total = v + s["residual"].double()
        v = v / torch.sqrt(v.pow(2).sum(dim=1, keepdim=True) / k + EPS) * s["gain"].double()
    q, step = to_codes(v)
    if kind != "block":
        out = {"values": q * step.unsqueeze(1), "scales": step}
        return dict(out, sum=total) if kind == "norm" else out
    # between the layers, and as the residual, rows are held in bf16
    u = product(q, step, s["w1"]).relu().bfloat16()
    q, step = to_codes(u.double())
    return {"out": product(q, step, s["w2"], total.bfloat16()), "sum": total}
