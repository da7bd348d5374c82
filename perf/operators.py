"""The calls a user makes to run the matrix products of a language model on low-bit codes, as timed cases: rows of floats to codes
and scales, linear layers on codes with their epilogue, and the same grouped by expert.

Sums of products of codes are integers and exact; what follows them is 32-bit arithmetic, rounded once.  Sizes are generic (powers
of two as hidden sizes, and odd ones).  Outputs are the caller's buffers, as in a serving program.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _quant(name, M, K, bits, signed, dtype):
    return {"name": name, "kind": "quantize", "M": M, "K": K, "bits": bits, "signed": signed, "dtype": dtype}


def _linear(name, M, K, N, p, q, xs, ws, w_store, out, act="none", bias=False, residual=False):
    return {"name": name, "kind": "linear", "M": M, "K": K, "N": N, "p": p, "q": q, "xs": xs, "ws": ws, "w_store": w_store, "out": out,
            "act": act, "bias": bias, "residual": residual}


def _grouped(name, E, T, tail, K, N, p, q, xs, ws, w_store, out, act="none", bias=False, residual=False):
    return {"name": name, "kind": "grouped", "E": E, "T": T, "tail": tail, "K": K, "N": N, "p": p, "q": q, "xs": xs, "ws": ws,
            "w_store": w_store, "out": out, "act": act, "bias": bias, "residual": residual}


def listed():
    return [
        # the hidden state of one new token: the smallest call, all latency
        _quant("quantize_token_4k_s8", 1, 4096, 8, True, "bf16"),
        # the hidden activations of a long prompt between the two products of an MLP
        _quant("quantize_prompt_4k_16k_s8", 4096, 16384, 8, True, "bf16"),
        # unsigned 4-bit codes (what follows a ReLU) of fp32 rows whose size divides nothing
        _quant("quantize_odd_u4", 1733, 5003, 4, False, "f32"),
        # one new token against 4-bit weights, two per byte: the weights are all there is to read
        _linear("token_4k_w4", 1, 4096, 4096, 8, 4, True, True, 4, "bf16"),
        # a few sequences decoded together: the first product of an MLP on 8-bit weights
        _linear("tokens8_4k_16k_w8_silu", 8, 4096, 16384, 8, 8, True, True, 8, "bf16", act="silu", bias=True),
        # a serving batch on 4-bit weights with the residual stream added
        _linear("tokens48_8k_8k_w4_residual", 48, 8192, 8192, 8, 4, True, True, 4, "f16", residual=True),
        # sizes that divide nothing, rows that start anywhere; unsigned 8-bit activations, requantised to unsigned 4-bit codes
        _linear("odd_333_1001_1501_u8_codes", 333, 1001, 1501, 8, 8, False, True, 8, "codes", bias=True),
        # exact sums of 4-bit codes, both sides signed
        _linear("sums_2k_s4", 2048, 2048, 2048, 4, 4, True, True, 8, "sums"),
        # a prompt through the two products of an MLP: 8-bit weights with GELU, then 4-bit weights with the residual
        _linear("prompt_4k_4k_16k_w8_gelu", 4096, 4096, 16384, 8, 8, True, True, 8, "bf16", act="gelu", bias=True),
        _linear("prompt_4k_16k_4k_w4_residual", 4096, 16384, 4096, 8, 4, True, True, 4, "bf16", residual=True),
        # experts while decoding: 128 rows over 64 experts of 4-bit weights, most with one row or two
        _grouped("experts64_decode_w4_silu", 64, 128, 0, 2048, 2048, 8, 4, True, True, 4, "bf16", act="silu"),
        # experts on a prompt: ragged thousands of rows, a padded batch whose last rows belong to none
        _grouped("experts8_prompt_w8", 8, 8192, 37, 4096, 4096, 8, 8, True, True, 8, "bf16", bias=True),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _size(rng, lo, hi, step):
    """A size of the range: a multiple of 128 as hidden sizes are, or any multiple of `step`."""
    v = _log_int(rng, lo, hi)
    step = 128 if v >= 256 and rng.random() < 0.6 else step
    return max(step, v // step * step)


def draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "linear", "grouped"])
    if kind == "quantize":
        M, K = _log_int(rng, 1, 4096), _log_int(rng, 16, 16384)
        signed = rng.random() < 0.7
        return {"kind": kind, "M": M, "K": K, "bits": rng.choice([8, 8, 4, 2, 6] if signed else [8, 4, 4, 1, 2]), "signed": signed,
                "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
    p, q = rng.choice([(8, 8), (8, 8), (8, 4), (8, 4), (4, 4), (4, 4), (2, 2), (5, 3), (8, 1), (7, 2)])
    xs, ws = rng.random() < 0.75, rng.random() < 0.8
    store = q if q in (1, 2, 4) and rng.random() < 0.75 else 8
    out = rng.choice(["bf16", "bf16", "bf16", "f16", "f32", "codes", "sums"])
    real = out in _TYPES
    case = {"kind": kind, "p": p, "q": q, "xs": xs, "ws": ws, "w_store": store, "out": out,
            "act": rng.choice(["none", "none", "relu", "silu", "gelu"]) if real else "none",
            "bias": out != "sums" and rng.random() < 0.4, "residual": real and rng.random() < 0.3}
    K = _size(rng, 64, 16384, 1 if store == 8 else 8 // store)
    N = _size(rng, 64, 16384, 1)
    rows = _log_int(rng, 1, 4096)
    most = (1 << 37) if K % 16 == 0 and N % 16 == 0 else 1 << 34
    if kind == "linear":
        while rows * K * N > most:
            rows = max(1, rows // 2) if rows >= K and rows >= N else rows
            N, K = (max(64, N // 2), K) if N >= K and N > rows else (N, max(64, K // 2 // 128 * 128)) if K > rows else (N, K)
        return {**case, "M": rows, "K": K, "N": N}
    E = rng.choice([2, 4, 8, 16, 32, 60, 64])
    while E * K * N > (1 << 28):
        N, K = (max(64, N // 2), K) if N >= K else (N, max(64, K // 2 // 128 * 128))
    rows = max(1, min(rows, most // (K * N)))
    return {**case, "E": E, "T": rows, "tail": rng.choice([0, 0, 5]), "K": K, "N": N}


def _range(bits, signed):
    return (-(1 << (bits - 1)), (1 << (bits - 1)) - 1) if signed else (0, (1 << bits) - 1)


def _codes(shape, bits, signed, g):
    """Codes as a quantiser leaves them: normal, with a deviation of a quarter of the range's width, clamped; one per byte."""
    lo, hi = _range(bits, signed)
    spread = max(0.5, (hi - lo + 1) / 8)
    v = torch.randn(shape, generator=g, device="cuda").mul_(spread)
    if not signed:
        v = v.abs_()
    v = v.round_().clamp_(lo, hi)
    return v.to(torch.int8 if signed else torch.uint8)


def _to_dense(codes, bits):
    """8 / bits codes per byte along the last axis, the first in the lowest bits, two's complement."""
    per = 8 // bits
    v = (codes.view(torch.uint8) & ((1 << bits) - 1)).reshape(*codes.shape[:-1], -1, per)
    out = v[..., 0].clone()
    for i in range(1, per):
        out |= v[..., i] << (i * bits)
    return out.contiguous()


def _popularity(E):
    """How often experts are chosen: some several times as often as others."""
    w = 1.0 / (np.arange(E) + 0.75 * E)
    return w / w.sum()


def _shift(case):
    """The requantisation that keeps typical sums inside the output codes."""
    lo, hi = _range(case["p"], case["xs"])
    wl, wh = _range(case["q"], case["ws"])
    typical = max(0.5, (hi - lo + 1) / 8) * max(0.5, (wh - wl + 1) / 8) * math.sqrt(case["K"])
    return max(0, int(math.log2(max(1.0, typical / 4))))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": case}
    if case["kind"] == "quantize":
        M, K = case["M"], case["K"]
        x = torch.randn(M, K, generator=g, device="cuda")
        x *= torch.rand(M, 1, generator=g, device="cuda") * 4 + 0.1          # rows of different size
        x[:, int(seed) % K] *= 8.0                                           # a channel with outliers, as hidden states have
        s["x"] = (x if case["signed"] else x.clamp_(min=0)).to(_TYPES[case["dtype"]])
        lo, hi = _range(case["bits"], case["signed"])
        s["lo"], s["hi"] = (lo, hi)
        s["top"] = torch.tensor(float(hi), device="cuda")
        s["codes"] = torch.empty(M, K, dtype=torch.int8 if case["signed"] else torch.uint8, device="cuda")
        s["scale"] = torch.empty(M, device="cuda")
        return s
    grouped = case["kind"] == "grouped"
    rows = case["T"] + case["tail"] if grouped else case["M"]
    lead = (case["E"],) if grouped else ()
    K, N = case["K"], case["N"]
    s["x"] = _codes((rows, K), case["p"], case["xs"], g)
    w = _codes((*lead, N, K), case["q"], case["ws"], g)
    s["w"] = w if case["w_store"] == 8 else _to_dense(w, case["w_store"])
    real = case["out"] in _TYPES
    s["x_scale"] = s["w_scale"] = s["bias"] = s["residual"] = s["requant"] = None
    if real:
        xr, wr = (max(0.5, float(1 << b) / 8) for b in (case["p"], case["q"]))
        s["x_scale"] = (torch.rand(rows, generator=g, device="cuda") + 0.5) / xr
        s["w_scale"] = (torch.rand(*lead, N, generator=g, device="cuda") + 0.5) / (wr * math.sqrt(K))
        if case["bias"]:
            s["bias"] = torch.randn(*lead, N, generator=g, device="cuda")
        if case["residual"]:
            s["residual"] = torch.randn(rows, N, generator=g, device="cuda").to(_TYPES[case["out"]])
        kind = _TYPES[case["out"]]
    elif case["out"] == "codes":
        s["requant"] = (_shift(case), 0, 15)
        if case["bias"]:
            s["bias"] = torch.randint(-1000, 1000, (*lead, N), generator=g, device="cuda", dtype=torch.int32)
        kind = torch.uint8
    else:
        kind = torch.int32
    s["out"] = torch.full((rows, N), 3, dtype=kind, device="cuda")
    if grouped:
        counts = np.random.default_rng(int(seed)).multinomial(case["T"], _popularity(case["E"]))
        bounds = np.concatenate([[0], np.cumsum(counts)])
        s["offsets"] = torch.tensor(bounds, dtype=torch.int32, device="cuda")
        s["capacity"] = int(counts.max())                 # the plan of the plain form: rows that the largest group has
    return s


def _values(stored, bits, signed):
    """Dense bytes to the codes that they hold, as 32-bit integers."""
    if bits == 8:
        return stored
    at = torch.arange(0, 8, bits, device=stored.device, dtype=torch.int32)
    v = (stored.to(torch.int32)[..., None] >> at) & ((1 << bits) - 1)
    if signed:
        v = v - ((v >> (bits - 1)) << bits)
    return v.flatten(-2)


def _exact_type(case):
    """32-bit floats where every partial sum of the products is a whole number below 2^24, else 64-bit ones."""
    (xl, xh), (wl, wh) = _range(case["p"], case["xs"]), _range(case["q"], case["ws"])
    return torch.float32 if max(-xl, xh) * max(-wl, wh) * case["K"] < 1 << 24 else torch.float64


def _epilogue(s, sums, x_scale, w_scale, bias, residual):
    case = s["case"]
    if case["out"] == "sums":
        return sums.to(torch.int32)
    if case["out"] == "codes":
        shift, lo, hi = s["requant"]
        v = sums.to(torch.int64)
        if bias is not None:
            v = v + bias
        return (v >> shift).clamp(lo, hi).to(torch.uint8)
    v = sums.to(torch.float32) * x_scale * w_scale
    if bias is not None:
        v = v + bias
    if case["act"] == "relu":
        v = torch.where(v < 0, torch.zeros_like(v), v)
    elif case["act"] == "silu":
        v = v / (1 + torch.exp(-v))
    elif case["act"] == "gelu":
        v = 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if residual is not None:
        v = v + residual.to(torch.float32)
    return v.to(_TYPES[case["out"]])


def _plain_quantize(s):
    v = s["x"].to(torch.float32)
    top = v.abs().amax(1) if s["case"]["signed"] else v.amax(1).clamp(min=0)
    scale = top / s["top"]
    codes = (v / scale[:, None]).round().clamp(s["lo"], s["hi"])
    codes = torch.where(torch.isnan(codes), torch.zeros_like(codes), codes)
    return codes.to(s["codes"].dtype), scale


def _plain_linear(s):
    case = s["case"]
    t = _exact_type(case)
    sums = s["x"].to(t) @ _values(s["w"], case["w_store"], case["ws"]).to(t).T
    return _epilogue(s, sums, s["x_scale"][:, None] if s["x_scale"] is not None else None, s["w_scale"], s["bias"], s["residual"])


def _plain_grouped(s):
    """Every group padded to the rows of the largest, one batched product, and each row's own result taken out."""
    case, off = s["case"], s["offsets"].to(torch.int64)
    t, rows = _exact_type(case), s["x"].shape[0]
    slot = (off[:-1, None] + torch.arange(s["capacity"], device=off.device)).clamp(max=rows - 1)
    sums = torch.bmm(s["x"].to(t)[slot], _values(s["w"], case["w_store"], case["ws"]).to(t).transpose(1, 2))
    row = torch.arange(rows, device=off.device)
    group = torch.searchsorted(off[1:].contiguous(), row, right=True)
    inside = ((row >= off[0]) & (group < case["E"]))[:, None]
    group = group.clamp(max=case["E"] - 1)
    sums = sums[group, (row - off[group]).clamp(0, s["capacity"] - 1)]
    pick = lambda v: v[group] if v is not None else None  # noqa: E731
    y = _epilogue(s, sums, s["x_scale"][:, None] if s["x_scale"] is not None else None, pick(s["w_scale"]), pick(s["bias"]), s["residual"])
    return torch.where(inside, y, s["out"])


def run(s):
    case = s["case"]
    if own:
        from paper_2208_00763_b200 import binding as hk
        if case["kind"] == "quantize":
            return hk.quantize_rows(s["x"], case["bits"], case["signed"], codes=s["codes"], scale=s["scale"])
        activation = {"none": hk.ACT_NONE, "relu": hk.ACT_RELU, "silu": hk.ACT_SILU, "gelu": hk.ACT_GELU}[case["act"]]
        if case["kind"] == "linear":
            return hk.linear(s["x"], s["w"], case["p"], case["q"], case["xs"], case["ws"], w_store_bits=case["w_store"],
                             x_scale=s["x_scale"], w_scale=s["w_scale"], bias=s["bias"], activation=activation, residual=s["residual"],
                             requant=s["requant"], out=s["out"])
        return hk.grouped_linear(s["x"], s["w"], s["offsets"], case["p"], case["q"], case["xs"], case["ws"], w_store_bits=case["w_store"],
                                 x_scale=s["x_scale"], w_scale=s["w_scale"], bias=s["bias"], activation=activation,
                                 residual=s["residual"], requant=s["requant"], out=s["out"])
    if case["kind"] == "quantize":
        return _plain_quantize(s)
    return _plain_linear(s) if case["kind"] == "linear" else _plain_grouped(s)


def work(case):
    if case["kind"] == "quantize":
        n = case["M"] * case["K"]
        return {"bytes": n * ({"f32": 4}.get(case["dtype"], 2) + 1) + 4 * case["M"], "flops": 3.0 * n}
    grouped = case["kind"] == "grouped"
    rows, K, N = case["T"] if grouped else case["M"], case["K"], case["N"]
    # weights of the experts that are chosen at all, on average over the routing
    mats = float((1 - (1 - _popularity(case["E"])) ** rows).sum()) if grouped else 1.0
    out = {"f32": 4, "sums": 4, "codes": 1}.get(case["out"], 2)
    real = case["out"] in _TYPES
    b = rows * K + mats * N * K * case["w_store"] / 8 + rows * N * out * (2 if case["residual"] else 1)
    b += (4 * rows + 4 * mats * N if real else 0) + (4 * mats * N if case["bias"] else 0) + (4 * (case["E"] + 1) if grouped else 0)
    return {"bytes": b, "flops": 2.0 * rows * N * K}


def exact(case, seed):
    """The definitions in 64 bits: codes as doubles (their sums stay far below 2^53), groups one after the other."""
    s = prepare(case, seed)
    if case["kind"] == "quantize":
        x = s["x"].double()
        lo, hi = _range(case["bits"], case["signed"])
        top = (x.abs() if case["signed"] else x.clamp(min=0)).max(dim=1).values
        # a code is defined on the scale as it is stored and on the quotient in 32 bits: rounding the 64-bit quotient gives just that
        stored = (top / hi).float()
        q = (x / stored.double()[:, None]).float().double().nan_to_num(0.0, hi, lo)
        return torch.round(q).clamp(lo, hi).to(s["codes"].dtype), top / hi

    def product(rows, w, xs, ws, b, r):
        if case["w_store"] == 8:
            codes = w.double()
        else:
            n = case["w_store"]
            parts = [(w.to(torch.int64) >> (i * n)) % (1 << n) for i in range(8 // n)]
            codes = torch.stack(parts, -1).reshape(w.shape[0], -1)
            codes = (codes - (codes >= 1 << (n - 1)).to(torch.int64) * (1 << n) if case["ws"] else codes).double()
        t = torch.einsum("mk,nk->mn", rows.double(), codes)
        if case["out"] == "sums":
            return t.to(torch.int32)
        if case["out"] == "codes":
            shift, lo, hi = s["requant"]
            return torch.floor((t if b is None else t + b.double()) / 2.0 ** shift).clamp(lo, hi).to(torch.uint8)
        t = t * xs.double()[:, None] * ws.double()[None, :]
        t = t if b is None else t + b.double()
        t = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "silu": lambda v: v * torch.sigmoid(v),
             "gelu": lambda v: v * 0.5 * torch.erfc(-v / math.sqrt(2.0))}[case["act"]](t)
        return t if r is None else t + r.double()

    none = lambda v, at: None if v is None else v[at]  # noqa: E731
    if case["kind"] == "linear":
        return product(s["x"], s["w"], s["x_scale"], s["w_scale"], s["bias"], s["residual"])
    out = s["out"].double() if case["out"] in _TYPES else s["out"].clone()
    ends = s["offsets"].tolist()
    for e in range(case["E"]):
        at = slice(ends[e], ends[e + 1])
        if ends[e + 1] > ends[e]:
            out[at] = product(s["x"][at], s["w"][e], none(s["x_scale"], at), none(s["w_scale"], e), none(s["bias"], e), none(s["residual"], at))
    return out
