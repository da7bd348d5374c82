"""The calls a user makes to run a mixture of experts, as timed cases: tokens sorted by expert, their rows brought into that order (as they
are, or quantised to 8-bit floating point with a scale for each block of 128 on the way), matrix products on such blocks, plain and grouped by
expert, and the experts' rows brought back to their tokens with weights, with the gradient of that.

Sizes are generic (powers of two as hidden sizes, and odd ones).  Outputs are the caller's buffers, as in a serving program.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_BLOCK = 128


def _sort(name, T, k, E, index, dropped):
    return {"name": name, "kind": "sort", "T": T, "k": k, "E": E, "index": index, "dropped": dropped}


def _rows(name, kind, T, k, E, H, dtype, dropped=0.0, residual=False, weights=True):
    return {"name": name, "kind": kind, "T": T, "k": k, "E": E, "H": H, "dtype": dtype, "dropped": dropped, "residual": residual, "weights": weights}


def _quantize(name, T, k, E, H, dtype, f8, dropped=0.0):
    return {"name": name, "kind": "quantize", "T": T, "k": k, "E": E, "H": H, "dtype": dtype, "f8": f8, "dropped": dropped}


def _linear(name, E, M, tail, K, N, f8, w_f8, out, act="none", bias=False, residual=False):
    return {"name": name, "kind": "linear", "E": E, "M": M, "tail": tail, "K": K, "N": N, "f8": f8, "w_f8": w_f8, "out": out, "act": act, "bias": bias,
            "residual": residual}


def listed():
    return [
        # the experts of one decoded token of each of 64 sequences: the smallest call, all latency
        _sort("sort_decode64_8of64", 64, 8, 64, "int64", 0.0),
        # a long prompt, padded: a twentieth of the tokens has no expert
        _sort("sort_prompt32k_8of256", 32768, 8, 256, "int64", 0.05),
        # rows of a size that divides nothing, which start anywhere
        _rows("rows_to_experts_odd_f16", "to", 5003, 3, 20, 1333, "f16", dropped=0.1),
        # the hidden states of a few sequences to their experts, quantised on the way
        _quantize("quantize_tokens8_to_8of64", 8, 8, 64, 4096, "bf16", "e4m3"),
        # a prompt's hidden states to their experts, quantised on the way
        _quantize("quantize_prompt8k_to_8of64", 8192, 8, 64, 4096, "bf16", "e4m3"),
        # the experts' results of a decoding batch back to its tokens, onto the residual stream
        _rows("rows_from_experts_decode32", "from", 32, 8, 64, 4096, "bf16", residual=True),
        # ... and of a prompt
        _rows("rows_from_experts_prompt8k", "from", 8192, 8, 64, 4096, "bf16", residual=True),
        # the gradient of that in training: for the experts' rows and the weights
        _rows("rows_from_grad_4k", "from_grad", 4096, 8, 64, 4096, "bf16"),
        # ... in 32 bits, at sizes that divide nothing, with tokens that some experts had no room for
        _rows("rows_from_grad_odd_f32", "from_grad", 1733, 3, 20, 5003, "f32", dropped=0.1),
        # one new token through a layer: the weights are all there is to read
        _linear("f8_token_4k_4k", 0, 1, 0, 4096, 4096, "e4m3", "e4m3", "bf16"),
        # the second product of an MLP on a prompt, onto the residual stream
        _linear("f8_prompt_4k_16k_4k_residual", 0, 4096, 0, 16384, 4096, "e4m3", "e4m3", "bf16", residual=True),
        # 32 experts on a prompt: ragged groups, a padded batch whose last rows belong to none
        _linear("f8_experts32_prompt_silu", 32, 16384, 37, 2048, 4096, "e4m3", "e4m3", "bf16", act="silu"),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _size(rng, lo, hi):
    """A size of the range: a multiple of 128 as hidden sizes are, or anything."""
    v = _log_int(rng, lo, hi)
    return v // 128 * 128 if v >= 256 and rng.random() < 0.6 else v


def draw(rng):
    kind = rng.choice(["sort", "to", "quantize", "from", "from_grad", "linear", "linear", "linear"])
    if kind == "linear":
        E = rng.choice([0, 0, 2, 4, 8, 32, 60, 64])
        K, N, M = _size(rng, 64, 16384), _size(rng, 64, 16384), _log_int(rng, 1, 8192)
        while max(E, 1) * K * N > (1 << 28) or M * K * N > (1 << 37):
            if max(E, 1) * K * N <= (1 << 28) and M >= 2048:
                M //= 2
            elif N >= K:
                N = max(64, N // 2)
            else:
                K = max(64, K // 2)
        out = rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])
        return {"kind": kind, "E": E, "M": M, "tail": rng.choice([0, 5]) if E else 0, "K": K, "N": N, "f8": rng.choice(["e4m3", "e4m3", "e4m3", "e5m2"]),
                "w_f8": rng.choice(["e4m3", "e4m3", "e4m3", "e5m2"]), "out": out, "act": rng.choice(["none", "none", "relu", "silu", "gelu"]),
                "bias": rng.random() < 0.4, "residual": rng.random() < 0.3}
    E = rng.choice([4, 8, 20, 64, 128, 256])
    k = rng.choice([1, 2, 2, 3, 4, 6, 8])
    k = min(k, E)
    dropped = rng.choice([0.0, 0.0, 0.05, 0.3])
    if kind == "sort":
        return {"kind": kind, "T": _log_int(rng, 1, 32768), "k": k, "E": E, "index": rng.choice(["int32", "int64"]), "dropped": dropped}
    H, dtype = _size(rng, 64, 8192), rng.choice(["bf16", "bf16", "f16", "f32"])
    most = (1 << 27) // (2 if dtype == "f32" else 1) // (k * H)
    T = min(_log_int(rng, 1, 8192), max(1, most))
    case = {"kind": kind, "T": T, "k": k, "E": E, "H": H, "dtype": dtype, "dropped": dropped}
    if kind == "quantize":
        if rng.random() < 0.3:
            case["k"] = case["E"] = 0                     # no experts: the rows of a dense layer
            case["dropped"] = 0.0
        return {**case, "f8": rng.choice(["e4m3", "e4m3", "e5m2"])}
    return {**case, "residual": kind == "from" and rng.random() < 0.5, "weights": kind != "to" and (kind == "from_grad" or rng.random() < 0.8)}


def _popularity(E):
    """How often experts are chosen: some several times as often as others."""
    w = 1.0 / (np.arange(E) + 0.75 * E)
    return w / w.sum()


def _route(case, g):
    """k different experts of each token and their weights, as a router chooses them; tokens, or some of their choices, without expert are -1."""
    T, k, E = case["T"], case["k"], case["E"]
    logits = torch.tensor(np.log(_popularity(E)), dtype=torch.float32, device="cuda") - torch.log(-torch.log(torch.rand(T, E, generator=g, device="cuda").clamp_(1e-20, 1 - 1e-7)))
    top, experts = torch.topk(logits, k, dim=1)
    weights = torch.softmax(top, 1)
    if case["dropped"]:
        one = torch.rand(T, k, generator=g, device="cuda") < case["dropped"] / 2
        whole = torch.rand(T, 1, generator=g, device="cuda") < case["dropped"] / 2
        experts = torch.where(one | whole, torch.full_like(experts, -1), experts)
    return experts, weights


def _plain_sort(experts, E):
    """Pairs of token and choice in the order of their experts, equal ones as they come; those without expert behind all, as -2 - place."""
    flat = experts.reshape(-1).to(torch.int64)
    key = torch.where((flat >= 0) & (flat < E), flat, torch.full_like(flat, E))
    ordered, order = torch.sort(key, stable=True)
    offsets = torch.searchsorted(ordered, torch.arange(E + 1, device=flat.device)).to(torch.int32)
    place = torch.empty_like(order)
    place[order] = torch.arange(flat.numel(), device=flat.device)
    slots = torch.where(key < E, place, -2 - place).to(torch.int32)
    return offsets, slots.reshape(experts.shape)


def _f8_buffer(rows, K, f8, g):
    """A matrix of 8-bit floats with rows on 16-byte boundaries, holding something."""
    wide = torch.randint(0, 0x70, (rows, (K + 15) // 16 * 16), generator=g, device="cuda", dtype=torch.uint8)
    return wide.view(_F8[f8])[:, :K]


def _hidden(rows, H, dtype, g, seed):
    """Hidden states: rows of different size, a channel with outliers."""
    x = torch.randn(rows, H, generator=g, device="cuda")
    x *= torch.rand(rows, 1, generator=g, device="cuda") * 4 + 0.1
    x[:, int(seed) % H] *= 8.0
    return x.to(_TYPES[dtype])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": case}
    kind = case["kind"]
    if kind == "linear":
        E, M, K, N = case["E"], case["M"], case["K"], case["N"]
        rows, lead = M + case["tail"], (E,) if E else ()
        kb, nb = -(-K // _BLOCK), -(-N // _BLOCK)
        wide = (K + 15) // 16 * 16
        # what a quantiser leaves: normal values, the largest of a block at the end of the type's range
        x = torch.randn(rows, wide, generator=g, device="cuda") * (140.0 if case["f8"] == "e4m3" else 18000.0)
        s["x"] = x.clamp_(-torch.finfo(_F8[case["f8"]]).max, torch.finfo(_F8[case["f8"]]).max).to(_F8[case["f8"]])[:, :K]
        del x
        w = torch.empty(*lead, N, wide, dtype=_F8[case["w_f8"]], device="cuda")
        for part in w if E else [w]:
            v = torch.randn(N, wide, generator=g, device="cuda") * (120.0 if case["w_f8"] == "e4m3" else 15000.0)
            part.copy_(v.clamp_(-torch.finfo(w.dtype).max, torch.finfo(w.dtype).max))
        s["w"] = w[..., :K]
        s["x_scale"] = (torch.rand(kb, rows, generator=g, device="cuda") + 0.2) / (140.0 if case["f8"] == "e4m3" else 18000.0)
        s["w_scale"] = (torch.rand(*lead, nb, kb, generator=g, device="cuda") + 0.5) / ((120.0 if case["w_f8"] == "e4m3" else 15000.0) * math.sqrt(K))
        s["bias"] = torch.randn(*lead, N, generator=g, device="cuda") if case["bias"] else None
        s["residual"] = torch.randn(rows, N, generator=g, device="cuda").to(_TYPES[case["out"]]) if case["residual"] else None
        s["out"] = torch.full((rows, N), 3, dtype=_TYPES[case["out"]], device="cuda")
        if E:
            counts = np.random.default_rng(int(seed)).multinomial(M, _popularity(E))
            s["offsets"] = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
            s["capacity"] = int(counts.max())             # the plan of the plain form: rows that the largest group has
        return s
    if kind == "quantize" and not case["k"]:
        s["x"] = _hidden(case["T"], case["H"], case["dtype"], g, seed)
        s["slots"], R = None, case["T"]
    else:
        experts, weights = _route(case, g)
        R = case["T"] * case["k"]
        if kind == "sort":
            s["experts"] = experts.to(getattr(torch, case["index"]))
            s["offsets"] = torch.empty(case["E"] + 1, dtype=torch.int32, device="cuda")
            s["slots"] = torch.empty(case["T"], case["k"], dtype=torch.int32, device="cuda")
            return s
        s["slots"] = _plain_sort(experts, case["E"])[1]
        if kind in ("to", "quantize"):
            s["x"] = _hidden(case["T"], case["H"], case["dtype"], g, seed)
    if kind == "quantize":
        s["values"] = _f8_buffer(R, case["H"], case["f8"], g)
        s["scale"] = torch.full((-(-case["H"] // _BLOCK), R), 0.5, device="cuda")
        return s
    t = _TYPES[case["dtype"]]
    s["weights"] = weights if case["weights"] else None
    if kind == "to":
        s["out"] = torch.full((R, case["H"]), 3, dtype=t, device="cuda")
        return s
    s["y"] = _hidden(R, case["H"], case["dtype"], g, seed)
    s["residual"] = torch.randn(case["T"], case["H"], generator=g, device="cuda").to(t) if case["residual"] else None
    if kind == "from":
        s["out"] = torch.empty(case["T"], case["H"], dtype=t, device="cuda")
        return s
    s["grad"] = torch.randn(case["T"], case["H"], generator=g, device="cuda").to(t)
    s["grad_y"] = torch.empty(R, case["H"], dtype=t, device="cuda")
    s["grad_weights"] = torch.empty(case["T"], case["k"], device="cuda")
    return s


def _token_of_place(slots, R):
    """Which token's row lies at each place, -1 for none."""
    T, k = slots.shape
    at = torch.full((R + 1,), -1, dtype=torch.int64, device=slots.device)
    pair = torch.arange(T * k, device=slots.device)
    flat = slots.reshape(-1).to(torch.int64)
    at[torch.where(flat >= 0, flat, torch.full_like(flat, R))] = pair // k
    return at[:R]


def _bytes(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t


def _to_places(rows, slots, before):
    """`before` with the rows of tokens at their places."""
    if slots is None:
        return rows
    token = _token_of_place(slots, before.shape[0])
    return torch.where((token >= 0)[:, None], _bytes(rows)[token.clamp(min=0)], _bytes(before)).view(before.dtype)


def _plain_quantize(s):
    case, x = s["case"], s["x"].to(torch.float32)
    top = torch.tensor(torch.finfo(_F8[case["f8"]]).max, device=x.device)
    M, K = x.shape
    blocks = torch.nn.functional.pad(x, (0, -K % _BLOCK)).reshape(M, -1, _BLOCK)
    scale = blocks.abs().amax(2) / top
    q = blocks / scale[..., None]
    q = torch.where((scale == 0)[..., None], torch.zeros_like(q), q).clamp(-top, top)
    values = q.reshape(M, -1)[:, :K].to(_F8[case["f8"]])
    return _to_places(values, s["slots"], s["values"]), (_to_places(scale, s["slots"], s["scale"].T)).T


def _plain_from(s):
    slots = s["slots"].to(torch.int64)
    rows = s["y"][slots.clamp(min=0)].to(torch.float32)
    if s["weights"] is not None:
        rows = rows * s["weights"][..., None]
    out = torch.where((slots >= 0)[..., None], rows, torch.zeros_like(rows)).sum(1)
    if s["residual"] is not None:
        out = out + s["residual"].to(torch.float32)
    return out.to(s["out"].dtype)


def _plain_from_grad(s):
    slots, grad = s["slots"].to(torch.int64), s["grad"].to(torch.float32)
    there = (slots >= 0)[..., None]
    parts = torch.where(there, grad[:, None, :] * s["weights"][..., None], torch.zeros((), device=grad.device))
    grad_y = torch.empty_like(s["grad_y"])
    grad_y[torch.where(slots >= 0, slots, -2 - slots).reshape(-1)] = parts.reshape(-1, grad.shape[1]).to(grad_y.dtype)
    dot = (grad[:, None, :] * s["y"][slots.clamp(min=0)].to(torch.float32)).sum(2)
    return grad_y, torch.where(there[..., 0], dot, torch.zeros_like(dot))


def _spread(scale, size, dim):
    """A scale for each value from one for each block."""
    return scale.repeat_interleave(_BLOCK, dim).narrow(dim, 0, size)


def _plain_linear(s):
    case = s["case"]
    K, N = case["K"], case["N"]
    x = s["x"].to(torch.float32) * _spread(s["x_scale"].T, K, 1)
    w = s["w"].to(torch.float32) * _spread(_spread(s["w_scale"], N, s["w_scale"].dim() - 2), K, s["w_scale"].dim() - 1)
    bias, rows = s["bias"], x.shape[0]
    if case["E"]:
        # every group padded to the rows of the largest, one batched product, and each row's own result taken out
        off = s["offsets"].to(torch.int64)
        slot = (off[:-1, None] + torch.arange(s["capacity"], device=off.device)).clamp(max=rows - 1)
        v = torch.bmm(x[slot], w.transpose(1, 2))
        row = torch.arange(rows, device=off.device)
        group = torch.searchsorted(off[1:].contiguous(), row, right=True)
        inside = ((row >= off[0]) & (group < case["E"]))[:, None]
        group = group.clamp(max=case["E"] - 1)
        v = v[group, (row - off[group]).clamp(0, s["capacity"] - 1)]
        bias = bias[group] if bias is not None else None
    else:
        v = x @ w.T
    if bias is not None:
        v = v + bias
    if case["act"] == "relu":
        v = torch.where(v < 0, torch.zeros_like(v), v)
    elif case["act"] == "silu":
        v = v / (1 + torch.exp(-v))
    elif case["act"] == "gelu":
        v = 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if s["residual"] is not None:
        v = v + s["residual"].to(torch.float32)
    v = v.to(s["out"].dtype)
    return torch.where(inside, v, s["out"]) if case["E"] else v


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        from paper_2208_00763_b200 import binding as hk
        if kind == "sort":
            return hk.sort_by_expert(s["experts"], case["E"], offsets=s["offsets"], slots=s["slots"])
        if kind == "to":
            return hk.rows_to_experts(s["x"], s["slots"], out=s["out"])
        if kind == "quantize":
            return hk.quantize_blocks(s["x"], _F8[case["f8"]], slots=s["slots"], values=s["values"], scale=s["scale"])
        if kind == "from":
            return hk.rows_from_experts(s["y"], s["slots"], s["weights"], residual=s["residual"], out=s["out"])
        if kind == "from_grad":
            return hk.rows_from_experts_grad(s["grad"], s["y"], s["slots"], s["weights"], grad_y=s["grad_y"], grad_weights=s["grad_weights"])
        activation = {"none": hk.ACT_NONE, "relu": hk.ACT_RELU, "silu": hk.ACT_SILU, "gelu": hk.ACT_GELU}[case["act"]]
        if case["E"]:
            return hk.grouped_linear_f8(s["x"], s["w"], s["offsets"], s["x_scale"], s["w_scale"], bias=s["bias"], activation=activation,
                                        residual=s["residual"], out=s["out"])
        return hk.linear_f8(s["x"], s["w"], s["x_scale"], s["w_scale"], bias=s["bias"], activation=activation, residual=s["residual"], out=s["out"])
    if kind == "sort":
        return _plain_sort(s["experts"], case["E"])
    if kind == "to":
        return _to_places(s["x"], s["slots"], s["out"])
    return {"quantize": _plain_quantize, "from": _plain_from, "from_grad": _plain_from_grad, "linear": _plain_linear}[kind](s)


def work(case):
    kind, size = case["kind"], 4 if case.get("dtype") == "f32" else 2
    if kind == "linear":
        M, K, N, E = case["M"], case["K"], case["N"], case["E"]
        # weights of the experts that are chosen at all, on average over the routing
        mats = float((1 - (1 - _popularity(E)) ** M).sum()) if E else 1.0
        out = 4 if case["out"] == "f32" else 2
        b = M * K + mats * N * K + 4.0 * M * -(-K // _BLOCK) + 4.0 * mats * -(-K // _BLOCK) * -(-N // _BLOCK)
        b += M * N * out * (2 if case["residual"] else 1) + (4 * mats * N if case["bias"] else 0) + (4 * (E + 1) if E else 0)
        return {"bytes": b, "flops": 2.0 * M * N * K}
    T, k = case["T"], case["k"]
    if kind == "sort":
        return {"bytes": T * k * (4.0 + (8 if case["index"] == "int64" else 4)) + 4 * (case["E"] + 1), "flops": 2.0 * T * k}
    H, kept = case["H"], T * k * (1 - case["dropped"] / 2) ** 2
    if kind == "to":
        return {"bytes": (T + kept) * H * size + 4.0 * T * k, "flops": 0.0}
    if kind == "quantize":
        kept = kept if k else T
        return {"bytes": T * H * size + kept * (H + 4.0 * -(-H // _BLOCK)) + 4.0 * T * k, "flops": 3.0 * T * H}
    if kind == "from":
        return {"bytes": (kept + T * (2 if case["residual"] else 1)) * H * size + T * k * (8.0 if case["weights"] else 4.0), "flops": 2.0 * kept * H}
    return {"bytes": (T + kept + T * k) * H * size + 12.0 * T * k, "flops": 3.0 * kept * H}


def exact(case, seed):
    """The definitions in 64 bits, one row, expert or group after the other where that says it best."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "sort":
        ids = s["experts"].flatten().cpu().numpy()
        place = np.full(ids.shape, -1, np.int64)
        ends, at = [0], 0
        for e in range(case["E"]):
            mine = np.nonzero(ids == e)[0]
            place[mine] = at + np.arange(len(mine))
            at += len(mine)
            ends.append(at)
        rest = np.nonzero((ids < 0) | (ids >= case["E"]))[0]
        place[rest] = -2 - (at + np.arange(len(rest)))
        return torch.tensor(ends, dtype=torch.int32), torch.tensor(place, dtype=torch.int32).reshape(s["slots"].shape)
    if kind == "linear":
        def product(x, xs, w, ws, b, r):
            v = torch.zeros(x.shape[0], w.shape[0], dtype=torch.float64, device=x.device)
            for j in range(xs.shape[0]):
                at = slice(j * _BLOCK, min((j + 1) * _BLOCK, case["K"]))
                part = torch.einsum("mk,nk->mn", x[:, at].double(), w[:, at].double())
                v += part * xs[j].double()[:, None] * ws[:, j].double().repeat_interleave(_BLOCK)[: case["N"]]
            v = v if b is None else v + b.double()
            v = {"none": lambda u: u, "relu": lambda u: u.clamp(min=0), "silu": lambda u: u * torch.sigmoid(u),
                 "gelu": lambda u: u * 0.5 * torch.erfc(-u / math.sqrt(2.0))}[case["act"]](v)
            return v if r is None else v + r.double()

        none = lambda v, at: None if v is None else v[at]  # noqa: E731
        if not case["E"]:
            return product(s["x"], s["x_scale"], s["w"], s["w_scale"], s["bias"], s["residual"])
        out, ends = s["out"].double(), s["offsets"].tolist()
        for e in range(case["E"]):
            at = slice(ends[e], ends[e + 1])
            if ends[e + 1] > ends[e]:
                out[at] = product(s["x"][at], s["x_scale"][:, at], s["w"][e], s["w_scale"][e], none(s["bias"], e), none(s["residual"], at))
        return out
    slots = s["slots"]
    if kind in ("to", "quantize"):
        if kind == "to":
            parts = [(s["out"].double(), s["x"].double())]
        else:
            top, x = torch.finfo(_F8[case["f8"]]).max, s["x"].double()
            wide = torch.zeros(x.shape[0], -(-x.shape[1] // _BLOCK) * _BLOCK, dtype=torch.float64, device=x.device)
            wide[:, : x.shape[1]] = x
            scale = wide.unflatten(1, (-1, _BLOCK)).abs().max(dim=2).values / top
            # a value is defined on the scale as it is stored
            values = (x / scale.float().double().repeat_interleave(_BLOCK, 1)[:, : x.shape[1]]).nan_to_num(0.0).clamp(-top, top)
            parts = [(s["values"].float().double(), values), (s["scale"].T.double(), scale)]
        for j in range(0 if slots is None else case["k"]):
            there = slots[:, j] >= 0
            for before, rows in parts:
                before[slots[there, j].long()] = rows[there]
        if kind == "to":
            return parts[0][0]
        return parts[0][slots is None], parts[1][slots is None].T
    if kind == "from":
        out = s["residual"].double() if s["residual"] is not None else torch.zeros(case["T"], case["H"], dtype=torch.float64, device="cuda")
        for j in range(case["k"]):
            there = slots[:, j] >= 0
            rows = s["y"][slots[there, j].long()].double()
            out[there] += rows if s["weights"] is None else rows * s["weights"][there, j].double()[:, None]
        return out
    grad_y = torch.zeros(s["grad_y"].shape, dtype=torch.float64, device="cuda")
    grad_w = torch.zeros(s["grad_weights"].shape, dtype=torch.float64, device="cuda")
    for j in range(case["k"]):
        there = slots[:, j] >= 0
        at = slots[there, j].long()
        grad_y[at] = s["grad"][there].double() * s["weights"][there, j].double()[:, None]
        grad_w[there, j] = torch.einsum("th,th->t", s["grad"][there].double(), s["y"][at].double())
    return grad_y, grad_w
