"""Products of 8-bit integers and products grouped by expert: what an expert-parallel rank multiplies besides its fused layer.

  quantize  rows of activations or weights to 8-bit integers with a scale for each row
  matmul    a dense product of 8-bit integers with a scale for each token and each output channel
  grouped   products grouped by expert with ragged sizes: rows sorted by expert (or looked up in the order of a dispatch)
            against each expert's matrix, in 8-bit integers, bf16 or fp32, plain or as the gated first half of an expert

`own` chooses between the framework's operators and plain torch forms of the same definitions (32-bit sums, rounded once at
the end).  `exact` computes the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2, "i8": 1}
_TINY = 2.0 ** -126        # the smallest scale of a row that is not all zeros


# ------------------------------------------------------------------------- cases

def _grouped(name, M, G, N, K, fmt, out="bf16", gated=False, k=0, skew=1.0, spare=0):
    """M rows of G experts, sizes by popularity (rank + 1) ** -skew; `spare` places behind the last expert's rows.
    k > 0: rows looked up through a dispatch permutation of assignments, k to a token."""
    return dict(name=name, kind="grouped", M=M, G=G, N=N, K=K, fmt=fmt, out=out, gated=gated, k=k, skew=skew, spare=spare)


def listed() -> list:
    return [
        # activations of a decode step, a view of a wider buffer
        dict(name="quantize_decode_250", kind="quantize", rows=250, K=4096, src="bf16", wide=2),
        # activations of a long prefill
        dict(name="quantize_prefill_20011", kind="quantize", rows=20011, K=7168, src="bf16", wide=1),
        # one new token through a projection
        dict(name="matmul_1", kind="matmul", M=1, N=7168, K=4096, out="bf16"),
        # a running batch, neither tokens nor channels a multiple of a tile, 32-bit result
        dict(name="matmul_61_odd", kind="matmul", M=61, N=4099, K=2064, out="f32"),
        # a prompt of ordinary length
        dict(name="matmul_777", kind="matmul", M=777, N=4096, K=7168, out="bf16"),
        # a large prefill batch
        dict(name="matmul_8192", kind="matmul", M=8192, N=4096, K=7168, out="bf16"),
        # a few tokens on one rank's experts: gate and up halves, weights streamed once
        _grouped("grouped_decode_gated_i8", 30, 17, 2048, 4096, "i8", gated=True, k=8, skew=0.8),
        # the second half of the experts for a running batch
        _grouped("grouped_decode_down_bf16", 250, 32, 4096, 1408, "bf16", skew=1.0, spare=6),
        # bring-up size in fp32
        _grouped("grouped_tiny_f32", 200, 5, 256, 128, "f32", out="f32", gated=True, k=2, skew=0.7),
        # an ordinary prefill in bf16: a few busy experts, many with a handful of rows
        _grouped("grouped_prefill_gated_bf16", 4159, 17, 1408, 4096, "bf16", gated=True, k=8, skew=1.2),
        # the second half of the experts of a prefill, in 8 bits
        _grouped("grouped_prefill_down_i8", 8111, 12, 7168, 2048, "i8", skew=1.0, spare=81),
        # a long prefill on the heaviest rank, in 8 bits
        _grouped("grouped_long_gated_i8", 19711, 9, 2048, 7168, "i8", gated=True, k=8, skew=1.0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn_size(rng, lo, hi, step):
    return max(step, _log_uniform(rng, lo, hi) // step * step)


_MOST_BYTES, _MOST_FLOPS, _MOST_WEIGHTS = 4.5e8, 5e11, 3e8       # of a drawn case


def draw(rng) -> dict:
    kind = rng.choice(["quantize", "matmul", "matmul", "grouped", "grouped", "grouped"])
    if kind == "quantize":
        K, src = _drawn_size(rng, 64, 16384, 16), rng.choice(["bf16", "bf16", "f32"])
        most = int(_MOST_BYTES / (_BYTES[src] + 1)) // K * 9 // 10
        return dict(kind=kind, rows=_log_uniform(rng, 1, min(30000, most)), K=K, src=src, wide=rng.choice([1, 1, 3]))
    if kind == "matmul":
        case = dict(kind=kind, M=_log_uniform(rng, 1, 16384), N=_log_uniform(rng, 64, 16384), K=_drawn_size(rng, 128, 16384, 16),
                    out=rng.choice(["bf16", "bf16", "f32"]))
    else:
        fmt = rng.choice(["i8", "i8", "bf16", "bf16", "f32"])
        top = 8192 if fmt != "f32" else 1024
        case = _grouped("", _log_uniform(rng, 1, 20000), _log_uniform(rng, 1, 128), _drawn_size(rng, 64, top, 8) + rng.choice([0, 0, 3]),
                        _drawn_size(rng, 64, top, {"i8": 16, "bf16": 8, "f32": 4}[fmt]), fmt,
                        out="f32" if fmt == "f32" else rng.choice(["bf16", "f32"]) if fmt == "i8" else "bf16", gated=rng.random() < 0.5,
                        k=rng.choice([0, 0, 1, 2, 8]), skew=rng.choice([0.0, 0.7, 1.0, 1.4]), spare=rng.choice([0, 0, 17]))
        del case["name"]
    # never more than the largest listed case: fewer rows, then fewer experts, then narrower matrices
    flops = _MOST_FLOPS if case.get("fmt") != "f32" else 2e10
    weights = lambda: case["N"] * case["K"] * case.get("G", 1) * (2 if case.get("gated") else 1)  # noqa: E731
    while work(case)["flops"] > flops or work(case)["bytes"] > _MOST_BYTES or weights() > _MOST_WEIGHTS:
        if case["M"] > 64 and work(case)["flops"] > flops:
            case["M"] = case["M"] * 2 // 3
        elif case.get("G", 1) > 1 and weights() > _MOST_WEIGHTS // 4:
            case["G"] = case["G"] * 2 // 3
        elif case["M"] > 64 and rng.random() < 0.5:
            case["M"] = case["M"] * 2 // 3
        else:
            case["N"] = max(64, case["N"] * 2 // 3)
    return case


def _sizes(case) -> np.ndarray:
    """Rows of each expert, a function of the case alone: popular ones far apart, some with none."""
    host = np.random.default_rng([case["M"], case["G"], case["N"]])
    weight = (np.arange(case["G"]) + 1.0) ** -case["skew"]
    ends = np.rint(np.cumsum(weight) / weight.sum() * case["M"]).astype(np.int64)
    return host.permutation(np.diff(ends, prepend=0))


def _tokens(case) -> int:
    """Rows of x: as many as there are products' rows, or about half of that behind a permutation; an expert takes a token once."""
    return case["M"] if case["k"] == 0 else max(1, case["M"] // 2, int(_sizes(case).max()))


# ----------------------------------------------------------------------- prepare

def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def _activations(g, rows, K, dtype):
    """Rows as layers meet them: tokens of different size, a few channels that stand out."""
    x = torch.randn((rows, K), generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=g, device=DEV))
    x *= 1.0 + 9.0 * (torch.rand(K, generator=g, device=DEV) < 0.01)
    return x.to(dtype)


def _codes(x):
    """Codes and scales of rows that a user's program has in 8 bits already."""
    scale = x.float().abs().amax(dim=-1).clamp(min=1e-20) / 127.0
    return torch.round(x.float() / scale[..., None]).to(torch.int8), scale


def _weights(g, G, N, K, fmt):
    """[G][N][K] and, in 8 bits, [G][N] scales; an expert at a time."""
    if fmt != "i8":
        return _randn(g, (G, N, K), _TYPES[fmt], K ** -0.5), None
    w, s = torch.empty((G, N, K), dtype=torch.int8, device=DEV), torch.empty((G, N), device=DEV)
    for e in range(G):
        w[e], s[e] = _codes(torch.randn((N, K), generator=g, device=DEV) * K ** -0.5)
    return w, s


def prepare(case: dict, seed: int) -> dict:
    g = torch.Generator(device=DEV).manual_seed(seed)
    state = dict(kind=case["kind"])
    if case["kind"] == "quantize":
        rows, K = case["rows"], case["K"]
        x = _activations(g, rows, K * case["wide"], _TYPES[case["src"]])[:, :K]
        state.update(x=x, codes=torch.zeros((rows, K), dtype=torch.int8, device=DEV), scale=torch.zeros(rows, device=DEV))
        return state
    if case["kind"] == "matmul":
        x, xs = _codes(_activations(g, case["M"], case["K"], torch.float32))
        w, ws = _weights(g, 1, case["N"], case["K"], "i8")
        state.update(x=x, x_scale=xs, w=w[0], w_scale=ws[0], out=torch.zeros((case["M"], case["N"]), dtype=_TYPES[case["out"]], device=DEV))
        return state
    # rows of this rank in the order of a dispatch: expert by expert, spare places at the end
    sizes, k, M = _sizes(case), case["k"], case["M"]
    host = np.random.default_rng(seed)
    tokens = _tokens(case)
    x = _activations(g, tokens, case["K"], torch.float32 if case["fmt"] == "i8" else _TYPES[case["fmt"]])
    xs = None
    if case["fmt"] == "i8":
        x, xs = _codes(x)
    src = None
    if k:
        # assignments token * k + j, ascending among an expert's rows
        picks = [np.sort(host.choice(tokens, int(n), replace=False)) * k + host.integers(0, k, int(n)) for n in sizes]
        src = torch.from_numpy(np.concatenate(picks + [np.zeros(case["spare"], np.int64)])).to(DEV, torch.int32)
    elif case["spare"]:
        pad = lambda t: torch.cat([t, t[:1].expand(case["spare"], *t.shape[1:])])  # noqa: E731
        x, xs = pad(x), None if xs is None else pad(xs)
    w, ws = _weights(g, case["G"], case["N"], case["K"], case["fmt"])
    up, ups = _weights(g, case["G"], case["N"], case["K"], case["fmt"]) if case["gated"] else (None, None)
    off = np.concatenate([[0], np.cumsum(sizes)])
    state.update(x=x, x_scale=xs, src=src, k=max(k, 1), w=w, w_scale=ws, up=up, up_scale=ups, off=torch.from_numpy(off).to(DEV, torch.int32),
                 bounds=off.tolist(), out=torch.zeros((M + case["spare"], case["N"]), dtype=_TYPES[case["out"]], device=DEV))
    if own:
        from paper_2603_28768_amd import binding
        state["handle"] = binding.GroupedMatmul(w, scales=ws, up=up, up_scales=ups, dtype=case["out"])
    return state


# --------------------------------------------------------------------------- run

def run(state: dict):
    if own:
        from paper_2603_28768_amd import binding
        if state["kind"] == "quantize":
            return binding.quantize_i8(state["x"], codes=state["codes"], scale=state["scale"])
        if state["kind"] == "matmul":
            return binding.matmul_i8(state["x"], state["x_scale"], state["w"], state["w_scale"], out=state["out"])
        return state["handle"](state["x"], state["off"], x_scale=state["x_scale"], src=state["src"], k=state["k"], out=state["out"])
    return {"quantize": _quantize_plain, "matmul": _matmul_plain, "grouped": _grouped_plain}[state["kind"]](state)


def _quantize_plain(s):
    # quotients in 64 bits, rounded to 32: the nearest code of a 32-bit quotient depends on its last bit
    x = s["x"].double()
    amax = x.abs().amax(dim=-1)
    scale = torch.where(amax > 0, (amax / 127.0).float().clamp(min=_TINY), 1.0)
    codes = torch.round((x / scale.double()[:, None]).float()).clamp(-127.0, 127.0)
    s["codes"].copy_(codes)
    s["scale"].copy_(scale)
    return s["codes"], s["scale"]


def _matmul_plain(s):
    y = torch.matmul(s["x"].float(), s["w"].float().T)
    s["out"].copy_(y * s["x_scale"][:, None] * s["w_scale"])
    return s["out"]


def _product(x, xs, w, ws):
    y = torch.matmul(x.float(), w.float().T)
    return y if xs is None else y * xs[:, None] * ws


def _grouped_plain(s):
    x, xs = s["x"], s["x_scale"]
    if s["src"] is not None:
        token = s["src"].long() // s["k"]
        x, xs = x[token], None if xs is None else xs[token]
    # a product for each expert that has rows: one batched product would pad all of them to the longest
    for e, (lo, hi) in enumerate(zip(s["bounds"], s["bounds"][1:])):
        if hi > lo:
            rows, scales = x[lo:hi], None if xs is None else xs[lo:hi]
            y = _product(rows, scales, s["w"][e], None if xs is None else s["w_scale"][e])
            if s["up"] is not None:
                y = y / (1.0 + torch.exp(-y)) * _product(rows, scales, s["up"][e], None if xs is None else s["up_scale"][e])
            s["out"][lo:hi] = y
    return s["out"]


# ------------------------------------------------------------------- work, exact

def work(case: dict) -> dict:
    if case["kind"] == "quantize":
        n = float(case["rows"]) * case["K"]
        return {"bytes": n * (_BYTES[case["src"]] + 1) + 4.0 * case["rows"], "flops": 3.0 * n}
    M, N, K = float(case["M"]), float(case["N"]), float(case["K"])
    if case["kind"] == "matmul":
        return {"bytes": M * K + N * K + 4 * (M + N) + M * N * _BYTES[case["out"]], "flops": 2 * M * N * K}
    es, mats = _BYTES[case["fmt"]], 2 if case["gated"] else 1
    live = float((_sizes(case) > 0).sum())                  # experts without rows are not read
    tokens = float(_tokens(case))
    scales = 4 * (tokens + live * N * mats) if case["fmt"] == "i8" else 0.0
    return {"bytes": tokens * K * es + live * N * K * es * mats + M * N * _BYTES[case["out"]] + scales + (4 * M if case["k"] else 0) + 4 * case["G"],
            "flops": 2 * M * N * K * mats}


def _exact_quantize(s):
    codes, scale = np.empty(s["codes"].shape, np.int8), np.empty(len(s["scale"]))
    for lo in range(0, len(codes), 1000):
        x = s["x"][lo:lo + 1000].cpu().double().numpy()
        amax = np.abs(x).max(axis=1)
        sc = np.where(amax > 0, np.maximum(amax / 127.0, _TINY), 1.0)
        stored = sc.astype(np.float32).astype(np.float64)          # codes are the nearest to quotients by what is stored
        codes[lo:lo + 1000] = np.clip(np.rint((x / stored[:, None]).astype(np.float32)), -127, 127)
        scale[lo:lo + 1000] = sc
    return torch.from_numpy(codes).to(DEV), torch.from_numpy(scale).to(DEV)


def exact(case: dict, seed: int):
    s = prepare(case, seed)
    if s["kind"] == "quantize":
        return _exact_quantize(s)
    if s["kind"] == "matmul":
        values = s["w"].double() * s["w_scale"].double()[:, None]
        return (s["x"].double() * s["x_scale"].double()[:, None]) @ values.T
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    at = torch.arange(len(out), device=DEV) if s["src"] is None else s["src"].long() // s["k"]
    for e in range(case["G"]):
        rows = torch.arange(s["bounds"][e], s["bounds"][e + 1], device=DEV)
        x = s["x"][at[rows]].double()
        if s["x_scale"] is not None:
            x = x * s["x_scale"][at[rows]].double()[:, None]
        sides = []
        for w, ws in ((s["w"], s["w_scale"]), (s["up"], s["up_scale"])):
            if w is not None:
                values = w[e].double()
                sides.append(x @ (values if ws is None else values * ws[e].double()[:, None]).T)
        out[rows] = sides[0] if len(sides) == 1 else sides[0] * torch.sigmoid(sides[0]) * sides[1]
    return out
