"""Microscaled 4-bit floating point (MXFP4, NVFP4): the operators as cases with inputs, one pass and necessary work.

A case is a plain dict.  Its "kind" says which operator a pass goes through:

  quantise     a matrix to 4-bit codes and block scales, and the values that these stand for (what a user looks at to
               judge a quantisation; activations are quantised the same way in front of every product)
  dequantise   codes and scales to values
  gemm         Y = alpha X W^T of two microscaled matrices
  grouped      rows sorted by expert, each group times its expert's weights; group borders are on the device

Formats: "mx" = blocks of 32 along K with power-of-two scales (E8M0), "nv" = blocks of 16 with E4M3 scales and one fp32
factor for the whole matrix.  Sizes are those of the benchmark configurations (LLaMA-3.1 8B and 70B linears with q/k/v
and gate/up merged) and generic ones; values: activations N(0,1) with 1 % of the channels times 20, weights N(0,0.02)
with a few large entries.
"""

import torch

own = False

BLOCK = {"mx": 32, "nv": 16}
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# a power of two that brings weights of about 0.1 at most into the range of E4M3 block scales
NV_FACTOR = 1024.0


def listed():
    return [
        # eight requests decode: activations in front of a product (launches and latency)
        {"name": "quantise_decode8", "kind": "quantise", "mode": "plain", "rows": 8, "K": 4096, "type": "f16", "fmt": "mx", "top": 1},
        # a prompt's tokens copied to their four experts each, while they are quantised
        {"name": "quantise_to_experts", "kind": "quantise", "mode": "gather", "rows": 8192, "K": 4096, "type": "bf16", "fmt": "mx", "top": 4},
        # a feed-forward block's inner activations: gate and up halves joined, then quantised
        {"name": "quantise_swiglu", "kind": "quantise", "mode": "swiglu", "rows": 2048, "K": 14336, "type": "f16", "fmt": "nv", "top": 1},
        # a small layer of odd width, looked at
        {"name": "dequantise_ragged", "kind": "dequantise", "rows": 1003, "K": 2880, "type": "f16", "fmt": "mx"},
        # a whole layer's weights back to 16 bits
        {"name": "dequantise_layer", "kind": "dequantise", "rows": 14336, "K": 4096, "type": "bf16", "fmt": "nv"},
        # one token through the merged q/k/v layer
        {"name": "decode1_qkv", "kind": "gemm", "M": 1, "N": 6144, "K": 4096, "type": "f16", "fmt": "mx"},
        # a batch that fills no tile through a layer of odd sizes
        {"name": "batch27_ragged", "kind": "gemm", "M": 27, "N": 5003, "K": 2880, "type": "bf16", "fmt": "mx"},
        # the large model's gate/up layer at a decoding batch of 64
        {"name": "batch64_gate_up_70b", "kind": "gemm", "M": 64, "N": 57344, "K": 8192, "type": "f16", "fmt": "nv"},
        # a long prompt: the largest work
        {"name": "prefill4096_gate_up", "kind": "gemm", "M": 4096, "N": 28672, "K": 4096, "type": "bf16", "fmt": "nv"},
        # sixteen requests decode, four experts of 64 each: most experts see one row or none
        {"name": "experts_decode16", "kind": "grouped", "M": 64, "N": 4096, "K": 2048, "E": 64, "type": "bf16", "fmt": "mx"},
        # a small batch of prompts, experts of odd sizes
        {"name": "experts_ragged", "kind": "grouped", "M": 1021, "N": 5760, "K": 2880, "E": 32, "type": "f16", "fmt": "mx"},
        # a long prompt over few experts
        {"name": "experts_prefill", "kind": "grouped", "M": 16384, "N": 4096, "K": 4096, "E": 8, "type": "bf16", "fmt": "nv"},
    ]


def _log(rng, lo, hi):
    """A whole number, its logarithm uniform over [lo, hi]."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["quantise", "dequantise", "gemm", "gemm", "grouped", "grouped"])
    fmt = rng.choice(["mx", "nv"])
    if kind in ("quantise", "dequantise"):
        K = 32 * _log(rng, 8, 512)
        rows = _log(rng, 1, min(16384, (1 << 26) // K))
        if kind == "dequantise":
            return {"kind": kind, "rows": max(16, rows), "K": K, "type": rng.choice(["f16", "bf16"]), "fmt": fmt}
        mode = rng.choice(["plain", "gather", "swiglu"])
        return {"kind": kind, "mode": mode, "rows": rows, "K": K, "type": rng.choice(["f16", "bf16", "f32"]), "fmt": fmt,
                "top": rng.choice([1, 2, 4, 8]) if mode == "gather" else 1}
    out = rng.choice(["f16", "bf16"])
    K = 32 * _log(rng, 32, 512)
    if kind == "gemm":
        N = _log(rng, 1000, min(57344, int(4.7e8 / K)))
        return {"kind": kind, "M": _log(rng, 1, min(4096, int(4.8e11 / (N * K)))), "N": N, "K": K, "type": out, "fmt": fmt}
    K = min(K, 8192)
    E = _log(rng, 2, 128)
    N = _log(rng, 512, max(513, min(8192, int(1.0e9 / (E * K)))))
    return {"kind": kind, "M": _log(rng, 1, min(16384, int(2.7e11 / (N * K)))), "N": N, "K": K, "E": E, "type": out, "fmt": fmt}


def _activations(gen, rows, K, dtype=torch.float32):
    x = torch.randn((rows, K), generator=gen, device="cuda", dtype=torch.float32)
    x[:, torch.randperm(K, generator=gen, device="cuda")[: (K + 99) // 100]] *= 20.0
    return x.to(dtype)


def _weights(gen, rows, K):
    w = torch.randn((rows, K), generator=gen, device="cuda", dtype=torch.float32) * 0.02
    return torch.where(torch.rand(w.shape, generator=gen, device="cuda") < 0.002, w * 6.0, w)


def _quantised(make, rows, K, fmt):
    """Codes and scales of a matrix that is made some rows at a time."""
    step = max(1, (1 << 26) // K)
    parts = [_quantise(make(min(step, rows - r)), fmt) for r in range(0, rows, step)]
    return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def _group_sizes(gen, M, E):
    """How many rows each expert has: a few popular experts, some that nobody asked for."""
    liked = torch.rand(E, generator=gen, device="cuda") + 0.1
    liked = torch.where(torch.rand(E, generator=gen, device="cuda") < 0.1, liked * 4.0, liked)
    liked = torch.where(torch.rand(E, generator=gen, device="cuda") < 0.1, liked * 0.0, liked)
    if not bool(liked.any()):
        liked += 1.0
    chosen = torch.multinomial(liked, M, replacement=True, generator=gen)
    return torch.bincount(chosen, minlength=E)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, K, fmt = case["kind"], case["K"], case["fmt"]
    state = {"case": case, "dtype": TYPES[case["type"]]}
    factor = torch.tensor([NV_FACTOR], device="cuda") if fmt == "nv" else None
    if kind == "quantise":
        rows, top = case["rows"], case["top"]
        if case["mode"] == "swiglu":         # what a product leaves: no outlier channels
            state["X"] = torch.randn((rows, 2 * K), generator=gen, device="cuda").to(TYPES[case["type"]])
        else:
            state["X"] = _activations(gen, -(-rows // top), K, TYPES[case["type"]])
        # (token, choice) pairs in the order of their experts
        state["index"] = torch.randperm(rows, generator=gen, device="cuda").int() if case["mode"] == "gather" else None
        return state
    if kind == "dequantise":
        scale = 1.0 if factor is None else NV_FACTOR
        state["codes"], state["scales"] = _quantised(lambda n: _weights(gen, n, K) * scale, case["rows"], K, fmt)
        state["alpha"] = None if factor is None else 1.0 / factor
        return state
    M, N, E = case["M"], case["N"], case.get("E", 1)
    scale = 1.0 if factor is None else NV_FACTOR
    state["x_codes"], state["x_scales"] = _quantised(lambda n: _activations(gen, n, K), M, K, fmt)
    state["w_codes"], state["w_scales"] = _quantised(lambda n: _weights(gen, n, K) * scale, E * N, K, fmt)
    state["alpha"] = None if factor is None else torch.full((E,), 1.0 / NV_FACTOR, device="cuda")
    if kind == "grouped":
        sizes = _group_sizes(gen, M, E)
        state["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), sizes.cumsum(0)]).int()
        state["largest"] = int(sizes.max())          # known to a program that has just routed its tokens
    return state


def _quantise(y, fmt):
    """fp32 [rows, K] -> codes uint8 [rows, K/2] (even columns in the low halves), scales uint8 [rows, K/block]."""
    rows, K = y.shape
    b = y.reshape(rows, K // BLOCK[fmt], BLOCK[fmt])
    amax = b.abs().amax(2)
    bad = ~torch.isfinite(amax)
    amax = torch.where(bad, torch.zeros_like(amax), amax)
    b = torch.where(bad[..., None], torch.zeros_like(b), b)
    if fmt == "mx":
        # floor(log2(amax)) is the exponent field; the largest E2M1 exponent is 2
        scales = torch.where(bad, 255, ((amax.view(torch.int32) >> 23) - 2).clamp_min(0)).to(torch.uint8)
        v = b.double().abs() * torch.exp2(127.0 - scales.double())[..., None]
    else:
        s = (amax / 6.0).clamp_max(448.0).to(torch.float8_e4m3fn)
        scales = torch.where(bad, 127, s.view(torch.uint8).int()).to(torch.uint8)
        s = s.double()
        v = b.double().abs() / torch.where(s == 0, torch.full_like(s, float("inf")), s)[..., None]
    # nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6; between two, the one with an even code
    code = ((v > 0.25).byte() + (v >= 0.75).byte() + (v > 1.25).byte() + (v >= 1.75).byte() + (v > 2.5).byte()
            + (v >= 3.5).byte() + (v > 5.0).byte())
    code = torch.where(bad[..., None], torch.zeros_like(code), code)
    code = (code + torch.signbit(b).byte() * 8).reshape(rows, K)
    return code[:, 0::2] + code[:, 1::2] * 16, scales.contiguous()


def _values(codes, scales, fmt):
    """fp32 values of codes and scales."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    c = table[torch.stack([codes & 15, codes >> 4], dim=2).int()].reshape(codes.shape[0], -1, BLOCK[fmt])
    if fmt == "mx":
        s = torch.where(scales == 255, torch.full((), float("nan"), device=codes.device), torch.exp2(scales.float() - 127.0))
    else:
        s = scales.view(torch.float8_e4m3fn).float()
    return (c * s[..., None]).reshape(codes.shape[0], -1)


def _own(state, case):
    import paper_2510_19482_b200 as elutq

    fmt = elutq.MX4_MXFP4 if case["fmt"] == "mx" else elutq.MX4_NVFP4
    K = case["K"]
    if case["kind"] == "quantise":
        flags = elutq.MX4_FLAG_SWIGLU if case["mode"] == "swiglu" else 0
        codes, scales = elutq.elutq_mx4_quantize(state["X"], case["rows"], K, fmt, flags=flags, index=state["index"], index_div=case["top"])
        values = torch.empty((case["rows"], K), dtype=torch.bfloat16, device="cuda")
        elutq.elutq_mx4_dequantize(codes, scales, values, case["rows"], K, fmt)
        return values
    if case["kind"] == "dequantise":
        values = torch.empty((case["rows"], K), dtype=state["dtype"], device="cuda")
        elutq.elutq_mx4_dequantize(state["codes"], state["scales"], values, case["rows"], K, fmt, alpha=state["alpha"])
        return values
    M, N = case["M"], case["N"]
    Y = torch.empty((M, N), dtype=state["dtype"], device="cuda")
    if case["kind"] == "gemm":
        elutq.elutq_mx4_gemm(state["x_codes"], state["x_scales"], state["w_codes"], state["w_scales"], Y, M, N, K, fmt, alpha=state["alpha"])
    else:
        elutq.elutq_mx4_gemm_grouped(state["x_codes"], state["x_scales"], state["w_codes"], state["w_scales"], state["offsets"], Y,
                                     M, N, K, case["E"], fmt, alpha=state["alpha"])
    return Y


def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    kind, fmt = case["kind"], case["fmt"]
    if kind == "quantise":
        X = state["X"].float()
        if case["mode"] == "gather":
            X = X[torch.div(state["index"], case["top"], rounding_mode="floor")]
        elif case["mode"] == "swiglu":
            # (64 bits: a value next to a border between two codes)
            g, u = X[:, : case["K"]].double(), X[:, case["K"]:].double()
            X = (g * u / (1.0 + torch.exp(-g))).float()
        return _values(*_quantise(X, fmt), fmt).bfloat16()
    if kind == "dequantise":
        v = _values(state["codes"], state["scales"], fmt)
        return (v if state["alpha"] is None else v * state["alpha"]).to(state["dtype"])
    x = _values(state["x_codes"], state["x_scales"], fmt)
    w = _values(state["w_codes"], state["w_scales"], fmt)
    if kind == "gemm":
        y = x @ w.T
        return (y if state["alpha"] is None else y * state["alpha"]).to(state["dtype"])
    # groups filled up to the largest: one batched product, then the rows that are real
    E, M, off = case["E"], case["M"], state["offsets"].long()
    at = torch.arange(M, device="cuda")
    group = torch.searchsorted(off, at, right=True) - 1
    padded = torch.zeros((E, state["largest"], case["K"]), device="cuda")
    padded[group, at - off[group]] = x
    y = torch.bmm(padded, w.reshape(E, case["N"], case["K"]).transpose(1, 2))[group, at - off[group]]
    return (y if state["alpha"] is None else y * state["alpha"][group][:, None]).to(state["dtype"])


def work(case):
    K, block = case["K"], BLOCK[case["fmt"]]
    row = K / 2 + K / block                          # bytes of a quantised row
    size = {"f16": 2, "bf16": 2, "f32": 4}[case["type"]]
    if case["kind"] == "quantise":
        read = -(-case["rows"] // case["top"]) * K * size * (2 if case["mode"] == "swiglu" else 1)
        return {"bytes": read + case["rows"] * (row + 2 * K), "flops": 0}
    if case["kind"] == "dequantise":
        return {"bytes": case["rows"] * (row + size * K), "flops": 0}
    M, N = case["M"], case["N"]
    # (of the experts' weights, those of experts with rows: about as many as M independent choices reach)
    used = case["E"] * (1.0 - (1.0 - 1.0 / case["E"]) ** M) if case["kind"] == "grouped" else 1
    return {"bytes": (M + used * N) * row + M * N * size, "flops": 2.0 * M * N * K}


def _exact_values(codes, scales, fmt):
    """Values in 64 bits from the fields of the formats: sign, exponent and mantissa."""
    def fields(c):
        e, m = (c >> 1) & 3, c & 1
        v = torch.where(e == 0, m.double() * 0.5, torch.ldexp(1.0 + m.double() * 0.5, e.double() - 1.0))
        return torch.where((c >> 3) > 0, -v, v)
    v = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device=codes.device)
    v[:, 0::2], v[:, 1::2] = fields(codes & 15), fields(codes >> 4)
    if fmt == "mx":
        s = torch.ldexp(torch.ones_like(scales, dtype=torch.float64), scales.double() - 127.0)
    else:
        e, m = (scales >> 3).double(), (scales & 7).double()
        s = torch.where(e == 0, torch.ldexp(m, torch.full_like(e, -9.0)), torch.ldexp(8.0 + m, e - 10.0))
    return v * s.repeat_interleave(BLOCK[fmt], dim=1)


def exact(case, seed):
    state = prepare(case, seed)
    K, fmt = case["K"], case["fmt"]
    if case["kind"] == "quantise":
        x = state["X"].double()
        if state["index"] is not None:
            x = x.index_select(0, state["index"].long() // case["top"])
        if case["mode"] == "swiglu":
            x = torch.sigmoid(x[:, :K]) * x[:, :K] * x[:, K:]
        b = x.reshape(case["rows"], -1, BLOCK[fmt])
        top = b.abs().max(dim=2, keepdim=True).values
        # (frexp: top = f 2^e with 0.5 <= f < 1; a logarithm would be off at powers of two)
        if fmt == "mx":
            s = torch.ldexp(torch.ones_like(top), torch.frexp(top).exponent - 3.0)
        else:
            # E4M3: three bits behind the leading one, no finer than 2^-9
            q = top / 6.0
            unit = torch.ldexp(torch.ones_like(q), (torch.frexp(q).exponent - 1.0).clamp_min(-6.0) - 3.0)
            s = (torch.round(q / unit) * unit).clamp_max(448.0)
        v = torch.where(s > 0, b / s, torch.zeros_like(b)).clamp(-6.0, 6.0)
        unit = torch.where(v.abs() < 2.0, 0.5, torch.where(v.abs() < 4.0, 1.0, 2.0))
        return (torch.round(v / unit) * unit * s).reshape(case["rows"], K)
    alpha = 1.0 if state["alpha"] is None else 1.0 / NV_FACTOR
    if case["kind"] == "dequantise":
        return _exact_values(state["codes"], state["scales"], fmt) * alpha
    x = _exact_values(state["x_codes"], state["x_scales"], fmt)
    N = case["N"]
    if case["kind"] == "gemm":
        return torch.matmul(x, _exact_values(state["w_codes"], state["w_scales"], fmt).T) * alpha
    y = torch.empty((case["M"], N), dtype=torch.float64, device="cuda")
    border = state["offsets"].tolist()
    for e in range(case["E"]):
        w = _exact_values(state["w_codes"][e * N : (e + 1) * N], state["w_scales"][e * N : (e + 1) * N], fmt)
        y[border[e] : border[e + 1]] = x[border[e] : border[e + 1]] @ w.T * alpha
    return y
