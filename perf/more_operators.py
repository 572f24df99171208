"""Attention of a serving step, between the q/k/v and the o layer: the operators as cases with inputs, one pass and necessary work.

A case is a plain dict.  Its "kind" says which operator a pass goes through:

  write    queries and keys of new tokens are rotated to their positions, keys and values go into a paged cache; a pass returns
           the rotated queries and what the cache holds for the new tokens
  read     the tokens of sequences, from the pages of a cache to dense rows
  decode   attention of the newest token(s) of every sequence over its part of the cache
  prefill  attention over prompts that lie one behind the other, every token up to itself; "context" tokens of an earlier
           part of the prompt come in front of the keys

Cache formats: "16" = the inputs' type, "e4m3" = 8 bits and a factor for each head, "nvfp4" = 4 bits, E4M3 scales of 16 values and a
factor for each head.  Head layouts are those of the benchmark's merged q/k/v layers (32 or 64 query heads over 8 of 128 values)
and generic ones.  Sequences of a batch have different lengths, which a case fixes: the longest first, the others spread
between it and "shortest" times it.
"""

import math

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # eight requests decode: their new tokens go into a 4-bit cache (launches and latency)
        {"name": "write_decode8", "kind": "write", "fmt": "nvfp4", "type": "f16", "B": 8, "longest": 5000, "shortest": 0.1, "new": 1,
         "Hq": 32, "Hkv": 8, "D": 128, "rot": 128, "interleaved": False, "page": 64},
        # ragged prompts; half of each head is rotated, neighbouring values as pairs
        {"name": "write_prompts", "kind": "write", "fmt": "e4m3", "type": "bf16", "B": 7, "longest": 1001, "shortest": 0.2, "new": 0,
         "Hq": 24, "Hkv": 6, "D": 64, "rot": 32, "interleaved": True, "page": 16},
        # a long prompt of the large model
        {"name": "write_long_prompt", "kind": "write", "fmt": "nvfp4", "type": "bf16", "B": 1, "longest": 16384, "shortest": 1.0, "new": 0,
         "Hq": 64, "Hkv": 8, "D": 128, "rot": 128, "interleaved": False, "page": 64},
        # a few short sequences looked at
        {"name": "read_short", "kind": "read", "fmt": "nvfp4", "type": "f16", "B": 3, "longest": 777, "shortest": 0.2,
         "Hkv": 8, "D": 64, "page": 32},
        # long contexts, to go in front of the next parts of their prompts
        {"name": "read_contexts", "kind": "read", "fmt": "e4m3", "type": "bf16", "B": 4, "longest": 32768, "shortest": 0.7,
         "Hkv": 8, "D": 128, "page": 64},
        # one request decodes, a short conversation
        {"name": "decode1_short", "kind": "decode", "fmt": "16", "type": "f16", "B": 1, "longest": 1000, "shortest": 1.0, "new": 1,
         "Hq": 32, "Hkv": 8, "D": 128, "page": 64},
        # one request of the large model decodes over a long document
        {"name": "decode1_long", "kind": "decode", "fmt": "e4m3", "type": "bf16", "B": 1, "longest": 131072, "shortest": 1.0, "new": 1,
         "Hq": 64, "Hkv": 8, "D": 128, "page": 64},
        # four drafted tokens are looked over at once, odd head layout, ragged batch
        {"name": "decode_drafts", "kind": "decode", "fmt": "nvfp4", "type": "f16", "B": 37, "longest": 6001, "shortest": 0.01, "new": 4,
         "Hq": 15, "Hkv": 5, "D": 64, "page": 16},
        # a serving batch
        {"name": "decode64", "kind": "decode", "fmt": "nvfp4", "type": "bf16", "B": 64, "longest": 16384, "shortest": 0.25, "new": 1,
         "Hq": 32, "Hkv": 8, "D": 128, "page": 64},
        # short prompts of different lengths
        {"name": "prefill_ragged", "kind": "prefill", "type": "f16", "B": 9, "longest": 517, "shortest": 0.05, "context": 0,
         "Hq": 12, "Hkv": 4, "D": 64},
        # the next parts of two prompts, over what came before
        {"name": "prefill_next_part", "kind": "prefill", "type": "bf16", "B": 2, "longest": 1024, "shortest": 0.6, "context": 3500,
         "Hq": 32, "Hkv": 8, "D": 128},
        # a long prompt: the largest work
        {"name": "prefill8192", "kind": "prefill", "type": "bf16", "B": 1, "longest": 8192, "shortest": 1.0, "context": 0,
         "Hq": 32, "Hkv": 8, "D": 128},
    ]


def _log(rng, lo, hi):
    """A whole number, its logarithm uniform over [lo, hi]."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["write", "read", "decode", "decode", "prefill", "prefill"])
    Hkv = rng.choice([1, 2, 4, 5, 8])
    case = {"kind": kind, "type": rng.choice(["f16", "bf16"]), "Hkv": Hkv, "D": rng.choice([64, 128, 128])}
    case["shortest"] = rng.choice([0.01, 0.2, 0.6, 1.0])
    if kind != "read":
        case["Hq"] = Hkv * rng.choice([1, 3, 4, 8])
    if kind == "prefill":
        case["B"] = _log(rng, 1, 16)
        longest = _log(rng, 1, 4096)
        case["context"] = rng.choice([0, 0, _log(rng, 1, 4096)])
        # (the plain form fills every sequence up to the longest)
        while case["B"] * case["Hq"] * longest * (longest + case["context"]) > 1.5e9:
            longest = longest * 3 // 4
        case["longest"] = longest
        return case
    case["fmt"] = rng.choice(["16", "e4m3", "nvfp4"])
    case["page"] = rng.choice([16, 32, 64, 128])
    case["B"] = _log(rng, 1, 96)
    case["longest"] = _log(rng, 1, max(2, min(65536, (524288 if kind == "decode" else 65536) // case["B"])))
    if kind == "write":
        case["new"] = rng.choice([0, 1])             # 0: whole prompts
        case["rot"] = rng.choice([case["D"], case["D"], case["D"] // 2, case["D"] // 4])
        case["interleaved"] = rng.choice([False, True])
    if kind == "decode":
        case["new"] = rng.choice([1, 1, 1, 2, 5])
    return case


def _lengths(case):
    """Lengths of the sequences (of a prompt: its new tokens), the longest first."""
    lo, hi = case["shortest"], case["longest"]
    return [hi] + [max(1, int(hi * (lo + (1.0 - lo) * ((i * 0.6180339887) % 1.0)))) for i in range(1, case["B"])]


def _new(case):
    """Lengths of the sequences that a write or a decoding step sees, the new tokens among them, and the number of new ones of each."""
    lens = _lengths(case)
    return (lens, lens) if case["new"] == 0 else ([n + case["new"] for n in lens], [case["new"]] * len(lens))


def _row_bytes(case):
    D = case["D"]
    return {"16": 2 * D, "e4m3": D, "nvfp4": D // 2 + D // 16}[case["fmt"]]


def _keys(gen, rows, H, D):
    """Keys have some large channels, the same ones in every row of a head."""
    x = torch.randn((rows, H, D), generator=gen, device="cuda")
    big = torch.rand((H, D), generator=gen, device="cuda") < 0.03
    return torch.where(big, x * 6.0, x)


def _offsets(counts):
    return torch.tensor([0] + counts, device="cuda").cumsum(0).int()


def _paged(gen, case, lens, state):
    """Pages in no order, some of them unused; a cache that is full of values (of other requests, or of these)."""
    page, H, D, fmt, B = case["page"], case["Hkv"], case["D"], case["fmt"], case["B"]
    need = [-(-n // page) for n in lens]
    wide = max(need)
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((B, wide), -1, dtype=torch.int32, device="cuda")
    at = torch.arange(wide, device="cuda")[None, :]
    count, start = torch.tensor(need, device="cuda")[:, None], _offsets(need)[:-1].long()[:, None]
    table = torch.where(at < count, order[(start + at).clamp_max(pages - 1)], table)
    state["table"] = table
    state["lens"] = torch.tensor(lens, device="cuda").int()
    state["factors"] = None if fmt == "16" else tuple(
        (torch.rand(H, generator=gen, device="cuda") + 0.5) * f for f in ((0.1, 0.02) if fmt == "e4m3" else (0.05, 0.02)))
    state["cache"] = []
    for i in range(2):
        values = []
        step = max(1, (1 << 26) // (page * H * D))
        for p in range(0, pages, step):
            n = min(step, pages - p)
            x = _keys(gen, n * page, H, D) if i == 0 else torch.randn((n * page, H, D), generator=gen, device="cuda")
            values.append([c.reshape(n, page, H, -1).transpose(1, 2) for c in _stored(x, i, state, case)])
        state["cache"].append([torch.cat(c).contiguous() for c in zip(*values)])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, dtype, H, D = case["kind"], TYPES[case["type"]], case["Hkv"], case["D"]
    state = {"case": case, "dtype": dtype}
    if kind == "prefill":
        lens = _lengths(case)
        Hq, rows, keys = case["Hq"], sum(lens), sum(n + case["context"] for n in lens)
        if case["context"] == 0:                     # what the merged layer leaves, rotated in place: q, k, v side by side
            qkv = torch.cat([torch.randn((rows, Hq, D), generator=gen, device="cuda"), _keys(gen, rows, H, D),
                             torch.randn((rows, H, D), generator=gen, device="cuda")], dim=1).to(dtype)
            state["q"], state["k"], state["v"] = qkv[:, :Hq], qkv[:, Hq : Hq + H], qkv[:, Hq + H :]
        else:
            state["q"] = torch.randn((rows, Hq, D), generator=gen, device="cuda").to(dtype)
            state["k"] = _keys(gen, keys, H, D).to(dtype)
            state["v"] = torch.randn((keys, H, D), generator=gen, device="cuda").to(dtype)
        state["cu_q"], state["cu_k"] = _offsets(lens), _offsets([n + case["context"] for n in lens])
        state["longest_k"] = case["longest"] + case["context"]
        return state
    if kind == "read":
        lens = _lengths(case)
        _paged(gen, case, lens, state)
        state["cu"], state["rows"], state["first"] = _offsets(lens), sum(lens), torch.zeros(case["B"], dtype=torch.int32, device="cuda")
        return state
    lens, new = _new(case)
    _paged(gen, case, lens, state)
    rows, Hq = sum(new), case["Hq"]
    if kind == "decode":
        state["q"] = torch.randn((rows, Hq, D), generator=gen, device="cuda").to(dtype)
        return state
    qkv = torch.cat([torch.randn((rows, Hq, D), generator=gen, device="cuda"), _keys(gen, rows, H, D),
                     torch.randn((rows, H, D), generator=gen, device="cuda")], dim=1).to(dtype)
    state["q"], state["k"], state["v"] = qkv[:, :Hq], qkv[:, Hq : Hq + H], qkv[:, Hq + H :]
    state["cu"], state["rows"] = _offsets(new), rows
    state["first"] = state["lens"] - (state["cu"][1:] - state["cu"][:-1])
    seq = torch.repeat_interleave(torch.arange(case["B"], device="cuda"), torch.tensor(new, device="cuda"))
    pos = state["first"].long()[seq] + torch.arange(rows, device="cuda") - state["cu"].long()[seq]
    state["positions"] = pos.int()
    state["slots"] = (state["table"].long()[seq, pos // case["page"]] * case["page"] + pos % case["page"]).int()
    # cosines and sines of all positions, made once for a model
    f = 500000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])
    angle = torch.arange(max(lens), device="cuda", dtype=torch.float64)[:, None] * f
    state["angles"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    return state


def _stored(x, i, state, case):
    """fp32 [rows, H, D] -> what the cache holds for it, keys (i = 0) or values (1): [values] or [codes] or [codes, scales]."""
    fmt = case["fmt"]
    if fmt == "16":
        return [x.to(state["dtype"])]
    y = x * (1.0 / state["factors"][i])[:, None]
    if fmt == "e4m3":
        return [y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)]
    b = y.reshape(*y.shape[:2], -1, 16)
    amax = b.abs().amax(3)
    bad = ~torch.isfinite(amax)
    amax = torch.where(bad, torch.zeros_like(amax), amax)
    b = torch.where(bad[..., None], torch.zeros_like(b), b)
    s = (amax / 6.0).clamp_max(448.0).to(torch.float8_e4m3fn)
    scales = torch.where(bad, 127, s.view(torch.uint8).int()).to(torch.uint8)
    s = s.double()
    v = b.double().abs() / torch.where(s == 0, torch.full_like(s, float("inf")), s)[..., None]
    # nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6; between two, the one with an even code
    code = ((v > 0.25).byte() + (v >= 0.75).byte() + (v > 1.25).byte() + (v >= 1.75).byte() + (v > 2.5).byte()
            + (v >= 3.5).byte() + (v > 5.0).byte())
    code = torch.where(bad[..., None], torch.zeros_like(code), code)
    code = (code + torch.signbit(b).byte() * 8).reshape(y.shape)
    return [code[..., 0::2] + code[..., 1::2] * 16, scales]


def _values(stored, i, state, case):
    """What is stored -> fp32 values [..., H, D]."""
    fmt = case["fmt"]
    if fmt == "16":
        return stored[0].float()
    if fmt == "e4m3":
        return stored[0].view(torch.float8_e4m3fn).float() * state["factors"][i][:, None]
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device="cuda")
    codes, scales = stored
    c = table[torch.stack([codes & 15, codes >> 4], dim=-1).int()].reshape(*scales.shape, 16)
    v = c * scales.view(torch.float8_e4m3fn).float()[..., None]
    return v.reshape(*codes.shape[:-1], -1) * state["factors"][i][:, None]


def _rotated(x, state, case):
    """fp32 [rows, H, D], the first `rot` values of a head in pairs turned by the angles of the rows' positions."""
    R, t = case["rot"], state["angles"][state["positions"].long()][:, None, :]
    c, s = t[..., : R // 2], t[..., R // 2 :]
    if case["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).reshape(*x.shape[:-1], R)
    else:
        a, b = x[..., : R // 2], x[..., R // 2 : R]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([turned, x[..., R:]], dim=-1)


def _tokens(i, state, case, page, at):
    """fp32 values of the cache's tokens (page, place in the page): [*page.shape, H, D]."""
    return _values([c[page, :, at] for c in state["cache"][i]], i, state, case)


def _places(state, case):
    """Page and place of every row of a read: sequence by sequence, from `first` on."""
    cu, row = state["cu"].long(), torch.arange(state["rows"], device="cuda")
    seq = torch.searchsorted(cu, row, right=True) - 1
    pos = state["first"].long()[seq] + row - cu[seq]
    return state["table"].long()[seq, pos // case["page"]], pos % case["page"]


def _attend(q, k, v, seen):
    """q [B, H, g, n, D], k and v [B, H, m, D], seen (bool) broadcast to [B, 1, 1, n, m] -> [B, H, g, n, D]; nothing seen: zeros."""
    B, H, g, n, D = q.shape
    s = torch.matmul(q.reshape(B, H, g * n, D) * (1.0 / math.sqrt(D)), k.transpose(2, 3)).reshape(B, H, g, n, -1)
    s = s.masked_fill_(~seen, float("-inf"))
    top = s.amax(4, keepdim=True)
    p = s.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = p.sum(4, keepdim=True)
    o = torch.matmul(p.reshape(B, H, g * n, -1), v).reshape(B, H, g, n, D)
    return o / torch.where(total == 0, torch.ones_like(total), total)


def _own(state, case):
    import paper_2510_19482_b200 as elutq

    kind = case["kind"]
    if kind == "prefill":
        out = torch.empty(state["q"].shape, dtype=state["dtype"], device="cuda")
        elutq.elutq_attn_prefill(state["q"], state["k"], state["v"], out, state["cu_q"], state["cu_k"], case["longest"])
        return out
    fmt = {"16": elutq.KV_16, "e4m3": elutq.KV_E4M3, "nvfp4": elutq.KV_NVFP4}[case["fmt"]]
    k, v = state["cache"]
    kf, vf = state["factors"] or (None, None)
    cache = elutq.KvCache(fmt, state["dtype"], k[0], v[0], *(() if len(k) == 1 else (k[1], v[1])), k_factor=kf, v_factor=vf)
    if kind == "decode":
        out = torch.empty(state["q"].shape, dtype=state["dtype"], device="cuda")
        elutq.elutq_attn_decode(cache, state["q"], out, state["table"], state["lens"], case["new"])
        return out
    if kind == "write":
        q = torch.empty(state["q"].shape, dtype=state["dtype"], device="cuda")
        elutq.elutq_kv_write(cache, state["k"], state["v"], state["slots"], q=state["q"], q_out=q, positions=state["positions"],
                             rope=state["angles"], flags=elutq.ROPE_INTERLEAVED if case["interleaved"] else 0)
    keys = torch.empty((state["rows"], case["Hkv"], case["D"]), dtype=state["dtype"], device="cuda")
    values = torch.empty_like(keys)
    elutq.elutq_kv_read(cache, state["table"], state["first"], state["cu"], keys, values)
    return (q, keys, values) if kind == "write" else (keys, values)


def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    kind, dtype, H, D, B = case["kind"], state["dtype"], case["Hkv"], case["D"], case["B"]
    if kind in ("write", "read"):
        if kind == "write":
            q, k = _rotated(state["q"].float(), state, case), _rotated(state["k"].float(), state, case)
            slot = state["slots"].long()
            page, at = slot // case["page"], slot % case["page"]
            for i, x in enumerate((k, state["v"].float())):
                for held, new in zip(state["cache"][i], _stored(x, i, state, case)):
                    held[page, :, at] = new
        page, at = _places(state, case)
        back = tuple(_tokens(i, state, case, page, at).to(dtype) for i in range(2))
        return (q.to(dtype), *back) if kind == "write" else back
    g = case["Hq"] // H
    if kind == "decode":
        n, lens = case["new"], state["lens"].long()
        pos = torch.arange(case["longest"] + n, device="cuda")
        page = state["table"].long()[:, pos // case["page"]]
        there = (pos[None, :] < lens[:, None])
        k, v = (torch.where(there[..., None, None], _tokens(i, state, case, page, (pos % case["page"]).expand_as(page)), 0.0).transpose(1, 2) for i in range(2))
        seen = pos[None, None, :] < (lens[:, None] - n + 1 + torch.arange(n, device="cuda"))[..., None]
        q = state["q"].float().reshape(B, n, H, g, D).permute(0, 2, 3, 1, 4)
        return _attend(q, k, v, seen[:, None, None]).permute(0, 3, 1, 2, 4).reshape(B * n, H * g, D).to(dtype)
    # sequences filled up to the longest: one batched product, then the rows that are real
    cu_q, cu_k = state["cu_q"].long(), state["cu_k"].long()
    nq, nk = cu_q[1:] - cu_q[:-1], cu_k[1:] - cu_k[:-1]
    i, j = torch.arange(case["longest"], device="cuda"), torch.arange(state["longest_k"], device="cuda")
    here, there = i < nq[:, None], j < nk[:, None]
    q = state["q"].float()[torch.where(here, cu_q[:-1, None] + i, 0)].reshape(B, -1, H, g, D).permute(0, 2, 3, 1, 4)
    k, v = (torch.where(there[..., None, None], state[x].float()[torch.where(there, cu_k[:-1, None] + j, 0)], 0.0).transpose(1, 2) for x in "kv")
    seen = (j[None, None, :] <= (nk - nq)[:, None, None] + i[None, :, None]) & there[:, None, :]
    return _attend(q, k, v, seen[:, None, None]).permute(0, 3, 1, 2, 4).reshape(B, -1, H * g, D)[here].to(dtype)


def work(case):
    D, H, size = case["D"], case["Hkv"], 2
    if case["kind"] == "prefill":
        lens = _lengths(case)
        pairs = sum(n * case["context"] + n * (n + 1) // 2 for n in lens)
        rows, keys = sum(lens), sum(n + case["context"] for n in lens)
        return {"bytes": (2 * rows * case["Hq"] + 2 * keys * H) * D * size, "flops": 4.0 * case["Hq"] * D * pairs}
    row = _row_bytes(case)
    if case["kind"] == "read":
        return {"bytes": sum(_lengths(case)) * 2 * H * (row + D * size), "flops": 0}
    lens, new = _new(case)
    if case["kind"] == "write":
        # (what the cache holds now is written, and read back)
        return {"bytes": sum(new) * (2 * case["Hq"] * D * size + 2 * H * (D * size + 2 * row + D * size) + 4 * case["rot"] + 8), "flops": 6.0 * sum(new) * (case["Hq"] + H) * case["rot"] / 2}
    seen = sum(n - case["new"] + 1 + t for n in lens for t in range(case["new"]))
    return {"bytes": sum(lens) * 2 * H * row + 2 * sum(new) * case["Hq"] * D * size, "flops": 4.0 * case["Hq"] * D * seen}


def _exact_values(stored, i, state, fmt):
    """64-bit values from the fields of the formats: sign, exponent and mantissa."""
    if fmt == "16":
        return stored[0].double()

    def e4m3(byte):
        e, m = ((byte >> 3) & 15).double(), (byte & 7).double()
        v = torch.where(e == 0, torch.ldexp(m, torch.full_like(e, -9.0)), torch.ldexp(8.0 + m, e - 10.0))
        return torch.where(byte >= 128, -v, v)

    factor = state["factors"][i].double()[:, None]
    if fmt == "e4m3":
        return e4m3(stored[0].int()) * factor
    codes, scales = stored
    v = torch.empty((*codes.shape[:-1], 2 * codes.shape[-1]), dtype=torch.float64, device="cuda")
    for part, nibble in enumerate((codes & 15, codes >> 4)):
        e, m = ((nibble >> 1) & 3).double(), (nibble & 1).double()
        x = torch.where(e == 0, m * 0.5, torch.ldexp(1.0 + m * 0.5, e - 1.0))
        v[..., part::2] = torch.where(nibble >= 8, -x, x)
    return v * e4m3(scales.int()).repeat_interleave(16, dim=-1) * factor


def _exact_stored(x, factor, fmt):
    """The values that a cache holds for x (64 bits, [rows, H, D]), from the definition of the formats."""
    y = x / factor.double()[:, None]
    def nearest_e4m3(q):                             # three bits behind the leading one, no finer than 2^-9
        unit = torch.ldexp(torch.ones_like(q), (torch.frexp(q).exponent - 1.0).clamp_min(-6.0) - 3.0)
        return (torch.round(q / unit) * unit).clamp(-448.0, 448.0)
    if fmt == "e4m3":
        return nearest_e4m3(y) * factor.double()[:, None]
    b = y.reshape(*y.shape[:2], -1, 16)
    s = nearest_e4m3(b.abs().max(dim=3, keepdim=True).values / 6.0)
    v = torch.where(s > 0, b / s, torch.zeros_like(b)).clamp(-6.0, 6.0)
    unit = torch.where(v.abs() < 2.0, 0.5, torch.where(v.abs() < 4.0, 1.0, 2.0))
    return (torch.round(v / unit) * unit * s).reshape(y.shape) * factor.double()[:, None]


def _exact_rows(q, k, v, shift):
    """One sequence, 64 bits: q [n, Hq, D], k and v [m, H, D]; row i sees the keys up to i + shift."""
    n, Hq, D = q.shape
    m, H, _ = k.shape
    out = torch.zeros((n, Hq, D), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 28) // max(1, m))
    for h in range(Hq):
        kh, vh = k[:, h * H // Hq], v[:, h * H // Hq]
        for r in range(0, n, step):
            row = torch.arange(r, min(n, r + step), device="cuda")
            s = (q[r : r + step, h] @ kh.T) / math.sqrt(D)
            s[torch.arange(m, device="cuda") > (row + shift)[:, None]] = float("-inf")
            w = torch.nan_to_num(torch.softmax(s, dim=1), nan=0.0)
            out[r : r + step, h] = w @ vh
    return out


def exact(case, seed):
    state = prepare(case, seed)
    kind, B = case["kind"], case["B"]
    if kind == "prefill":
        cq, ck = state["cu_q"].tolist(), state["cu_k"].tolist()
        return torch.cat([_exact_rows(state["q"][cq[b] : cq[b + 1]].double(), state["k"][ck[b] : ck[b + 1]].double(), state["v"][ck[b] : ck[b + 1]].double(),
                                      case["context"]) for b in range(B)])
    page, fmt = case["page"], case["fmt"]
    lens, table = state["lens"].tolist(), state["table"].long()
    if kind == "write":
        R, pos = case["rot"], state["positions"].double()
        f = torch.exp(torch.arange(R // 2, device="cuda", dtype=torch.float64) * (-2.0 / R * math.log(500000.0)))
        turn = torch.polar(torch.ones((len(pos), R // 2), dtype=torch.float64, device="cuda"), pos[:, None] * f)[:, None]
        def rotate(x):
            x = x.double()
            pairs = x[..., :R].reshape(*x.shape[:2], R // 2, 2) if case["interleaved"] else x[..., :R].reshape(*x.shape[:2], 2, R // 2).transpose(2, 3)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            z = z if case["interleaved"] else z.transpose(2, 3)
            return torch.cat([z.reshape(*x.shape[:2], R), x[..., R:]], dim=2)
        held = (rotate(state["k"]), state["v"].double())
        if fmt != "16":
            held = tuple(_exact_stored(x, state["factors"][i], fmt) for i, x in enumerate(held))
        return (rotate(state["q"]), *held)

    def sequence(b, i):                              # all tokens of a sequence, page by page
        pages = table[b, : -(-lens[b] // page)]
        held = [c[pages].transpose(1, 2).flatten(0, 1)[: lens[b]] for c in state["cache"][i]]
        return _exact_values(held, i, state, fmt)

    if kind == "read":
        return tuple(torch.cat([sequence(b, i) for b in range(B)]) for i in range(2))
    n = case["new"]
    return torch.cat([_exact_rows(state["q"][b * n : b * n + n].double(), sequence(b, 0), sequence(b, 1), lens[b] - n) for b in range(B)])
