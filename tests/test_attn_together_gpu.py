"""The attention of a layer as it is used: merged q/k/v linear, rotation and cache, attention over the prompt, over its next part, over single tokens, o linear; captured
and replayed; several streams and threads; caches past 32-bit offsets; sizes drawn at random."""

import threading

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
import workloads
from gpu_util import pack_layer
from kv_util import HALF_STEP, TYPES, Paged, dev, ints, rounded
from oracle import attention, hlq
from test_attn_decode_gpu import check as check_decode
from test_attn_decode_gpu import data
from test_attn_prefill_gpu import check as check_prefill
from test_attn_prefill_gpu import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_a_layer_from_prompt_to_single_tokens(fmt):
    """A small layer (8 query heads over 2 key heads of 64) on HLQ weights: two prompts, a second part of each, then decoding steps."""
    Hq, H, D, K, page = 8, 2, 64, 512, 16
    qkv = workloads.hlq_layer(3, "qkv", 3, 128, (Hq + 2 * H) * D, K)
    o = workloads.hlq_layer(4, "o", 3, 128, K, Hq * D)
    qkv_packed, o_packed = pack_layer(qkv), pack_layer(o)
    rng = np.random.default_rng(fmt)
    parts, steps = ([150, 37], [70, 5]), 3
    lens = [sum(p) for p in zip(*parts)]
    p = Paged(rng, fmt, "f16", [n + steps for n in lens], H, D, page)
    rope = elutq.elutq_rope_table(4096, D, 10000.0, elutq.ROPE_BANDS, factor=8.0)
    table = rope.cpu().numpy()
    k_all, v_all = [[] for _ in lens], [[] for _ in lens]       # rotated keys and values, in 16 bits

    def linear(x, packed, N, rows):
        y = torch.empty((rows, N), dtype=torch.float16, device="cuda")
        elutq.elutq_lut_gemm(x, packed, y, rows, N, x.shape[1])
        return y

    def step(counts, start):
        """Merged rows of new tokens, written and rotated: (rows as made, rotated rows on the device, positions)."""
        rows = sum(counts)
        x = dev(rng.standard_normal((rows, K)) * 0.5, "f16")
        y = linear(x, qkv_packed, (Hq + 2 * H) * D, rows)
        merged = y.clone().view(rows, Hq + 2 * H, D)
        pos = np.concatenate([np.arange(s, s + n) for s, n in zip(start, counts)])
        slots = np.concatenate([p.slots(b, np.arange(s, s + n)) for b, (s, n) in enumerate(zip(start, counts))])
        q, k, v = merged[:, :Hq], merged[:, Hq : Hq + H], merged[:, Hq + H :]
        elutq.elutq_kv_write(p.cache, k, v, ints(slots), q=q, q_out=q, k_out=k, positions=ints(pos), rope=rope)
        made = y.float().cpu().numpy().reshape(rows, Hq + 2 * H, D)
        turned = rounded(attention.rotate(made[:, : Hq + H], table, pos, False), "f16")
        assert np.array_equal(merged.float().cpu().numpy(), np.concatenate([turned, made[:, Hq + H :]], axis=1))
        at = 0
        for b, n in enumerate(counts):
            k_all[b].append(turned[at : at + n, Hq:])
            v_all[b].append(made[at : at + n, Hq + H :])
            at += n
        return turned[:, :Hq], q, k, v, attention.rotate(made[:, Hq : Hq + H], table, pos, False), made[:, Hq + H :], slots

    def kept(exact_k, exact_v, slots):
        """What the oracle says that the cache holds for them."""
        if fmt == 0:
            return rounded(exact_k, "f16").astype(np.float64), exact_v.astype(np.float64)
        return tuple(attention.held(*attention.stored(x, fmt, p.factors[i]), fmt, p.factors[i]) for i, x in enumerate((exact_k, exact_v)))

    held = [[], []], [[], []]
    # the prompts
    tq, q, k, v, ek, ev, slots = step(parts[0], [0, 0])
    out = torch.empty((sum(parts[0]), Hq, D), dtype=torch.float16, device="cuda")
    cu = ints(np.cumsum([0] + list(parts[0])))
    elutq.elutq_attn_prefill(q, k, v, out, cu, cu, max(parts[0]))
    check_prefill(out.double().cpu().numpy(), tq, np.concatenate([x[-1] for x in k_all]), np.concatenate([x[-1] for x in v_all]), list(parts[0]), list(parts[0]), "f16")
    hk, hv = kept(ek, ev, slots)
    for b, (a, z) in enumerate(((0, 150), (150, 187))):
        held[0][b].append(hk[a:z])
        held[1][b].append(hv[a:z])
    # their second parts, over what the cache gives back of the first
    tq, q, k, v, ek, ev, slots = step(parts[1], parts[0])
    total = [a + z for a, z in zip(*parts)]
    back = torch.empty((2, sum(total), H, D), dtype=torch.float16, device="cuda")
    cu_k, first = ints(np.cumsum([0] + total)), None
    elutq.elutq_kv_read(p.cache, p.table_d, first, cu_k, back[0], back[1])
    out = torch.empty((sum(parts[1]), Hq, D), dtype=torch.float16, device="cuda")
    elutq.elutq_attn_prefill(q, back[0], back[1], out, ints(np.cumsum([0] + list(parts[1]))), cu_k, max(parts[1]))
    hk, hv = kept(ek, ev, slots)
    for b, (a, z) in enumerate(((0, 70), (70, 75))):
        held[0][b].append(hk[a:z])
        held[1][b].append(hv[a:z])
    both = [[rounded(np.concatenate(x).astype(np.float32), "f16") for x in h] for h in held]
    assert np.array_equal(back.float().cpu().numpy(), np.stack([np.concatenate(x) for x in both]))
    check_prefill(out.double().cpu().numpy(), tq, np.concatenate(both[0]), np.concatenate(both[1]), list(parts[1]), total, "f16")
    # single tokens
    for n in range(steps):
        tq, q, k, v, ek, ev, slots = step([1, 1], [t + n for t in total])
        hk, hv = kept(ek, ev, slots)
        for b in range(2):
            held[0][b].append(hk[b : b + 1])
            held[1][b].append(hv[b : b + 1])
        out = torch.empty((2, Hq, D), dtype=torch.float16, device="cuda")
        elutq.elutq_attn_decode(p.cache, q, out, p.table_d, ints([t + n + 1 for t in total]))
        p.lens, p.held = [t + n + 1 for t in total], [[np.concatenate(x) for x in h] for h in held]
        check_decode(out.double().cpu().numpy(), p, tq, 1, D ** -0.5, Hq)
        y = linear(out.view(2, Hq * D), o_packed, K, 2)
        ref = hlq.matmul(out.view(2, Hq * D).cpu().numpy(), o.planes, o.scales, o.offsets, 128)
        assert hlq.rel_fro_error(y.cpu().numpy(), ref) <= 1e-3


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("short", [True, False])
def test_captured_and_replayed_with_other_lengths(fmt, short):
    """Lengths, tables, slots and positions are on the device: one graph of a decoding step serves every step.  (Short tables take one launch, long ones two and a workspace.)"""
    rng = np.random.default_rng(fmt)
    Hq, H, D, page, B = 8, 2, 128, 16, 3
    room = 400 if short else 9000
    k, v = data(rng, [room] * B, H, D)
    p = Paged(rng, fmt, "bf16", [room] * B, H, D, page, k, v)
    q = torch.zeros((B, Hq, D), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    lens = ints([0] * B)
    need = elutq.elutq_attn_decode_workspace_bytes(p.cache, p.table.shape[1], B, 1, Hq)
    assert (need == 0) == short
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        elutq.elutq_attn_decode(p.cache, q, out, p.table_d, lens)
    full = [[x.copy() for x in h] for h in p.held]
    for n in ([room, 1, 17], [0, room - 1, 300], [5, 5, 5]):
        x = rounded(rng.standard_normal((B, Hq, D)), "bf16")
        q.copy_(dev(x, "bf16"))
        lens.copy_(ints(n))
        graph.replay()
        p.lens, p.held = n, [[x[:m] for x, m in zip(h, n)] for h in full]
        check_decode(out.double().cpu().numpy(), p, x, 1, D ** -0.5, Hq)


def test_prompts_and_writes_captured_and_replayed():
    rng = np.random.default_rng(1)
    Hq, H, D, rows = 4, 2, 128, 300
    p = Paged(rng, 2, "bf16", [rows], H, D, 16)
    merged = torch.zeros((rows, Hq + 2 * H, D), dtype=torch.bfloat16, device="cuda")
    q, k, v = merged[:, :Hq], merged[:, Hq : Hq + H], merged[:, Hq + H :]
    out, kr, vr = torch.zeros_like(q.contiguous()), torch.zeros((rows, H, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((rows, H, D), dtype=torch.bfloat16, device="cuda")
    whole = ints([0, rows])
    cu, slots, positions = ints([0, 100, rows]), ints(p.slots(0, np.arange(rows))), ints(np.arange(rows))
    rope = elutq.elutq_rope_table(rows, D)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        elutq.elutq_kv_write(p.cache, k, v, slots, q=q, q_out=q, k_out=k, positions=positions, rope=rope)
        elutq.elutq_attn_prefill(q, k, v, out, cu, cu, 256)
        elutq.elutq_kv_read(p.cache, p.table_d, None, whole, kr, vr)
    for borders in ([0, 100, rows], [0, 255, rows], [0, 256, 256]):
        x = rounded(rng.standard_normal((rows, Hq + 2 * H, D)), "bf16")
        merged.copy_(dev(x, "bf16"))
        cu.copy_(ints(borders))
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        turned = rounded(attention.rotate(x[:, : Hq + H], rope.cpu().numpy(), np.arange(rows), False), "bf16")
        n = list(np.diff(borders))
        m = borders[-1]
        check_prefill(out.double().cpu().numpy()[:m], turned[:m, :Hq], turned[:m, Hq:], x[:m, Hq + H :], n, n, "bf16")
        assert (out[m:] == 3).all()
        stored = [attention.stored(y, 2, p.factors[i]) for i, y in enumerate((attention.rotate(x[:, Hq : Hq + H], rope.cpu().numpy(), np.arange(rows), False), x[:, Hq + H :]))]
        for i, got in enumerate((kr, vr)):
            assert np.array_equal(got.float().cpu().numpy(), rounded(attention.held(*stored[i], 2, p.factors[i]).astype(np.float32), "bf16"))


@pytest.mark.parametrize("fmt", [0, 2])
def test_several_threads_and_streams(fmt):
    """Two calls at once, each on a stream of its own with a workspace of its own, give what they give alone."""
    rng = np.random.default_rng(fmt)
    lens, H, Hq, D = [6000, 20, 3000], 2, 8, 128
    ps = [Paged(np.random.default_rng(s), fmt, "f16", lens, H, D, 16, *data(np.random.default_rng(s), lens, H, D)) for s in range(2)]
    qs = [dev(rounded(rng.standard_normal((3, Hq, D)), "f16"), "f16") for _ in range(2)]
    qp, kp, vp = zip(*[[dev(x, "f16") for x in make(np.random.default_rng(s), [700], [700], Hq, H, D, "f16")] for s in range(2)])
    cu = ints([0, 700])
    want = []
    for i in range(2):
        d, r = torch.empty_like(qs[i]), torch.empty_like(qp[i])
        elutq.elutq_attn_decode(ps[i].cache, qs[i], d, ps[i].table_d, ps[i].lens_d)
        elutq.elutq_attn_prefill(qp[i], kp[i], vp[i], r, cu, cu, 700)
        want.append((d, r))
    torch.cuda.synchronize()
    errors = []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            ws = torch.empty(elutq.elutq_attn_decode_workspace_bytes(ps[i].cache, ps[i].table.shape[1], 3, 1, Hq), dtype=torch.uint8, device="cuda")
            d, r = torch.empty_like(qs[i]), torch.empty_like(qp[i])
            stream.wait_stream(torch.cuda.default_stream())
            for _ in range(30):
                elutq.elutq_attn_decode(ps[i].cache, qs[i], d, ps[i].table_d, ps[i].lens_d, workspace=ws, stream=stream)
                elutq.elutq_attn_prefill(qp[i], kp[i], vp[i], r, cu, cu, 700, stream=stream)
            stream.synchronize()
            assert torch.equal(d, want[i][0]) and torch.equal(r, want[i][1])
        except Exception as ex:
            errors.append(ex)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    with pytest.raises(elutq.ElutqError):                 # a stream of one's own without a workspace
        elutq.elutq_attn_decode(ps[0].cache, qs[0], torch.empty_like(qs[0]), ps[0].table_d, ps[0].lens_d, stream=torch.cuda.Stream())


def test_a_cache_past_32_bits():
    """Pages behind 4 GiB of keys."""
    rng = np.random.default_rng(0)
    H, D, page, pages = 8, 128, 64, 36000                 # 131072 bytes a page: 4.7 GB
    k, v = (torch.zeros((pages, H, page, D), dtype=torch.float16, device="cuda") for _ in range(2))
    cache = elutq.KvCache(elutq.KV_16, torch.float16, k, v)
    n = 150
    far = [pages - 1, 3, pages - 2]
    x = [rounded(rng.standard_normal((n, H, D)), "f16") for _ in range(2)]
    pos = np.arange(n)
    slots = np.array(far)[pos // page] * page + pos % page
    elutq.elutq_kv_write(cache, dev(x[0], "f16"), dev(x[1], "f16"), ints(slots))
    back = torch.empty((2, n, H, D), dtype=torch.float16, device="cuda")
    table = ints([far])
    elutq.elutq_kv_read(cache, table, None, ints([0, n]), back[0], back[1])
    assert np.array_equal(back.float().cpu().numpy(), np.stack(x))
    q = rounded(rng.standard_normal((1, H, D)), "f16")
    out = torch.empty((1, H, D), dtype=torch.float16, device="cuda")
    elutq.elutq_attn_decode(cache, dev(q, "f16"), out, table, ints([n]))
    want, mag, span, big = attention.attend(q, x[0], x[1], D ** -0.5, [n])
    assert (np.abs(out.double().cpu().numpy() - want) <= attention.tolerance(want, mag, span, big, D, n, HALF_STEP["f16"], HALF_STEP["f16"])).all()


def test_rows_past_32_bits():
    """Dense rows whose offsets pass 2^32 bytes: few tokens, far apart."""
    rng = np.random.default_rng(0)
    Hq, H, D, n, ld = 2, 1, 64, 70, 1 << 25               # 64 MB from token to token
    q, k, v = make(rng, [n], [n], Hq, H, D, "bf16")
    wide = torch.zeros(n * ld, dtype=torch.bfloat16, device="cuda")
    views = [torch.as_strided(wide, (n, h, D), (ld, D, 1), at) for h, at in ((Hq, 0), (H, 256), (H, 512), (Hq, 1024))]
    for view, x in zip(views, (q, k, v)):
        view.copy_(dev(x, "bf16"))
    cu = ints([0, n])
    elutq.elutq_attn_prefill(views[0], views[1], views[2], views[3], cu, cu, n)
    check_prefill(views[3].double().cpu().numpy(), q, k, v, [n], [n], "bf16")


@pytest.mark.parametrize("seed", range(24))
def test_random_sizes(seed):
    rng = np.random.default_rng(1000 + seed)
    fmt, dtype, D = int(rng.integers(0, 3)), ["f16", "bf16"][seed % 2], int(rng.choice([64, 128]))
    H, group, new = int(rng.integers(1, 9)), int(rng.integers(1, 9)), int(rng.choice([1, 1, 2, 3, 7]))
    page, B = 16 * int(rng.integers(1, 9)), int(np.exp(rng.uniform(0, np.log(40))))
    longest = int(np.exp(rng.uniform(0, np.log(40000 / B))))
    lens = [int(x) for x in rng.integers(0, longest + 1, B)]
    p = Paged(rng, fmt, dtype, lens, H, D, page, *data(rng, lens, H, D))
    q = rounded(rng.standard_normal((B * new, H * group, D)), dtype)
    out = torch.full((B * new, H * group, D), float("nan"), dtype=TYPES[dtype], device="cuda")
    elutq.elutq_attn_decode(p.cache, dev(q, dtype), out, p.table_d, p.lens_d, new)
    check_decode(out.double().cpu().numpy(), p, q, new, D ** -0.5, H * group)
    # a prompt of the same heads
    counts = [int(x) for x in rng.integers(0, 300, int(rng.integers(1, 6)))] + [1]
    keys = [max(0, n + int(rng.integers(-20, 200))) for n in counts]
    if sum(keys) == 0:
        keys[0] = 1
    q, k, v = make(rng, counts, keys, H * group, H, D, dtype)
    out = torch.full(q.shape, float("nan"), dtype=TYPES[dtype], device="cuda")
    elutq.elutq_attn_prefill(dev(q, dtype), dev(k, dtype), dev(v, dtype), out, ints(np.cumsum([0] + counts)), ints(np.cumsum([0] + keys)), max(counts) + int(rng.integers(0, 300)),
                             causal=bool(seed % 3))
    check_prefill(out.double().cpu().numpy(), q, k, v, counts, keys, dtype, causal=bool(seed % 3), rows=[0, 1, 50, 127, 128, 129, 255, 256, 298])
