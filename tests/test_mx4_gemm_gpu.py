"""Products of microscaled 4-bit matrices against the 64-bit oracle, element by element.

Tolerance: products of codes and scales are exact in fp32.  A sum of K terms in the tensor core is off by at most 2^-23 of the terms'
magnitudes per addition, K * 2^-23 * |X| |W|^T in all; alpha's product adds 2^-24 of the result, the output's rounding half a step (fp16
2^-11, bf16 2^-8 of the result, fp32 2^-24).
"""

import numpy as np
import pytest
import torch

import paper_2510_19482_b200 as elutq
from oracle import mx4

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
STEP = {"f16": 2.0**-11, "bf16": 2.0**-8, "f32": 2.0**-24}


def _matrix(rng, rows, K, fmt):
    codes = rng.integers(0, 256, (rows, K // 2), dtype=np.uint8)
    scales = rng.integers(122, 130, (rows, K // 32)) if fmt == 0 else rng.integers(0, 127, (rows, K // 16))
    return codes, scales.astype(np.uint8)


def _dev(*arrays):
    return [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


def _assert_close(got, want, A, K, out, where=""):
    got = got.double().cpu().numpy()
    tol = K * 2.0**-23 * A + (STEP[out] * 1.001 + 2.0**-23) * np.abs(want) + (2.0**-24 if out == "f16" else 0.0)
    bad = ~(np.abs(got - want) <= tol)
    if out == "f16":
        bad &= ~(np.isinf(got) & (np.abs(want) > 65500.0))
    assert not bad.any(), f"{where}: {int(bad.sum())} of {bad.size} off, first at {np.argwhere(bad)[0]}: got {got[bad][0]}, want {want[bad][0]}"


def _gemm(rng, M, N, K, fmt, out, alpha=None):
    xc, xs = _matrix(rng, M, K, fmt)
    wc, ws = _matrix(rng, N, K, fmt)
    a = None if alpha is None else torch.tensor([alpha], device="cuda")
    Y = torch.full((M, N), float("nan"), dtype=TYPES[out], device="cuda")
    elutq.elutq_mx4_gemm(*_dev(xc, xs, wc, ws), Y, M, N, K, fmt, alpha=a)
    assert elutq.elutq_device_status() == 0
    f = 1.0 if alpha is None else float(np.float32(alpha))
    _assert_close(Y, mx4.matmul(xc, xs, wc, ws, fmt, f), mx4.magnitude(xc, xs, wc, ws, fmt, f), K, out, f"{M} x {N} x {K}")


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("M,N,K", [(1, 128, 256), (1, 1, 32), (2, 7, 64), (3, 129, 96), (8, 128, 512), (8, 300, 288), (9, 131, 1056), (16, 256, 768), (17, 384, 2880),
                                   (27, 500, 1440), (32, 128, 4096), (33, 250, 1024), (64, 1000, 2048), (65, 129, 544)])
def test_small_batches(fmt, M, N, K):
    _gemm(np.random.default_rng(M * N + K + fmt), M, N, K, fmt, "f32")


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("M,N,K", [(100, 257, 512), (128, 128, 256), (129, 300, 800), (200, 1000, 1024), (208, 129, 288), (209, 640, 512), (256, 256, 2048), (257, 385, 320),
                                   (300, 20000, 256), (511, 513, 1056), (512, 1024, 1024), (777, 2500, 512), (1500, 3000, 288), (4096, 512, 256)])
def test_large_batches(fmt, M, N, K):
    _gemm(np.random.default_rng(M * N + K + fmt), M, N, K, fmt, "f32")


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("M,N,K", [(2048, 20000, 1440), (1000, 30000, 1024), (64, 57344, 2048), (16, 40000, 1056)])
def test_many_tiles_and_steps_for_each_sm(fmt, M, N, K):
    """Rings and accumulators used many times over; some of the rows are compared."""
    rng = np.random.default_rng(M + fmt)
    xc, xs = _matrix(rng, M, K, fmt)
    wc, ws = _matrix(rng, N, K, fmt)
    Y = torch.full((M, N), float("nan"), device="cuda")
    elutq.elutq_mx4_gemm(*_dev(xc, xs, wc, ws), Y, M, N, K, fmt)
    assert elutq.elutq_device_status() == 0
    assert not torch.isnan(Y).any()
    rows = np.unique(np.concatenate([[0, M - 1], rng.integers(0, M, 14)]))
    _assert_close(Y[torch.from_numpy(rows).cuda()], mx4.matmul(xc[rows], xs[rows], wc, ws, fmt), mx4.magnitude(xc[rows], xs[rows], wc, ws, fmt), K, "f32")


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("out", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(1, 1000, 1024), (5, 77, 1536), (70, 259, 512), (300, 300, 512), (300, 1048, 512), (128, 1000, 256), (9, 200, 256), (250, 136, 64), (1030, 2056, 96)])
def test_output_types_and_alpha(fmt, out, M, N, K):
    _gemm(np.random.default_rng(M + N + K), M, N, K, fmt, out, alpha=None if fmt == 0 else 0.0037)
    _gemm(np.random.default_rng(M + N + K), M, N, K, fmt, out, alpha=-1.7)


def _grouped(rng, borders, N, K, E, fmt, out, M, alpha=None):
    xc, xs = _matrix(rng, M, K, fmt)
    wc, ws = _matrix(rng, E * N, K, fmt)
    Y = torch.full((M, N), -77.0, dtype=TYPES[out], device="cuda")
    a = None if alpha is None else torch.from_numpy(alpha).cuda()
    elutq.elutq_mx4_gemm_grouped(*_dev(xc, xs, wc, ws), torch.tensor(borders, dtype=torch.int32, device="cuda"), Y, M, N, K, E, fmt, alpha=a)
    assert elutq.elutq_device_status() == 0
    top = 0                                                        # what has been taken
    touched = np.zeros(M, dtype=bool)
    for e in range(E):
        lo = max(min(max(borders[e], 0), M), top)
        hi = min(max(borders[e + 1], 0), M)
        if hi <= lo:
            continue
        top, touched[lo:hi] = hi, True
        f = 1.0 if alpha is None else float(alpha[e])
        w = wc[e * N : (e + 1) * N], ws[e * N : (e + 1) * N]
        _assert_close(Y[lo:hi], mx4.matmul(xc[lo:hi], xs[lo:hi], *w, fmt, f), mx4.magnitude(xc[lo:hi], xs[lo:hi], *w, fmt, f), K, out, f"group {e}")
    assert (Y[torch.from_numpy(~touched).cuda()] == -77.0).all()


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("name,sizes,N,K", [
    ("one row each", [1] * 9, 256, 512), ("most empty", [0, 0, 3, 0, 0, 0, 1, 0], 300, 288), ("one group", [50], 130, 1024), ("all in one", [0, 0, 200, 0], 129, 512),
    ("ragged", [5, 0, 17, 64, 1, 130, 0, 33], 385, 544), ("large", [300, 1, 260, 700], 512, 768), ("many groups", [i % 3 for i in range(100)], 64, 96),
    ("skewed", [900] + [2] * 30, 256, 256), ("nothing", [0, 0, 0], 128, 256), ("a thousand", [1 if i % 97 == 0 else 0 for i in range(1024)], 16, 64)])
def test_groups(fmt, name, sizes, N, K):
    rng = np.random.default_rng(len(sizes) + N)
    borders = [0, *np.cumsum(sizes).tolist()]
    M = max(borders[-1], 1)
    _grouped(rng, borders, N, K, len(sizes), fmt, "f32", M)
    # rows in front of the first group and behind the last one
    _grouped(rng, [b + 3 for b in borders], N, K, len(sizes), fmt, "bf16", M + 11, alpha=rng.standard_normal(len(sizes)).astype(np.float32))


def test_borders_out_of_order_and_out_of_range():
    rng = np.random.default_rng(1)
    for borders in ([0, 20, 10, 30], [-5, 10, 2**31 - 1, 40], [0, 100, 100, 100], [40, 30, 20, 10], [-9, -7, -3, -1], [7, 3, 12, 9]):
        _grouped(rng, borders, 200, 288, 3, 0, "f32", 40)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("M", [1, 70, 300])
def test_nan_scales_stay_in_their_row(fmt, M):
    rng = np.random.default_rng(M)
    N, K = 200, 544
    xc, xs = _matrix(rng, M, K, fmt)
    wc, ws = _matrix(rng, N, K, fmt)
    want, A = mx4.matmul(xc, xs, wc, ws, fmt), mx4.magnitude(xc, xs, wc, ws, fmt)
    nan = 255 if fmt == 0 else 127
    rx, rw = M - 1, 131
    xs[rx, 3] = nan
    ws[rw, -1] = nan
    Y = torch.zeros((M, N), device="cuda")
    elutq.elutq_mx4_gemm(*_dev(xc, xs, wc, ws), Y, M, N, K, fmt)
    got = Y.cpu()
    assert torch.isnan(got[rx]).all() and torch.isnan(got[:, rw]).all()
    keep = np.ones((M, N), dtype=bool)
    keep[rx], keep[:, rw] = False, False
    _assert_close(got[torch.from_numpy(keep)], want[keep], A[keep], K, "f32")


@pytest.mark.parametrize("fmt", [0, 1])
def test_odd_scale_bases_and_extreme_scales(fmt):
    """Scales need no alignment.  E8M0 scales far apart: sums of very different magnitudes."""
    rng = np.random.default_rng(8)
    M, N, K = 40, 150, 512
    xc, xs = _matrix(rng, M, K, fmt)
    wc, ws = _matrix(rng, N, K, fmt)
    if fmt == 0:
        xs[:] = rng.integers(90, 160, xs.shape)
        ws[:] = rng.integers(100, 150, ws.shape)
    want, A = mx4.matmul(xc, xs, wc, ws, fmt), mx4.magnitude(xc, xs, wc, ws, fmt)
    dxc, dwc = _dev(xc, wc)
    for off in range(17):
        odd = []
        for s in (xs, ws):
            buf = torch.zeros(s.size + 32, dtype=torch.uint8, device="cuda")
            buf[off : off + s.size] = torch.from_numpy(s).cuda().reshape(-1)
            odd.append(buf[off : off + s.size])
        Y = torch.full((M, N), float("nan"), device="cuda")
        elutq.elutq_mx4_gemm(dxc, odd[0], dwc, odd[1], Y, M, N, K, fmt)
        _assert_close(Y, want, A, K, "f32", f"offset {off}")


def test_neighbouring_memory_is_left_alone():
    rng = np.random.default_rng(2)
    for M, N in ((1, 130), (13, 129), (130, 257), (300, 129)):
        xc, xs = _matrix(rng, M, 256, 0)
        wc, ws = _matrix(rng, N, 256, 0)
        buf = torch.full((M * N + 512,), float("nan"), dtype=torch.float16, device="cuda")
        Y = buf[256 : 256 + M * N]
        elutq.elutq_mx4_gemm(*_dev(xc, xs, wc, ws), Y, M, N, 256, 0)
        assert torch.isnan(buf[:256]).all() and torch.isnan(buf[256 + M * N :]).all() and not torch.isnan(Y).any()


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (40, 1024, 2048), (600, 1500, 1024)])
def test_the_same_call_gives_the_same_bits_alone_and_beside_another(M, N, K):
    rng = np.random.default_rng(4)
    args = _dev(*_matrix(rng, M, K, 1), *_matrix(rng, N, K, 1))
    first = torch.empty((M, N), device="cuda")
    elutq.elutq_mx4_gemm(*args, first, M, N, K, 1)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.empty((M, N), device="cuda") for _ in range(12)]
    torch.cuda.synchronize()
    for i, y in enumerate(outs):
        elutq.elutq_mx4_gemm(*args, y, M, N, K, 1, stream=streams[i % 3])
    torch.cuda.synchronize()
    assert all(torch.equal(y, first) for y in outs)


def test_an_expert_layer_captured_and_replayed():
    """Gathered rows quantised, the experts' gate and up product, SwiGLU and quantised again, the experts' down product: one graph, new inputs and borders."""
    T, top, E, H, F, fmt = 12, 2, 5, 256, 384, 1
    R = T * top
    gen = torch.Generator(device="cuda").manual_seed(0)
    w1 = elutq.elutq_mx4_quantize(torch.randn((E * 2 * F, H), generator=gen, device="cuda") * 0.1, E * 2 * F, H, fmt)
    w2 = elutq.elutq_mx4_quantize(torch.randn((E * H, F), generator=gen, device="cuda") * 0.1, E * H, F, fmt)
    X = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
    index = torch.zeros(R, dtype=torch.int32, device="cuda")
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    mid, out = torch.empty((R, 2 * F), device="cuda"), torch.empty((R, H), device="cuda")
    xq = [torch.empty((R, H // 2), dtype=torch.uint8, device="cuda"), torch.empty((R, H // 16), dtype=torch.uint8, device="cuda")]
    hq = [torch.empty((R, F // 2), dtype=torch.uint8, device="cuda"), torch.empty((R, F // 16), dtype=torch.uint8, device="cuda")]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        elutq.elutq_mx4_quantize(X, R, H, fmt, codes=xq[0], scales=xq[1], index=index, index_div=top, n_rows=offsets[E:])
        elutq.elutq_mx4_gemm_grouped(*xq, *w1, offsets, mid, R, 2 * F, H, E, fmt)
        elutq.elutq_mx4_quantize(mid, R, F, fmt, codes=hq[0], scales=hq[1], flags=elutq.MX4_FLAG_SWIGLU, n_rows=offsets[E:])
        elutq.elutq_mx4_gemm_grouped(*hq, *w2, offsets, out, R, H, F, E, fmt)
    for seed in range(3):
        rng = np.random.default_rng(seed)
        X.copy_(torch.from_numpy(rng.standard_normal((T, H))))
        expert = rng.integers(0, E, R)
        order = np.argsort(expert, kind="stable")
        taken = R - 3 * seed                       # the last rows are routed nowhere
        sizes = np.bincount(expert[order[:taken]], minlength=E)
        index.copy_(torch.from_numpy(order.astype(np.int32)))
        offsets.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)))
        out.fill_(-5.0)
        graph.replay()
        torch.cuda.synchronize()
        x = X.float().cpu().numpy()[order // top]
        assert np.array_equal(xq[0].cpu().numpy()[:taken], mx4.quantize(x[:taken], fmt)[0])
        # each step against the oracle on what the step before it left
        g = expert[order]
        cpu = lambda pair: [t.cpu().numpy() for t in pair]  # noqa: E731
        for q, w, n, K, y in ((xq, w1, 2 * F, H, mid), (hq, w2, H, F, out)):
            qc, qs, wc, ws = *cpu(q), *cpu(w)
            for r in range(taken):
                mine = slice(g[r] * n, (g[r] + 1) * n)
                a = qc[r : r + 1], qs[r : r + 1], wc[mine], ws[mine]
                _assert_close(y[r : r + 1], mx4.matmul(*a, fmt), mx4.magnitude(*a, fmt), K, "f32", f"row {r}")
        m = mid.cpu().double().numpy()[:taken]
        h = m[:, :F] / (1 + np.exp(-m[:, :F])) * m[:, F:]
        hv = mx4.values(*[c[:taken] for c in cpu(hq)], fmt)
        assert (hv != mx4.values(*mx4.quantize(h.astype(np.float32), fmt), fmt)).mean() < 1e-3
        assert (out[taken:] == -5.0).all()


def test_waits_that_run_out_are_reported():
    rng = np.random.default_rng(3)
    for M, N, K in ((1, 256, 4096), (300, 300, 2048)):
        args = _dev(*_matrix(rng, M, K, 0), *_matrix(rng, N, K, 0))
        Y = torch.empty((M, N), device="cuda")
        elutq.elutq_mx4_test_wait_expiry(*args, Y, M, N, K, 0, 1000)
        assert elutq.elutq_device_status() == 0x7C05
        elutq.elutq_release_scratch()
        assert elutq.elutq_device_status() == 0
        elutq.elutq_mx4_gemm(*args, Y, M, N, K, 0)
        assert elutq.elutq_device_status() == 0
