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


@pytest.mark.parametrize("out", ["f16", "bf16"])
@pytest.mark.parametrize("N", [1, 31, 33, 127, 129, 250, 257, 511, 514, 1001, 1003, 1012])
@pytest.mark.parametrize("M", [9, 65, 130, 300])
def test_rows_of_results_that_start_anywhere(out, N, M):
    """16-bit results of every alignment, and what is beside them is left alone."""
    rng = np.random.default_rng(M + N)
    K = 160
    xc, xs = _matrix(rng, M, K, 1)
    wc, ws = _matrix(rng, N, K, 1)
    buf = torch.full((M * N + 64,), float("nan"), dtype=TYPES[out], device="cuda")
    Y = buf[32 : 32 + M * N].reshape(M, N)
    elutq.elutq_mx4_gemm(*_dev(xc, xs, wc, ws), Y, M, N, K, 1, alpha=torch.tensor([0.01], device="cuda"))
    assert torch.isnan(buf[:32]).all() and torch.isnan(buf[32 + M * N :]).all()
    f = float(np.float32(0.01))
    _assert_close(Y, mx4.matmul(xc, xs, wc, ws, 1, f), mx4.magnitude(xc, xs, wc, ws, 1, f), K, out)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("M,N,K", [(3, 40, 32 * 17), (140, 300, 32 * 33), (300, 333, 32 * 101), (40, 130, 32 * 7)])
def test_scales_of_every_alignment(fmt, M, N, K):
    """Rows of an odd number of scales from every base: first and last rows next to memory that is not theirs (NaN scales)."""
    rng = np.random.default_rng(M + K)
    xc, xs = _matrix(rng, M, K, fmt)
    wc, ws = _matrix(rng, N, K, fmt)
    want, A = mx4.matmul(xc, xs, wc, ws, fmt), mx4.magnitude(xc, xs, wc, ws, fmt)
    dxc, dwc = _dev(xc, wc)
    for off in range(0, 18):
        odd = []
        for s in (xs, ws):
            buf = torch.full((s.size + 64,), 255 if fmt == 0 else 127, dtype=torch.uint8, device="cuda")
            buf[off : off + s.size] = torch.from_numpy(s).cuda().reshape(-1)
            odd.append(buf[off : off + s.size])
        Y = torch.full((M, N), float("nan"), device="cuda")
        elutq.elutq_mx4_gemm(dxc, odd[0], dwc, odd[1], Y, M, N, K, fmt)
        _assert_close(Y, want, A, K, "f32", f"offset {off}")


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


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("N", [257, 511, 515, 543, 770])
def test_groups_whose_rows_of_results_start_anywhere(fmt, N):
    """Groups from odd and even rows on, large enough for tiles of two CTAs, in 16 bits."""
    rng = np.random.default_rng(N + fmt)
    borders = [1, 300, 301, 301, 811, 1000]
    _grouped(rng, borders, N, 224, 5, fmt, "bf16", 1003, alpha=rng.standard_normal(5).astype(np.float32))
    _grouped(rng, [b - 1 for b in borders], N, 224, 5, fmt, "f16", 1003, alpha=np.full(5, 2.0**-9, dtype=np.float32))


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("M,N,K", [(66, 130, 4096), (80, 300, 7200), (96, 1000, 3584), (96, 4096, 4128), (150, 257, 2880), (190, 128, 9216)])
def test_clusters_over_many_rows(fmt, M, N, K):
    _gemm(np.random.default_rng(M * N + K + fmt), M, N, K, fmt, "f32")
    _gemm(np.random.default_rng(M * N + K + fmt), M, N, K, fmt, "bf16", alpha=0.37)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("K", [32, 64, 96, 160, 288, 480, 1056, 2144])
def test_groups_with_scales_of_every_alignment(fmt, K):
    """Borders anywhere, rows of few scales: pieces in front of the first and behind the last row belong to others."""
    rng = np.random.default_rng(K + fmt)
    sizes, N = [1, 2, 0, 37, 200], 35
    borders = [0, *np.cumsum(sizes).tolist()]
    M, E = borders[-1], len(sizes)
    xc, xs = _matrix(rng, M, K, fmt)
    wc, ws = _matrix(rng, E * N, K, fmt)
    dxc, dwc, db = *_dev(xc, wc), torch.tensor(borders, dtype=torch.int32, device="cuda")
    for off in (0, 1, 5, 8, 13, 15):
        odd = []
        for s in (xs, ws):
            buf = torch.full((s.size + 64,), 255 if fmt == 0 else 127, dtype=torch.uint8, device="cuda")
            buf[off : off + s.size] = torch.from_numpy(s).cuda().reshape(-1)
            odd.append(buf[off : off + s.size])
        Y = torch.full((M, N), float("nan"), device="cuda")
        elutq.elutq_mx4_gemm_grouped(dxc, odd[0], dwc, odd[1], db, Y, M, N, K, E, fmt)
        for e, (lo, hi) in enumerate(zip(borders, borders[1:])):
            if hi > lo:
                w = wc[e * N : (e + 1) * N], ws[e * N : (e + 1) * N]
                _assert_close(Y[lo:hi], mx4.matmul(xc[lo:hi], xs[lo:hi], *w, fmt, 1.0), mx4.magnitude(xc[lo:hi], xs[lo:hi], *w, fmt, 1.0), K, "f32", f"group {e}, {off}")


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


def test_the_ends_of_the_power_of_two_scales():
    """E8M0 bytes 0 to 254: scales of both operands whose product is 1, or near the ends of fp32."""
    rng = np.random.default_rng(12)
    M, N, K = 9, 140, 128
    xc, _ = _matrix(rng, M, K, 0)
    wc, _ = _matrix(rng, N, K, 0)
    for bx, bw in ((0, 254), (254, 0), (1, 253), (127, 127), (0, 127 + 8), (20, 140), (254, 100), (190, 180)):
        xs, ws = np.full((M, K // 32), bx, dtype=np.uint8), np.full((N, K // 32), bw, dtype=np.uint8)
        Y = torch.full((M, N), float("nan"), device="cuda")
        elutq.elutq_mx4_gemm(*_dev(xc, xs, wc, ws), Y, M, N, K, 0)
        _assert_close(Y, mx4.matmul(xc, xs, wc, ws, 0), mx4.magnitude(xc, xs, wc, ws, 0), K, "f32", f"{bx}, {bw}")


@pytest.mark.parametrize("seed", range(24))
def test_random_calls(seed):
    rng = np.random.default_rng(1000 + seed)

    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    for _ in range(3):
        fmt, out = int(rng.integers(0, 2)), ["f16", "bf16", "f32"][int(rng.integers(0, 3))]
        K = 32 * log(1, 90)
        if rng.random() < 0.5:
            _gemm(rng, log(1, 700), log(1, 3000), K, fmt, out, alpha=None if rng.random() < 0.5 else float(np.exp2(rng.integers(-9, 3))))
        else:
            E = log(1, 60)
            sizes = rng.multinomial(log(1, 900), rng.dirichlet(np.full(E, 0.3)))
            borders = [0, *np.cumsum(sizes).tolist()]
            _grouped(rng, borders, log(1, 700), K, E, fmt, out, max(borders[-1], 1) + int(rng.integers(0, 20)), alpha=np.exp2(rng.integers(-9, 3, E)).astype(np.float32))


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


def test_what_the_binding_turns_down():
    rng = np.random.default_rng(0)
    M, N, K, E = 8, 64, 128, 2
    xc, xs, wc, ws = _dev(*_matrix(rng, M, K, 0), *_matrix(rng, E * N, K, 0))
    Y = torch.zeros((M, N), device="cuda")
    off = torch.tensor([0, 3, 8], dtype=torch.int32, device="cuda")
    X = torch.randn((M, K), device="cuda")
    before = elutq.elutq_launch_count()

    def refused(call):
        with pytest.raises(elutq.ElutqError) as e:
            call()
        assert e.value.status == -1

    def gemm(xc=xc, xs=xs, wc=wc[:N], ws=ws[:N], Y=Y, alpha=None):
        elutq.elutq_mx4_gemm(xc, xs, wc, ws, Y, M, N, K, 0, alpha=alpha)

    def grouped(offsets=off, wc=wc, alpha=None):
        elutq.elutq_mx4_gemm_grouped(xc, xs, wc, ws, offsets, Y, M, N, K, E, 0, alpha=alpha)

    refused(lambda: gemm(xc=xc.cpu()))
    refused(lambda: gemm(Y=Y.cpu()))
    refused(lambda: gemm(xc=xc[:-1]))
    refused(lambda: gemm(ws=ws[:10]))
    refused(lambda: gemm(xs=xs.float()))
    refused(lambda: gemm(Y=Y.double()))
    refused(lambda: gemm(Y=torch.zeros((N, M), device="cuda").T))
    refused(lambda: gemm(alpha=torch.ones(1, dtype=torch.float64, device="cuda")))
    refused(lambda: gemm(wc=wc))
    refused(lambda: gemm(wc=torch.cat([wc, wc], dim=1)[:N, : K // 2]))
    refused(lambda: grouped(offsets=off.long()))
    refused(lambda: grouped(offsets=off[:2]))
    refused(lambda: grouped(wc=wc[:N]))
    refused(lambda: grouped(alpha=torch.ones(1, device="cuda")))
    refused(lambda: elutq.elutq_mx4_quantize(X.cpu(), M, K, 0))
    refused(lambda: elutq.elutq_mx4_quantize(X, M, K, 0, flags=elutq.MX4_FLAG_SWIGLU))
    refused(lambda: elutq.elutq_mx4_quantize(X.T, M, K, 0))
    refused(lambda: elutq.elutq_mx4_quantize(X, M, K, 0, index=torch.zeros(M, dtype=torch.int64, device="cuda")))
    refused(lambda: elutq.elutq_mx4_quantize(X, M, K, 0, n_rows=torch.zeros(1, dtype=torch.int32)))
    refused(lambda: elutq.elutq_mx4_quantize(X, M, K, 0, codes=xc[:-1]))
    refused(lambda: elutq.elutq_mx4_dequantize(xc, xs, Y[:, :32].contiguous(), M, K, 0))
    refused(lambda: elutq.elutq_mx4_quantize(X.double(), M, K, 0))
    assert elutq.elutq_launch_count() == before
    gemm()
    grouped()
    assert elutq.elutq_device_status() == 0


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (40, 3000, 2048), (512, 2048, 1024)])
def test_operands_written_just_before(M, N, K):
    """Weights, activations and factor come from kernels right in front of the product, over and over, with nothing waited for; another product and an HLQ layer
    that has just been packed come behind it."""
    from gpu_util import x_dev
    import workloads
    from oracle import hlq
    from workloads import synth

    gen = torch.Generator(device="cuda").manual_seed(M)
    W = [torch.randn((N, K), generator=gen, device="cuda").bfloat16() for _ in range(3)]
    X = [torch.randn((M, K), generator=gen, device="cuda").bfloat16() for _ in range(3)]
    factors = [0.5, 2.0, -1.0]
    qw, qx = [elutq.elutq_mx4_quantize(w, N, K, 1) for w in W], [elutq.elutq_mx4_quantize(x, M, K, 1) for x in X]
    want = []
    for i in range(3):
        y = torch.empty((M, N), device="cuda")
        elutq.elutq_mx4_gemm(*qx[i], *qw[i], y, M, N, K, 1)
        torch.cuda.synchronize()
        want.append(y * factors[i])
    layers = [workloads.hlq_layer(i, "behind", 2, 128, 512, 1024) for i in range(2)]
    hx = synth.activations(1, "behind/x", 1, 1024)
    planes = [(torch.from_numpy(l.planes).cuda(), *(torch.from_numpy(v.view(np.int16)).cuda().view(torch.float16) for v in (l.scales, l.offsets))) for l in layers]
    packed = elutq.elutq_pack(*planes[0], 2, 128, 512, 1024)
    hxd = x_dev(hx)
    wc, ws, xc, xs, alpha = torch.empty_like(qw[0][0]), torch.empty_like(qw[0][1]), torch.empty_like(qx[0][0]), torch.empty_like(qx[0][1]), torch.empty(1, device="cuda")
    outs, hys = [torch.empty((M, N), device="cuda") for _ in range(12)], [torch.empty((1, 512), dtype=torch.float16, device="cuda") for _ in range(12)]
    torch.cuda.synchronize()
    for k in range(12):
        i = k % 3
        elutq.elutq_pack(*planes[k % 2], 2, 128, 512, 1024, packed=packed)
        elutq.elutq_mx4_quantize(W[i], N, K, 1, codes=wc, scales=ws)
        elutq.elutq_mx4_quantize(X[i], M, K, 1, codes=xc, scales=xs)
        alpha.fill_(factors[i])
        elutq.elutq_mx4_gemm(xc, xs, wc, ws, outs[k], M, N, K, 1, alpha=alpha)
        elutq.elutq_lut_gemm(hxd, packed, hys[k], 1, 512, 1024)
    torch.cuda.synchronize()
    for k in range(12):
        assert torch.equal(outs[k], want[k % 3]), k
        l = layers[k % 2]
        assert hlq.rel_fro_error(hys[k].cpu().numpy(), hlq.matmul(hx, l.planes, l.scales, l.offsets, 128)) <= 1e-3


def test_more_than_2_31_values():
    """Offsets beyond 32 bits: the last rows of large weights, results and inputs."""
    K, N, M = 64, 70_000, 33_000                     # Y: 2.3e9 values
    rng = np.random.default_rng(9)
    xc, xs = _matrix(rng, M, K, 0)
    wc, ws = _matrix(rng, N, K, 0)
    Y = torch.empty((M, N), dtype=torch.float16, device="cuda")
    elutq.elutq_mx4_gemm(*_dev(xc, xs, wc, ws), Y, M, N, K, 0)
    rows = np.array([0, 12_345, M - 2, M - 1])
    part = (xc[rows], xs[rows], wc, ws)
    _assert_close(Y[torch.from_numpy(rows).cuda()], mx4.matmul(*part, 0), mx4.magnitude(*part, 0), K, "f16")
    del Y
    # weights of more than 2^32 values (2^31 bytes of codes), the last rows of which are compared
    K, N, M = 16384, 300_000, 3
    xc, xs = _matrix(rng, M, K, 0)
    gen = torch.Generator(device="cuda").manual_seed(1)
    wc = torch.randint(0, 256, (N, K // 2), generator=gen, dtype=torch.uint8, device="cuda")
    ws = torch.randint(122, 130, (N, K // 32), generator=gen, dtype=torch.uint8, device="cuda")
    Y = torch.empty((M, N), device="cuda")
    elutq.elutq_mx4_gemm(*_dev(xc, xs), wc, ws, Y, M, N, K, 0)
    part = (xc, xs, wc[-300:].cpu().numpy(), ws[-300:].cpu().numpy())
    _assert_close(Y[:, -300:], mx4.matmul(*part, 0), mx4.magnitude(*part, 0), K, "f32")
    # the same bytes back as values and as codes again
    V = torch.empty((N, K), dtype=torch.bfloat16, device="cuda")
    elutq.elutq_mx4_dequantize(wc, ws, V, N, K, 0)
    assert np.array_equal(V[-40:].double().cpu().numpy(), mx4.values(wc[-40:].cpu().numpy(), ws[-40:].cpu().numpy(), 0))
    c2, s2 = elutq.elutq_mx4_quantize(V, N, K, 0)
    want = mx4.quantize(V[-40:].float().cpu().numpy(), 0)
    assert np.array_equal(c2[-40:].cpu().numpy(), want[0]) and np.array_equal(s2[-40:].cpu().numpy(), want[1])
