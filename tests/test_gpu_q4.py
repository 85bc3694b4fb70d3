"""Weights in 4 bits against plain forms: the quantiser and its inverse value by value, the product where float32 has to be
exact (integers and powers of two) and where it rounds (against 64 bits, within the roundings that the sums can make)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def spd_mod():
    from paper_2404_08856_amd import spd
    return spd


def to_bf16(x):
    """float32 array rounded to bfloat16 values (nearest, even on ties), NaN kept."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def quantize_ref(w, G):
    """(integers [N, K], scales [N, groups] as bfloat16 values) by the definition, float32 quotients."""
    N, K = w.shape
    groups = (K + G - 1) // G
    q, scales = np.zeros((N, K), dtype=np.int64), np.zeros((N, groups), dtype=np.float32)
    for i in range(groups):
        part = w[:, G * i:G * (i + 1)].astype(np.float32)
        a = np.max(np.abs(part), axis=1)
        fine = np.isfinite(a)
        s = to_bf16(np.where(fine, a, np.float32(0)) * (np.float32(1) / np.float32(7)))
        quot = np.divide(part, s[:, None], out=np.zeros_like(part), where=(fine & (s != 0))[:, None])
        q[:, G * i:G * (i + 1)] = np.clip(np.rint(quot), -8, 7)
        scales[:, i] = np.where(fine, s, np.float32(np.nan))
    return q, scales


def pack_nibbles(q):
    q = np.pad(q & 15, ((0, 0), (0, q.shape[1] % 2)))
    return (q[:, 0::2] | (q[:, 1::2] << 4)).astype(np.uint8)


def device_matrix(q, scales, G):
    """Q4Matrix of integers q [N, K] and bfloat16 scales [N, groups]."""
    return spd_mod().Q4Matrix(torch.from_numpy(pack_nibbles(q)).cuda(), torch.from_numpy(scales).to(torch.bfloat16).cuda(), q.shape[1], G)


def values(q, scales, G):
    return q.astype(np.float64) * np.repeat(scales.astype(np.float64), G, axis=1)[:, :q.shape[1]]


def view(t, pad):
    """t as a view into a buffer `pad` columns wider, NaN beside it."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, :t.shape[1]] = t.cuda()
    return wide[:, :t.shape[1]]


@pytest.mark.parametrize("N,K,G,bf16,pad", [(1, 1, 32, False, 0), (3, 31, 32, True, 1), (16, 64, 64, False, 0), (5, 129, 128, True, 3),
                                            (7, 520, 64, False, 1), (33, 4099, 32, False, 0), (2, 11008, 128, True, 0)])
def test_quantizer_and_its_inverse(N, K, G, bf16, pad):
    spd = spd_mod()
    rng = np.random.default_rng(N * K + G)
    w = (rng.standard_normal((N, K)) * np.exp2(rng.integers(-30, 8, (N, 1)))).astype(np.float32)
    w[:, : min(K, 3)] = 0                                  # (a whole group of zeros where K is that short)
    if bf16:
        w = to_bf16(w)
    dw = view(torch.from_numpy(w).to(torch.bfloat16 if bf16 else torch.float32), pad)
    q = torch.full((N, (K + 1) // 2), 255, dtype=torch.uint8, device="cuda")
    s = torch.full((N, (K + G - 1) // G), -1.0, dtype=torch.bfloat16, device="cuda")
    spd.spd_q4_quantize(dw, G, q, s)
    want_q, want_s = quantize_ref(w, G)
    assert np.array_equal(s.float().cpu().numpy(), want_s)
    assert np.array_equal(q.cpu().numpy(), pack_nibbles(want_q))
    for dtype in (torch.float32, torch.bfloat16):
        out = view(torch.zeros((N, K), dtype=dtype), pad)
        spd.spd_q4_dequantize(q, s, G, out)
        want = values(want_q, want_s, G).astype(np.float32)    # 8 bits times 4 bits: exact
        got = out.float().cpu().numpy()
        assert np.array_equal(got, want if dtype == torch.float32 else to_bf16(want))
        if pad:
            assert torch.isnan(out._base[:, K:].float()).all()


def test_quantizer_groups_that_are_not_finite_zero_or_tiny():
    spd = spd_mod()
    w = np.ones((6, 96), dtype=np.float32)
    w[0, 40] = np.nan
    w[1, 40] = -np.inf
    w[2, 32:64] = 0
    w[3] = 1e-41                                          # a denormal scale
    w[4] = 3.0e38
    w[5, ::2] = 3.5                                        # quotients of a half: to the even integer
    dw = torch.from_numpy(w).cuda()
    q = torch.empty((6, 48), dtype=torch.uint8, device="cuda")
    s = torch.empty((6, 3), dtype=torch.bfloat16, device="cuda")
    spd.spd_q4_quantize(dw, 32, q, s)
    want_q, want_s = quantize_ref(w, 32)
    assert np.array_equal(s.float().cpu().numpy(), want_s, equal_nan=True) and np.isnan(want_s[:2, 1]).all()
    assert np.array_equal(q.cpu().numpy(), pack_nibbles(want_q))


SHAPES = [(1, 16, 32, 32), (1, 1, 1, 32), (2, 17, 127, 64), (3, 40, 128, 128), (4, 16, 129, 32), (5, 100, 256, 128), (6, 48, 1000, 64),
          (8, 256, 1024, 32), (9, 33, 257, 128), (12, 64, 384, 64), (13, 16, 4096, 128), (16, 31, 2049, 32), (17, 272, 640, 128),
          (31, 80, 1152, 64), (40, 528, 515, 32), (64, 65, 3001, 128), (64, 1040, 768, 64), (1, 4112, 1280, 128), (5, 4100, 130, 64)]


# every way that a few rows' digits are held: blocks of K that waves keep (1, 2, 4 each), any K; one row, up to 4, 5, up to 8, up to 12, up to 16
LONG = [(rows, N, K, G) for rows in (1, 3, 5, 7, 11, 14) for N, K, G in ((48, 900, 128), (48, 2000, 64), (4128, 1150, 32), (33, 4100, 128), (64, 5555, 32), (17, 8200, 64), (31, 11008, 128), (16, 17000, 64))]


WIDE = [(7, 4112, 4200, 64), (8, 4112, 4300, 128), (4, 4112, 8300, 128), (2, 8208, 8200, 32), (5, 300, 12400, 64)]     # few rows of matrices that are large both ways


@pytest.mark.parametrize("rows,N,K,G", SHAPES + LONG + WIDE)
@pytest.mark.parametrize("bf16", [False, True])
def test_product_of_integers_is_exact(rows, N, K, G, bf16):
    """Integers up to 60 (15 where K is over 4096) and scales that are powers of two up to 2: every sum is a multiple of 1/4 below 2^22
    (60 * 8 * 2 * 4096 and 15 * 8 * 2 * 17000 are), so float32 has it exactly in any order."""
    spd = spd_mod()
    rng = np.random.default_rng(rows + 7 * N + 31 * K + G)
    top = 60 if K <= 4096 else 15
    x = rng.integers(-top, top + 1, (rows, K)).astype(np.float64)
    x[:, rng.integers(0, K)] = top
    if rows > 2:
        x[1] = 0
    q = rng.integers(-8, 8, (N, K))
    scales = np.exp2(rng.integers(-2, 2, (N, (K + G - 1) // G))).astype(np.float32)
    m = device_matrix(q, scales, G)
    dx = view(torch.from_numpy(x).to(torch.bfloat16 if bf16 else torch.float32), K % 3)
    y = view(torch.full((rows, N), -1.0), N % 2)
    spd.spd_q4_matmul(m, dx, y)
    assert np.array_equal(y.double().cpu().numpy(), x @ values(q, scales, G).T)
    if N % 2:
        assert torch.isnan(y._base[:, N:]).all()


@pytest.mark.parametrize("rows,N,K,G", [(1, 33, 1000, 32), (6, 40, 4500, 128), (20, 64, 3000, 64), (40, 528, 4096, 128), (64, 31, 17000, 32)])
@pytest.mark.parametrize("power", [-88, 88])
def test_scales_far_from_one(rows, N, K, G, power):
    """As above times a power of two that every result bears (2^22 * 2^88; 2^-2 * 2^-88): as exact."""
    spd = spd_mod()
    rng = np.random.default_rng(rows + K)
    x = rng.integers(-15, 16, (rows, K)).astype(np.float64)
    q = rng.integers(-8, 8, (N, K))
    scales = np.exp2(rng.integers(-2, 2, (N, (K + G - 1) // G)) + power).astype(np.float32)
    y = torch.empty((rows, N), device="cuda")
    spd.spd_q4_matmul(device_matrix(q, scales, G), torch.from_numpy(x.astype(np.float32)).cuda(), y)
    assert np.array_equal(y.double().cpu().numpy(), x @ values(q, scales, G).T)


@pytest.mark.parametrize("rows,N,K,G", SHAPES + LONG[::5])
@pytest.mark.parametrize("kind", ["normal", "one-sided", "outliers", "tiny", "huge"])
def test_product_within_its_roundings(rows, N, K, G, kind):
    """Against 64 bits.  A row's digits leave out at most 2^-29 of its largest magnitude per entry; their magnitudes add up to at
    most |x| + 2^-6 of that largest one; a result is the sum of at most groups + 20 numbers, each addition rounding by 2^-24 of a sum of magnitudes."""
    spd = spd_mod()
    rng = np.random.default_rng(rows + 7 * N + 31 * K + G + len(kind))
    x = rng.standard_normal((rows, K))
    if kind == "one-sided":
        x = np.abs(x) + 3
    elif kind == "outliers":
        x[:, rng.integers(0, K, 1 + K // 200)] *= 1000
    elif kind == "tiny":
        x *= 1e-24
    elif kind == "huge":
        x *= 1e33
    x = x.astype(np.float32).astype(np.float64)
    groups = (K + G - 1) // G
    q = np.clip(np.rint(rng.standard_normal((N, K)) * 3), -8, 7).astype(np.int64)
    scales = to_bf16(0.01 * (0.5 + rng.random((N, groups))))
    y = torch.empty((rows, N), dtype=torch.float32, device="cuda")
    spd.spd_q4_matmul(device_matrix(q, scales, G), torch.from_numpy(x.astype(np.float32)).cuda(), y)
    w = values(q, scales, G)
    top = np.max(np.abs(x), axis=1, keepdims=True)
    mass, weight = np.abs(x) @ np.abs(w).T, np.sum(np.abs(w), axis=1)[None]
    tol = (groups + 20) * 2.0 ** -24 * (mass + 2.0 ** -6 * top * weight) + 2.0 ** -29 * top * weight
    assert np.all(np.abs(y.double().cpu().numpy() - x @ w.T) <= tol)


def test_rows_and_features_that_are_not_finite_keep_to_themselves():
    spd = spd_mod()
    rng = np.random.default_rng(5)
    for rows in (3, 12, 40):
        x = rng.integers(-9, 10, (rows, 300)).astype(np.float32)
        q = rng.integers(-8, 8, (35, 300))
        scales = np.ones((35, 10), dtype=np.float32)
        want = (x.astype(np.float64) @ values(q, scales, 32).T)
        x[1, 299], x[2, 0] = np.nan, -np.inf
        scales[20, 3] = np.nan
        y = torch.empty((rows, 35), dtype=torch.float32, device="cuda")
        spd.spd_q4_matmul(device_matrix(q, scales, 32), torch.from_numpy(x).cuda(), y)
        got = y.double().cpu().numpy()
        bad = np.zeros((rows, 35), dtype=bool)
        bad[1:3], bad[:, 20] = True, True
        assert np.isnan(got[bad]).all() and np.array_equal(got[~bad], want[~bad])


def test_calls_on_two_streams_and_a_captured_call():
    """Each call has its own workspace; a captured one is replayed on new inputs with eager calls between the replays."""
    spd = spd_mod()
    rng = np.random.default_rng(9)
    for rows in (5, 40):
        q, scales = rng.integers(-8, 8, (528, 900)), np.ones((528, 8), dtype=np.float32)
        m, w = device_matrix(q, scales, 128), values(q, scales, 128)
        torch.cuda.synchronize()
        new = lambda: rng.integers(-60, 61, (rows, 900)).astype(np.float64)
        streams, outs, xs = [torch.cuda.Stream() for _ in range(2)], [], []
        for s in streams:
            xs.append(new())
            dx = torch.from_numpy(xs[-1]).float().cuda()
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                y = torch.empty((rows, 528), device="cuda")
                for _ in range(3):
                    spd.spd_q4_matmul(m, dx, y)
                outs.append((y, dx))
        torch.cuda.synchronize()
        for x, (y, _) in zip(xs, outs):
            assert np.array_equal(y.double().cpu().numpy(), x @ w.T)
        static, y = torch.zeros((rows, 900), device="cuda"), torch.empty((rows, 528), device="cuda")
        ws = torch.empty(max(1, spd.spd_q4_matmul_workspace_bytes(rows, 528, 900)), dtype=torch.uint8, device="cuda")
        spd.spd_q4_matmul(m, static, y, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            spd.spd_q4_matmul(m, static, y, ws)
        eager = torch.empty_like(y)
        for _ in range(3):
            x = new()
            static.copy_(torch.from_numpy(x).float())
            graph.replay()
            torch.cuda.synchronize()
            assert np.array_equal(y.double().cpu().numpy(), x @ w.T)
            spd.spd_q4_matmul(m, static, eager, ws)
            torch.cuda.synchronize()
            assert torch.equal(eager, y)


@pytest.mark.parametrize("bf16", [False, True])
def test_quantizer_next_to_ties(bf16):
    """Quotients at and next to every half: n + 1/2 times the scale, exactly, one step of float32 below and above, for scales of all magnitudes."""
    spd = spd_mod()
    rng = np.random.default_rng(3)
    rows = []
    for e in list(range(-140, 120, 13)) + [-126, -127, -133]:
        s = to_bf16([np.ldexp(1 + rng.integers(0, 128) / 128, e)])[0]
        half = (np.arange(-7, 7) + 0.5).astype(np.float32) * s
        w = np.concatenate([[7 * s], half, np.nextafter(half, np.float32(np.inf)), np.nextafter(half, np.float32(-np.inf)), np.zeros(64)])[:64]
        rows.append(w.astype(np.float32))
    w = np.stack(rows)
    w = to_bf16(w) if bf16 else w
    q, s = torch.empty((len(w), 32), dtype=torch.uint8, device="cuda"), torch.empty((len(w), 1), dtype=torch.bfloat16, device="cuda")
    spd.spd_q4_quantize(torch.from_numpy(w).to(torch.bfloat16 if bf16 else torch.float32).cuda(), 64, q, s)
    want_q, want_s = quantize_ref(w, 64)
    assert np.array_equal(s.float().cpu().numpy(), want_s) and np.array_equal(q.cpu().numpy(), pack_nibbles(want_q))
