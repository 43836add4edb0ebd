"""Products with 8-bit activations on the GPU (``matmul_fp8``,
``dequant_matmul_fp8``) against the oracle's numbers multiplied in float64.

Operands are given in 8 bits, so what may differ is the sums.
  * Every product enters exactly and sums are float32: m products and two
    operations on each of the ceil(m / 128) blocks round at most (m + 2 G)
    times, 2^-24 of the magnitudes each.
  * Results in 16 bits round once more, by half a step: 2^-11 (float16, or
    2^-25 below its normal range), 2^-8 (bfloat16).
  * Results in 16 bits of products in tiles come from the matrix cores' 8-bit
    products.  These add eight neighbouring products after cutting each, towards
    zero, to a multiple of 2^(E - 13), E the largest sum of the two factors'
    exponents among the eight (an exponent is at least -6, the subnormals' and
    zero's; measured on gfx950 with products of powers of two beside a larger
    one), and add the sums of eights cut at 2^-23 of the largest.  Seven of
    eight products lose less than 2^(E - 13) each (the largest's 8 bits stay),
    and sixteen eights 2^(E' - 23) each, so an eight's share is below 8 x 2^(E -
    13) plus 16 x 2^-23 of the magnitudes a block.
"""

import numpy as np
import pytest
import torch

import paper_2602_08376_amd as ok
from oracle import fp8 as o8
from oracle import infer as oi

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ok.library()


def in_tiles(n, T):
    """Whether the sizes may be beyond the kernel for few tokens."""
    return T > 32 and -(-n // 32) * -(-T // 32) > 1280


def leading(v, scale):
    """2^exponent of e4m3 values times their scales."""
    e = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    return gpu(np.exp2(e) * scale)


def gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def check(Y, W, X, tokens_first=False):
    """Y against W X, both (what they stand for, e4m3 values) in host arrays."""
    (W, w), (X, x) = W, X
    (n, m), T = W.shape, X.shape[0]
    Y = Y.t() if tokens_first else Y
    got, ref = Y.double(), gpu(W) @ gpu(X).t()
    a = gpu(np.abs(W)) @ gpu(np.abs(X)).t()
    b = (m + 2 * -(-m // 128)) * 2.0 ** -24 * a
    # operands below float32's normal range (which is bfloat16's) may count as 0:
    # each is off by less than 2^-126 then
    b += 2.0 ** -126 * (gpu(np.abs(W)) @ gpu((np.abs(X) < 2.0 ** -126).astype(np.float64)).t())
    b += 2.0 ** -126 * (gpu((np.abs(W) < 2.0 ** -126).astype(np.float64)) @ gpu(np.abs(X)).t())
    if Y.dtype != torch.float32:
        if in_tiles(n, T):
            def per(v, u):              # a value's scale: what it stands for over it
                return np.divide(v, u, out=np.ones_like(v), where=u != 0)

            # (a zero's scale: that of its block)
            sw, sx = (np.maximum.reduceat(np.where(u != 0, np.abs(per(v, u)), 0.0), np.arange(0, m, 128), axis=1)
                      .repeat(128, 1)[:, :m] for v, u in ((W, w), (X, x)))
            lw, lx = leading(w, sw), leading(x, sx)
            for k in range(0, m, 8):
                most = torch.zeros_like(a)
                for i in range(k, min(m, k + 8)):
                    most = torch.maximum(most, torch.outer(lw[:, i], lx[:, i]))
                b += 8 * 2.0 ** -13 * most
            b += 16 * 2.0 ** -23 * a
        b += (2.0 ** -11 if Y.dtype == torch.float16 else 2.0 ** -8) * (ref.abs() + b)
        if Y.dtype == torch.float16:
            b += 2.0 ** -25
            # from 65520 on, half a step above the largest number, a result
            # rounds to infinity
            over = got.isinf()
            assert bool((got.sign() * ref + b)[over].ge(65520.0).all())
            got, ref = got.masked_fill(over, 0.0), ref.masked_fill(over, 0.0)
    err = (got - ref).abs()
    worst = float((err / (b + 1e-300)).max())
    print(f"max err / bound {worst:.3f}")
    assert bool((err <= b).all()), worst


def eight_bits(rows, m, seed, block_rows=1, pad=0, spread=2.0):
    """An 8-bit array on the GPU whose rows have NaN behind their last value and
    end with the storage, its scales likewise; and what it stands for."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, m)) * np.exp(spread * rng.standard_normal((1, m)))
    v, e = o8.quantize(x, block_rows)
    m16, G4 = -(-m // 16) * 16, -(-e.shape[1] // 4) * 4
    ld, lds = m16 + 16 * pad, G4 + 4 * pad
    buf = torch.full(((rows - 1) * ld + m16,), 0x7F, dtype=torch.uint8, device=DEV)
    V = torch.as_strided(buf, (rows, m), (ld, 1)).view(torch.float8_e4m3fn)
    V.copy_(torch.from_numpy(v).float().to(torch.float8_e4m3fn))
    sb = torch.full(((e.shape[0] - 1) * lds + G4,), 0xFF, dtype=torch.uint8, device=DEV)
    S = torch.as_strided(sb, e.shape, (lds, 1))
    S.copy_(torch.from_numpy((e + 127).astype(np.uint8)))
    return V, S.view(torch.float8_e8m0fnu), o8.dequantize(v, e, block_rows), v


SIZES = [(1, 1, 1), (5, 3, 2), (16, 128, 16), (17, 129, 1), (16, 127, 15), (33, 1000, 17), (40, 300, 7), (130, 640, 33),
         (257, 1025, 1), (64, 4096, 3), (300, 2500, 65), (8193, 256, 20), (4100, 200, 130), (16400, 136, 9),
         (2100, 144, 1003), (600, 784, 600), (2100, 1100, 1003), (4300, 200, 4100), (4352, 1296, 4097),
         (300, 700, 4500), (33000, 260, 40)]


@pytest.mark.parametrize("y", list(TYPES))
@pytest.mark.parametrize("n,m,T", SIZES)
@pytest.mark.parametrize("rows,scales,tokens_first", [(128, "e8m0", False), (128, "f32", True), (1, "e8m0", True),
                                                      (1, "f32", False)])
def test_matmul(n, m, T, rows, scales, tokens_first, y):
    pad = (n + T) % 3
    W8, ws, W, w = eight_bits(n, m, n + m, rows, pad, spread=1.0)
    X8, xs, X, x = eight_bits(T, m, T + m, 1, pad)
    if scales == "f32":
        ws = ws.float() * (1 + torch.rand(ws.shape, device=DEV))
        W = w * o8.expand(ws.double().cpu().numpy(), n, m, rows)
    Y = ok.matmul_fp8(W8, ws, X8, xs, tokens_first=tokens_first, dtype=TYPES[y])
    assert Y.dtype == TYPES[y] and Y.shape == ((T, n) if tokens_first else (n, T))
    check(Y, (W, w), (X, x), tokens_first)


def codes(n, m, bits, group, seed):
    rng = np.random.default_rng(seed)
    g = m if group <= 0 or group >= m else group
    G = -(-m // g)
    q = rng.integers(0, 1 << bits, size=(n, m), dtype=np.uint8)
    S = (0.01 * np.exp(rng.standard_normal((n, G)))).astype(np.float32)
    Z = rng.integers(0, 1 << bits, size=(n, G)).astype(np.float32)
    w = q - np.repeat(Z, g, 1)[:, :m].astype(np.float64)
    P = torch.from_numpy(q).to(DEV)
    return (ok.pack_codes(P, bits), torch.from_numpy(S).to(DEV), torch.from_numpy(Z).to(DEV),
            (np.repeat(S.astype(np.float64), g, 1)[:, :m] * w, w))


@pytest.mark.parametrize("y,tokens_first", [("f32", False), ("f32", True), ("f16", False), ("bf16", True)])
@pytest.mark.parametrize("n,m,T,group", [(1, 1, 1, 0), (5, 3, 2, 0), (16, 128, 16, 128), (17, 129, 1, 128), (16, 127, 15, 0),
                                         (33, 1000, 17, 128), (40, 300, 7, 256), (130, 640, 33, 0), (257, 1025, 1, 384),
                                         (300, 2500, 65, 128), (8193, 256, 20, 128), (16400, 136, 9, 0),
                                         (2100, 144, 1003, 128), (600, 784, 600, 256), (2100, 1100, 1003, 512),
                                         (4352, 1296, 4097, 128), (4300, 200, 4100, 0),
                                         (33000, 260, 40, 128), (300, 700, 6500, 128)])
@pytest.mark.parametrize("bits", [1, 2, 3, 4])
def test_dequant_matmul(n, m, T, group, bits, y, tokens_first):
    P, S, Z, W = codes(n, m, bits, group, n + m + bits)
    X8, xs, *X = eight_bits(T, m, T + m, 1, (n + T) % 3)
    Y = ok.dequant_matmul_fp8(P, S, Z, m, bits, group, X8, xs, tokens_first=tokens_first, dtype=TYPES[y])
    assert Y.dtype == TYPES[y] and Y.shape == ((T, n) if tokens_first else (n, T))
    check(Y, W, X, tokens_first)


@pytest.mark.parametrize("T", [1, 5, 40, 700, 9000])
def test_every_e4m3_value_and_scale(T):
    # one feature holds each value of the format on both sides, the other blocks
    # nothing; scales over their whole range, products inside float32's
    m = 256
    W8 = torch.zeros(256, m, dtype=torch.uint8, device=DEV)
    W8[:, 5] = torch.arange(256, dtype=torch.uint8, device=DEV)
    X8 = torch.zeros(T, m, dtype=torch.uint8, device=DEV)
    X8[:, 5] = (torch.arange(T, device=DEV) * 7 % 256).to(torch.uint8)
    xs = torch.full((T, 4), 127, dtype=torch.uint8, device=DEV)
    xs[:, 0] = (torch.arange(T, device=DEV) * 37 % 100 + 80).to(torch.uint8)
    w = torch.full((2, 4), 127, dtype=torch.uint8, device=DEV)
    w[1] = 60
    f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    want = torch.outer(W8[:, 5].view(f8).double() * torch.where(torch.arange(256, device=DEV) < 128, 1.0, 2.0 ** -67),
                       X8[:, 5].view(f8).double() * xs[:, 0].view(e8).double()).float()
    for ws in (w.view(e8)[:, :2], w.view(e8)[:, :2].float()):
        Y = ok.matmul_fp8(W8.view(f8), ws, X8.view(f8), xs.view(e8)[:, :2])
        # a NaN times another row's zero is a NaN too, but only in its own row and column
        bad = W8[:, 5].view(f8).isnan()[:, None] | X8[:, 5].view(f8).isnan()[None, :]
        assert torch.equal(Y.isnan(), bad)
        assert torch.equal(Y[~bad], want[~bad])


def test_slices_of_rows_and_features():
    W8, ws, W, w = eight_bits(200, 520, 1, 1, 2)
    X8, xs, X, x = eight_bits(90, 520, 2, 1, 1)
    for r, k in ((slice(7, 71), 520), (slice(1, 2), 384), (slice(0, 90), 130), (slice(89, 90), 5)):
        G = -(-k // 128)
        Y = ok.matmul_fp8(W8[3:150, :k], ws[3:150, :G], X8[r, :k], xs[r, :G])
        check(Y, (W[3:150, :k], w[3:150, :k]), (X[r, :k], x[r, :k]))


def test_zeros_are_rounded_into_the_box():
    P, S, Z, _ = codes(40, 256, 3, 128, 3)
    X8, xs, _, _ = eight_bits(9, 256, 4)
    want = ok.dequant_matmul_fp8(P, S, Z, 256, 3, 128, X8, xs)
    assert torch.equal(ok.dequant_matmul_fp8(P, S, Z + 0.25, 256, 3, 128, X8, xs), want)
    Z[0], Z[1] = 0.0, 7.0
    want = ok.dequant_matmul_fp8(P, S, Z, 256, 3, 128, X8, xs)
    Z[0], Z[1] = -3.0, 1e30
    assert torch.equal(ok.dequant_matmul_fp8(P, S, Z, 256, 3, 128, X8, xs), want)


@pytest.mark.parametrize("T", [1, 300])
def test_chain_norm_product_norm(T):
    """A layer as a program runs it: norm of the stream, product, its result
    added to the stream by the next norm, codes product on that; against the
    oracle at each step on the GPU's own inputs."""
    m, n, bits = 640, 384, 4
    rng = np.random.default_rng(T)
    stream = torch.from_numpy(rng.standard_normal((T, m)).astype(np.float32)).to(DEV)
    x0 = torch.zeros_like(stream)
    gain = torch.ones(m, device=DEV)
    X8, xs = ok.rmsnorm_fp8(x0, gain, 1e-5, residual=stream)
    W8, ws = ok.quantize_fp8(torch.from_numpy(0.05 * rng.standard_normal((m, m))).float().to(DEV), block_rows=128)
    Y = ok.matmul_fp8(W8, ws, X8, xs, tokens_first=True, dtype=torch.bfloat16)
    X8b, xsb = ok.rmsnorm_fp8(Y, gain, 1e-5, residual=stream)
    P, S, Z, W = codes(n, m, bits, 128, 5)
    out = ok.dequant_matmul_fp8(P, S, Z, m, bits, 128, X8b, xsb)

    def wide(v, s, rows=1):
        v, e = v.double().cpu().numpy(), s.view(torch.uint8).cpu().numpy().astype(np.int64) - 127
        return o8.dequantize(v, e, rows), v

    check(Y, wide(W8, ws, 128), wide(X8, xs), True)
    y, _ = o8.rmsnorm(stream.cpu().numpy(), None, None, 1e-5)
    assert np.array_equal(o8.dequantize(*o8.quantize(y)), wide(X8b, xsb)[0])   # the stream holds h itself: float32
    check(out, W, wide(X8b, xsb))


@pytest.mark.parametrize("T", [1, 24, 700])
def test_streams_and_graphs(T):
    X8, xs, _, _ = eight_bits(T, 520, 1)
    W8, ws, _, _ = eight_bits(300, 520, 2, 128)
    P, S, Z, _ = codes(300, 520, 4, 128, 3)

    def both():
        return (ok.matmul_fp8(W8, ws, X8, xs, dtype=torch.bfloat16, tokens_first=True),
                ok.dequant_matmul_fp8(P, S, Z, 520, 4, 128, X8, xs))

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g, h = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a = both()
    with torch.cuda.graph(h):
        b = both()
    for i in range(4):
        if i == 2:
            X8.copy_(X8.float().mul(0.5).to(X8.dtype))
            want = both()
        g.replay()
        h.replay()
        torch.cuda.synchronize()
        torch.ones(100, device=DEV).sum().item()
        assert all(torch.equal(p, q) for p, q in zip(a, want)), i
        assert all(torch.equal(p, q) for p, q in zip(b, want)), i


@pytest.mark.parametrize("n,T", [(300, 5), (2100, 1003), (4300, 4100)])
@pytest.mark.parametrize("y", ["f32", "bf16"])
def test_ends_of_the_scales(n, T, y):
    # activations at the smallest scale and near the largest, weights that bring
    # them back towards 1 (448 times a weight's scale is a float32)
    m = 256
    X8, xs, X, x = eight_bits(T, m, 1)
    W8, ws, W, w = eight_bits(n, m, 2, 128)
    for code in (0, 1, 3, 240, 246):
        xs.view(torch.uint8).fill_(code)
        up = 2.0 ** min(127 - code, 119)
        Y = ok.matmul_fp8(W8, torch.full(ws.shape, up, device=DEV), X8, xs, dtype=TYPES[y])
        check(Y, (w * up, w), (x * 2.0 ** (code - 127), x))


def test_oracles_weights_are_the_layers():
    # S (Q - Z) of the codes as the packed product of 16-bit activations sees it
    P, S, Z, (W, _) = codes(30, 256, 4, 128, 9)
    q = oi.unpack_codes(P.cpu().numpy().view(np.uint32), 256, 4)
    want = np.repeat(S.cpu().numpy(), 128, 1) * (q - np.repeat(Z.cpu().numpy(), 128, 1))
    assert np.allclose(W, want, rtol=1e-6)


@pytest.mark.parametrize("m", [1, 130, 384, 500, 640, 1300])
@pytest.mark.parametrize("n,T", [(1925, 3845), (2048, 4096)])
def test_whole_rounds_of_float32_results(n, T, m):
    # enough tiles of 256 tokens x 128 channels for one each on 256 CUs, from
    # one block of features to several
    X8, xs, *X = eight_bits(T, m, T + m, 1, 1)
    W8, ws, W, w = eight_bits(n, m, n + m, 128, 1, spread=1.0)
    check(ok.matmul_fp8(W8, ws, X8, xs, tokens_first=m % 4 == 0), (W, w), X, m % 4 == 0)
    f = ws.float() * (1 + torch.rand(ws.shape, device=DEV))
    check(ok.matmul_fp8(W8, f, X8, xs), (w * o8.expand(f.double().cpu().numpy(), n, m, 128), w), X)
    P, S, Z, W = codes(n, m, 3, 128, m)
    check(ok.dequant_matmul_fp8(P, S, Z, m, 3, 128, X8, xs), W, X)


@pytest.mark.parametrize("y", ["bf16", "f16"])
@pytest.mark.parametrize("m", [1, 130, 384, 500, 1300])
@pytest.mark.parametrize("n,T", [(3871, 3900), (4096, 4096)])
def test_whole_rounds_of_16_bit_results(n, T, m, y):
    # the same of tiles of 256 tokens x 256 channels
    X8, xs, *X = eight_bits(T, m, T + m, 1, 1)
    W8, ws, W, w = eight_bits(n, m, n + m, 128, 1, spread=1.0)
    first = m % 4 == 0
    check(ok.matmul_fp8(W8, ws, X8, xs, tokens_first=first, dtype=TYPES[y]), (W, w), X, first)
    f = ws.float() * (1 + torch.rand(ws.shape, device=DEV))
    check(ok.matmul_fp8(W8, f, X8, xs, tokens_first=not first, dtype=TYPES[y]),
          (w * o8.expand(f.double().cpu().numpy(), n, m, 128), w), X, not first)
    P, S, Z, W = codes(n, m, 4, 128, m)
    check(ok.dequant_matmul_fp8(P, S, Z, m, 4, 128, X8, xs, tokens_first=first, dtype=TYPES[y]), W, X, first)
