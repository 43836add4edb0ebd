"""Products with 8-bit activations on the GPU (``matmul_fp8``,
``dequant_matmul_fp8``) against the float64 oracle.

Operands are given in 8 bits, so what may differ is the sums.  With float32
results every product enters exactly and sums are float32: m products and two
operations on each of the ceil(m / 128) blocks round at most (m + 2 G) times,
2^-24 of the magnitudes each.  Results in 16 bits round once more, by half a
step: 2^-11 (float16, or 2^-25 below its normal range), 2^-8 (bfloat16)."""

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


def bound(W, X, y, ref):
    """What a result of type y may differ by from ref."""
    m = W.shape[1]
    a = o8.absolute(W, X)
    b = (m + 2 * -(-m // 128)) * 2.0 ** -24 * a
    if y == "f16":
        b = b + 2.0 ** -11 * (np.abs(ref) + b) + 2.0 ** -25
    if y == "bf16":
        b = b + 2.0 ** -8 * (np.abs(ref) + b)
    return b


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


def check(Y, ref, b):
    got = Y.double().cpu().numpy()
    if Y.dtype == torch.float16:
        # from 65520 on, half a step above the largest number, a result rounds
        # to infinity
        over = np.isinf(got)
        assert np.all((np.sign(got) * ref + b)[over] >= 65520.0)
        got, ref, b = got[~over], ref[~over], b[~over]
    err = np.abs(got - ref)
    worst = float(np.max(err / (b + 1e-300)))
    print(f"max err / bound {worst:.3f}")
    assert np.all(err <= b), worst


SIZES = [(1, 1, 1), (5, 3, 2), (16, 128, 16), (17, 129, 1), (16, 127, 15), (33, 1000, 17), (40, 300, 7), (130, 640, 33),
         (257, 1025, 1), (64, 4096, 3), (300, 2500, 65), (8193, 256, 20), (4100, 200, 130), (16400, 136, 9),
         (2100, 144, 1003), (600, 784, 600)]


@pytest.mark.parametrize("y", list(TYPES))
@pytest.mark.parametrize("n,m,T", SIZES)
@pytest.mark.parametrize("rows,scales,tokens_first", [(128, "e8m0", False), (128, "f32", True), (1, "e8m0", True),
                                                      (1, "f32", False)])
def test_matmul(n, m, T, rows, scales, tokens_first, y):
    pad = (n + T) % 3
    W8, ws, W, w = eight_bits(n, m, n + m, rows, pad, spread=1.0)
    X8, xs, X, _ = eight_bits(T, m, T + m, 1, pad)
    if scales == "f32":
        ws = ws.float() * (1 + torch.rand(ws.shape, device=DEV))
        W = w * o8.expand(ws.double().cpu().numpy(), n, m, rows)
    Y = ok.matmul_fp8(W8, ws, X8, xs, tokens_first=tokens_first, dtype=TYPES[y])
    assert Y.dtype == TYPES[y] and Y.shape == ((T, n) if tokens_first else (n, T))
    ref = o8.matmul(W, X)
    check(Y.t() if tokens_first else Y, ref, bound(W, X, y, ref))


def codes(n, m, bits, group, seed):
    rng = np.random.default_rng(seed)
    g = m if group <= 0 or group >= m else group
    G = -(-m // g)
    q = rng.integers(0, 1 << bits, size=(n, m), dtype=np.uint8)
    S = (0.01 * np.exp(rng.standard_normal((n, G)))).astype(np.float32)
    Z = rng.integers(0, 1 << bits, size=(n, G)).astype(np.float32)
    W = np.repeat(S.astype(np.float64), g, 1)[:, :m] * (q - np.repeat(Z, g, 1)[:, :m])
    P = torch.from_numpy(q).to(DEV)
    return ok.pack_codes(P, bits), torch.from_numpy(S).to(DEV), torch.from_numpy(Z).to(DEV), W


@pytest.mark.parametrize("y,tokens_first", [("f32", False), ("f32", True), ("f16", False), ("bf16", True)])
@pytest.mark.parametrize("n,m,T,group", [(1, 1, 1, 0), (5, 3, 2, 0), (16, 128, 16, 128), (17, 129, 1, 128), (16, 127, 15, 0),
                                         (33, 1000, 17, 128), (40, 300, 7, 256), (130, 640, 33, 0), (257, 1025, 1, 384),
                                         (300, 2500, 65, 128), (8193, 256, 20, 128), (16400, 136, 9, 0),
                                         (2100, 144, 1003, 128), (600, 784, 600, 256)])
@pytest.mark.parametrize("bits", [1, 2, 3, 4])
def test_dequant_matmul(n, m, T, group, bits, y, tokens_first):
    P, S, Z, W = codes(n, m, bits, group, n + m + bits)
    X8, xs, X, _ = eight_bits(T, m, T + m, 1, (n + T) % 3)
    Y = ok.dequant_matmul_fp8(P, S, Z, m, bits, group, X8, xs, tokens_first=tokens_first, dtype=TYPES[y])
    assert Y.dtype == TYPES[y] and Y.shape == ((T, n) if tokens_first else (n, T))
    ref = o8.matmul(W, X)
    check(Y.t() if tokens_first else Y, ref, bound(W, X, y, ref))


@pytest.mark.parametrize("T", [1, 5, 40, 700])
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
    W8, ws, W, _ = eight_bits(200, 520, 1, 1, 2)
    X8, xs, X, _ = eight_bits(90, 520, 2, 1, 1)
    for r, k in ((slice(7, 71), 520), (slice(1, 2), 384), (slice(0, 90), 130), (slice(89, 90), 5)):
        G = -(-k // 128)
        Y = ok.matmul_fp8(W8[3:150, :k], ws[3:150, :G], X8[r, :k], xs[r, :G])
        ref = o8.matmul(W[3:150, :k], X[r, :k])
        check(Y, ref, bound(W[3:150, :k], X[r, :k], "f32", ref))


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
        return o8.dequantize(v.double().cpu().numpy(), s.view(torch.uint8).cpu().numpy().astype(np.int64) - 127, rows)

    Xa, Wa = wide(X8, xs), wide(W8, ws, 128)
    ref = o8.matmul(Wa, Xa)
    check(Y.t(), ref, bound(Wa, Xa, "bf16", ref))
    Xb = wide(X8b, xsb)
    y, _ = o8.rmsnorm(stream.cpu().numpy(), None, None, 1e-5)
    v, e = o8.quantize(y)
    assert np.array_equal(o8.dequantize(v, e), Xb)           # the stream holds h itself: float32
    ref = o8.matmul(W, Xb)
    check(out, ref, bound(W, Xb, "f32", ref))


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


def test_oracles_weights_are_the_layers():
    # S (Q - Z) of the codes as the packed product of 16-bit activations sees it
    P, S, Z, W = codes(30, 256, 4, 128, 9)
    q = oi.unpack_codes(P.cpu().numpy().view(np.uint32), 256, 4)
    want = np.repeat(S.cpu().numpy(), 128, 1) * (q - np.repeat(Z.cpu().numpy(), 128, 1))
    assert np.allclose(W, want, rtol=1e-6)
