"""Arrays in 8 bits on the GPU (``quantize_fp8``, ``rmsnorm_fp8``) against the
float64 oracle, bit for bit: both are defined by one rounding of a float64
value, and the values' float64 error (about m 2^-53) moves none of them across
a border in these inputs."""

import numpy as np
import pytest
import torch

import paper_2602_08376_amd as ok
from oracle import fp8 as o8

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ok.library()


def tensor(rows, m, dtype, seed, pad=0, shift=0):
    """Rows of very different channels in a wider buffer that is NaN elsewhere
    and ends at the last element."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, m)) * np.exp(2 * rng.standard_normal((1, m)))
    buf = torch.full((shift + (rows - 1) * (m + pad) + m,), float("nan"), dtype=dtype, device=DEV)
    t = torch.as_strided(buf, (rows, m), (m + pad, 1), shift)
    t.copy_(torch.from_numpy(x).to(dtype))
    return t


def host(t):
    return t.double().cpu().numpy()


def exponents(s):
    return s.view(torch.uint8).cpu().numpy().astype(np.int64) - 127


def same(v, s, want, e):
    assert v.dtype == torch.float8_e4m3fn and s.dtype == torch.float8_e8m0fnu
    assert np.array_equal(exponents(s), e)
    assert np.array_equal(host(v), want, equal_nan=True)


def zero_to_16(v):
    """The bytes behind a row's last value, up to a multiple of 16."""
    m = v.shape[1]
    wide = torch.as_strided(v.view(torch.uint8), (v.shape[0], -(-m // 16) * 16), (v.stride(0), 1))
    assert not wide[:, m:].any()


@pytest.mark.parametrize("x", list(TYPES))
@pytest.mark.parametrize("rows,m,pad,shift", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 129, 0, 1), (5, 127, 3, 0),
                                              (2, 2500, 1, 3), (130, 640, 8, 0), (9, 14336, 0, 0),
                                              (2049, 513, 0, 0), (700, 4096, 0, 0)])
def test_quantize_rows(x, rows, m, pad, shift):
    X = tensor(rows, m, TYPES[x], rows + m, pad, shift)
    v, s = ok.quantize_fp8(X)
    same(v, s, *o8.quantize(host(X)))
    zero_to_16(v)


@pytest.mark.parametrize("x", list(TYPES))
@pytest.mark.parametrize("T,m,pad,shift", [(1, 1, 0, 0), (1, 300, 0, 1), (7, 128, 5, 0), (64, 127, 0, 0), (65, 260, 0, 1),
                                           (130, 1000, 3, 1)])
def test_quantize_features_first(x, T, m, pad, shift):
    X = tensor(m, T, TYPES[x], T + m, pad, shift)
    v, s = ok.quantize_fp8(X, features_first=True)
    same(v, s, *o8.quantize(host(X).T))
    zero_to_16(v)


@pytest.mark.parametrize("x", list(TYPES))
@pytest.mark.parametrize("n,m,pad", [(1, 1, 0), (128, 128, 0), (129, 257, 1), (300, 1000, 0), (127, 100, 4)])
def test_quantize_blocks(x, n, m, pad):
    X = tensor(n, m, TYPES[x], n + m, pad)
    v, s = ok.quantize_fp8(X, block_rows=128)
    same(v, s, *o8.quantize(host(X), 128))
    zero_to_16(v)


def test_ties_borders_and_what_is_not_a_number():
    # a row for each: every tie and every number of the format with 448 beside
    # them (scale 1), largest magnitudes either side of the scale's border, the
    # smallest and largest floats, blocks of zeros, blocks with NaN and infinities
    p = o8._POSITIVE
    rows = [np.concatenate([p, [448.0]]), np.concatenate([(p[1:] + p[:-1]) / 2, [448.0, -448.0]]),
            -np.concatenate([(p[1:] + p[:-1]) / 2, [448.0, 0.0]]),
            np.r_[448.0, np.zeros(127)], np.r_[np.nextafter(np.float32(448), np.float32(500)), np.zeros(127)],
            np.r_[2.0 ** -149, np.zeros(127)], np.r_[2.0 ** -126, -2.0 ** -140, np.zeros(126)],
            np.r_[3.4028234663852886e38, 1.0, np.zeros(126)], np.zeros(128), -np.zeros(128),
            np.r_[np.nan, 3.0, np.inf, -np.inf, 1e-3, np.zeros(123)], np.full(128, np.inf), np.full(128, np.nan)]
    x = np.array(rows, dtype=np.float32)
    X = torch.from_numpy(x).to(DEV)
    want, e = o8.quantize(x.astype(np.float64))
    same(*ok.quantize_fp8(X), want, e)
    same(*ok.quantize_fp8(X.t().contiguous(), features_first=True), want, e)
    for r in range(len(rows)):      # a block of 128 rows, all but one of them zeros
        B = torch.zeros(128, 128, device=DEV)
        B[77] = X[r]
        same(*ok.quantize_fp8(B, block_rows=128), *o8.quantize(host(B), 128))


SMALL = [(1, 1, 0, 0), (1, 4096, 0, 0), (3, 127, 0, 1), (2, 129, 5, 0), (5, 2500, 0, 0), (4, 8192, 0, 0),
         (2, 8193, 0, 1), (3, 14336, 0, 0), (2, 32768, 0, 0), (2, 32777, 3, 0)]
LARGE = [(600, 2049, 0, 0), (520, 5000, 0, 0), (1030, 4097, 1, 0)]
NORMS = [(a, b, *c) for a in TYPES for b in [None, *TYPES] for c in SMALL] + \
        [(*t, *c) for t in (("f32", "f32"), ("bf16", "f16"), ("f16", None)) for c in LARGE]


@pytest.mark.parametrize("x,r,T,m,pad,shift", NORMS)
def test_norm(x, r, T, m, pad, shift):
    X = tensor(T, m, TYPES[x], T + m, pad, shift)
    R = None if r is None else tensor(T, m, TYPES[r], T + m + 1, shift, pad)
    gain = torch.from_numpy(np.random.default_rng(m).standard_normal(m).astype(np.float32)).to(DEV)
    before = None if R is None else R.clone()
    y, h = o8.rmsnorm(X.float().cpu().numpy(), None if R is None else R.float().cpu().numpy(),
                      gain.cpu().numpy(), 1e-5)
    want = o8.quantize(y)
    if R is not None:
        out = torch.empty_strided(R.shape, R.stride(), dtype=R.dtype, device=DEV)
        same(*ok.rmsnorm_fp8(X, gain, 1e-5, residual=R, residual_out=out), *want)
        assert torch.equal(R, before)
        assert torch.equal(out.cpu(), torch.from_numpy(h).to(R.dtype))
        v, s = ok.rmsnorm_fp8(X, gain, 1e-5, residual=R)             # in place
        assert torch.equal(R, out)
    else:
        v, s = ok.rmsnorm_fp8(X, gain, 1e-5)
    same(v, s, *want)
    zero_to_16(v)


@pytest.mark.parametrize("m", [256, 5000, 40000])
def test_norm_of_extreme_rows(m):
    rng = np.random.default_rng(m)
    x = rng.standard_normal((8, m)).astype(np.float32)
    x[0] = 0.0                       # nothing: eps alone
    x[1] *= np.float32(1e30)         # squares beyond float32
    x[2] *= np.float32(1e-30)        # and below it
    x[3, m // 2] = np.inf
    x[4, 0] = np.nan
    x[5, :] = 0.0
    x[5, m - 1] = -2.5               # one feature holds everything
    x[6, 7] = 1e6
    X = torch.from_numpy(x).to(DEV)
    for eps in (1e-5, 0.0):
        y, _ = o8.rmsnorm(x, None, None, eps)
        y[3:5] = np.nan
        if eps == 0.0:
            y[0] = np.nan
        same(*ok.rmsnorm_fp8(X, None, eps), *o8.quantize(y))
    # x + residual beyond float32 is infinite
    big = torch.full((2, m), 3e38, device=DEV)
    big[1] = 1.0
    v, _ = ok.rmsnorm_fp8(big, None, 1e-5, residual=big.clone())
    assert bool(v[0].float().isnan().all()) and not bool(v[1].float().isnan().any())


def test_norm_gain_beyond_float32():
    x = torch.ones(1, 256, device=DEV)
    gain = torch.ones(256, device=DEV)
    gain[3], gain[200] = float("inf"), float("nan")
    x[0, 7] = 100.0
    gain[7] = 3e38
    y, _ = o8.rmsnorm(x.cpu().numpy(), None, gain.cpu().numpy(), 0.0)
    same(*ok.rmsnorm_fp8(x, gain, 0.0), *o8.quantize(y))


def test_streams_and_graphs():
    X = tensor(33, 700, torch.float16, 1)
    R = tensor(33, 700, torch.float32, 2)
    want = ok.rmsnorm_fp8(X, None, 1e-6, residual=R.clone())
    wq = ok.quantize_fp8(X)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ok.rmsnorm_fp8(X, None, 1e-6, residual=R.clone())
    side.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
    out = torch.empty_like(R)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a = ok.rmsnorm_fp8(X, None, 1e-6, residual=R, residual_out=out)
        b = ok.quantize_fp8(X)
    for i in range(4):
        if i == 2:
            X.mul_(3.0)              # new inputs in the same place
            want, wq = ok.rmsnorm_fp8(X, None, 1e-6, residual=R.clone()), ok.quantize_fp8(X)
        g.replay()
        torch.cuda.synchronize()
        torch.ones(100, device=DEV).sum().item()
        for got, w in ((a, want), (b, wq)):
            assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(got, w)), i
