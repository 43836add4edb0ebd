"""Scales at the ends of their range in the product of packed codes with 8-bit
activations: a finite result stays finite and within the bounds of the other
products, however large or small the two scales behind it are by themselves."""

import numpy as np
import pytest
import torch

import paper_2602_08376_amd as ok
from oracle import fp8 as o8
from test_gpu_fp8_products import TYPES, check, codes, eight_bits

pytestmark = pytest.mark.gpu
DEV = "cuda"
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ok.library()


def times(W, S):
    """What codes stand for with other scales: (S (Q - Z), Q - Z)."""
    w = W[1]
    g = 128 if S.shape[1] > 1 else w.shape[1]
    return S.double().cpu().numpy().repeat(g, 1)[:, :w.shape[1]] * w, w


# (one token, a few, a second row of lanes, tiles; layers whose workgroups take 16, 32 and 64 channels)
SIZES = [(300, 1), (300, 24), (5200, 24), (10300, 5), (10300, 24), (2100, 1003)]


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("n,T", SIZES)
@pytest.mark.parametrize("bits,group", [(4, 128), (3, 0), (1, 128)])
def test_codes_at_the_ends_of_the_scales(bits, group, n, T, y):
    # activations at the smallest scales and near the largest, weights that bring
    # them back towards 1; 15 x 2 times a weight's scale is a float32
    m = 384
    P, S, Z, W = codes(n, m, bits, group, n + bits)
    X8, xs, X, x = eight_bits(T, m, T + m)
    S = S / torch.exp2(torch.floor(torch.log2(S)))                     # 1 to 2
    for code in (0, 1, 3, 127, 240, 246):
        xs.view(torch.uint8).fill_(code)
        s = S * 2.0 ** min(127 - code, 119)
        Y = ok.dequant_matmul_fp8(P, s, Z, m, bits, group, X8, xs, dtype=TYPES[y])
        assert bool(Y.isfinite().all()), code
        check(Y, times(W, s), (x * 2.0 ** (code - 127), x))


@pytest.mark.parametrize("n,T", SIZES)
def test_both_ends_in_one_row(n, T):
    # the first group's weights large and its activations small, the others the other way round
    m, bits = 384, 4
    P, S, Z, W = codes(n, m, bits, 128, n)
    X8, xs, X, x = eight_bits(T, m, T)
    S = S / torch.exp2(torch.floor(torch.log2(S)))
    s = S * torch.tensor([2.0 ** 110, 2.0 ** -100, 2.0 ** -119], device=DEV)
    c = torch.tensor([17, 227, 246], dtype=torch.uint8, device=DEV)
    xs.view(torch.uint8).copy_(c.expand(T, 3))
    Y = ok.dequant_matmul_fp8(P, s, Z, m, bits, 128, X8, xs)
    e = o8.expand(np.array([[17, 227, 246]]) - 127, T, m, T)
    assert bool(Y.isfinite().all())
    check(Y, times(W, s), (np.ldexp(x, e), x))


@pytest.mark.parametrize("T", [1, 24, 1003])
def test_a_large_feature_and_a_small_scale(T):
    # 15 x 448 times 2^116 is no float32, times 2^-20 it is one
    n, m = 2100, 256
    P = ok.pack_codes(torch.full((n, m), 15, dtype=torch.uint8, device=DEV), 4)
    S, Z = torch.full((n, 2), 2.0 ** -20, device=DEV), torch.full((n, 2), 15.0, device=DEV)
    Z[:, 0] = 0.0
    X8 = torch.zeros(T, m, device=DEV)
    X8[:, 3] = 448.0
    xs = torch.full((T, 4), 127 + 116, dtype=torch.uint8, device=DEV)
    Y = ok.dequant_matmul_fp8(P, S, Z, m, 4, 128, X8.to(F8), xs.view(E8)[:, :2])
    assert bool((Y == 15.0 * 448.0 * 2.0 ** 96).all())


@pytest.mark.parametrize("n,T", SIZES)
def test_a_code_of_255_among_codes(n, T):
    m, group = 384, 128
    P, S, Z, W = codes(n, m, 4, group, 3)
    X8, xs, X, x = eight_bits(T, m, 4)
    want = ok.dequant_matmul_fp8(P, S, Z, m, 4, group, X8, xs)
    t = T // 2
    b = xs.view(torch.uint8)
    b[t, 1] = 255
    for zero in (False, True):
        if zero:
            X8[t] = 0.0                                                # infinite times 0
        got = ok.dequant_matmul_fp8(P, S, Z, m, 4, group, X8, xs)
        assert not bool(got[:, t].isfinite().any())
        keep = torch.arange(T, device=DEV) != t
        assert torch.equal(got[:, keep], want[:, keep])


def large_weights(n, m, seed):
    """e4m3 numbers of at least 16 in magnitude."""
    rng = np.random.default_rng(seed)
    w = o8.round_e4m3(np.exp2(rng.uniform(4, 8.8, (n, m))) * rng.choice([-1.0, 1.0], (n, m)))
    return torch.from_numpy(w).float().to(F8).to(DEV), w


def e8m0(codes, m):
    """Scales of one row for each of `codes`' rows, padded to four."""
    s = torch.zeros(codes.shape[0], -(-codes.shape[1] // 4) * 4, dtype=torch.uint8, device=DEV)
    s[:, :codes.shape[1]] = codes
    return s.view(E8)[:, :codes.shape[1]]


PRODUCTS = [(40, 1), (300, 24), (6000, 24), (2100, 1003), (4096, 4096)]


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("n,T", PRODUCTS)
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -130, 1.7 * 2.0 ** -129, 2.0 ** -127, "e8m0"])
def test_weight_scales_below_the_normal_range(scale, n, T, y):
    # with activations near the largest float32: a block of weights 0, or of
    # weights from 2^-126 on by a scale below it
    m = 256
    W8, w = large_weights(n, m, n)
    X8, xs, X, x = eight_bits(T, m, T)
    xs.view(torch.uint8)[:, 0] = 246
    xs.view(torch.uint8)[:, 1] = 127
    if scale == "e8m0":
        ws = e8m0(torch.tensor([[0, 127]], dtype=torch.uint8, device=DEV).expand(n, 2), m)
    else:
        ws = torch.tensor([[scale, 1.0]], device=DEV).expand(n, 2).contiguous()
    Y = ok.matmul_fp8(W8, ws, X8, xs, dtype=TYPES[y])
    assert bool(Y.isfinite().all())
    if scale == 0.0:
        none = X8.clone().view(torch.uint8)
        none[:, :128] = 0
        assert torch.equal(Y, ok.matmul_fp8(W8, ws, none.view(F8), xs, dtype=TYPES[y]))
        return
    W = w * np.repeat(ws.double().cpu().numpy(), 128, 1)
    check(Y, (W, w), (np.ldexp(x, np.repeat([[119, 0]], 128, 1)), x))


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("n,T", PRODUCTS)
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -127])
def test_code_scales_below_the_normal_range(scale, n, T, y):
    m = 256
    P, S, Z, (_, w) = codes(n, m, 4, 128, n)
    X8, xs, X, x = eight_bits(T, m, T)
    xs.view(torch.uint8)[:, 0] = 246
    xs.view(torch.uint8)[:, 1] = 127
    S[:, 0] = scale
    call = lambda v: ok.dequant_matmul_fp8(P, S, Z, m, 4, 128, v, xs, dtype=TYPES[y])  # noqa: E731
    Y = call(X8)
    assert bool(Y.isfinite().all())
    if scale == 0.0:
        none = torch.zeros(T, m, device=DEV)
        none[:, 128:] = X8[:, 128:].float()
        assert torch.equal(Y, call(none.to(F8)))
        return
    check(Y, times((None, w), S), (np.ldexp(x, np.repeat([[119, 0]], 128, 1)), x))
