"""How exact the products' sums are.

Results in 16 bits of products in tiles add eight neighbouring products after
cutting each, towards zero, to a multiple of 2^(E - 13), E the largest sum of
the factors' exponents among the eight.  Operands whose exact result is 0 (a
half of the features again, negated, in another order within each block) leave
nothing but these cuts, which 16 bits hold to their own precision, so the rule is
held element by element.  What else rounds are the float32 sums: 2 G additions
of blocks, each off by up to 2^-24 of a sum as large as the half's result, and
16 of eights in each block, up to 2^-23 of the block's, G^-1/2 of it: together a
root mean square of ((2 G) / 3 + 2 G x 16 x 4 / 3 / G)^1/2 2^-24 = 8 x 2^-24 of the
half's result for G = 32; four times that is allowed.  (A cut one bit higher
would be off by as much as the cuts themselves, 1e-5 or more.)
"""

import pytest
import torch

import paper_2602_08376_amd as ok
import test_gpu_fp8_products as products

pytestmark = pytest.mark.gpu
DEV = "cuda"
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ok.library()


def operands(n, T, m, kind, scales, seed):
    """(W8, its scales, X8, its scales) of Gaussian numbers; 'channels': with
    log-normal channel scales, of which 1% are 50 times larger, as the package's
    synthetic layers have them."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    X, W = torch.randn(T, m, generator=g, device=DEV), 0.02 * torch.randn(n, m, generator=g, device=DEV)
    if kind == "channels":
        c = torch.exp(torch.randn(m, generator=g, device=DEV))
        c[torch.randperm(m, generator=g, device=DEV)[:m // 100]] *= 50.0
        X *= c
    W8, ws = ok.quantize_fp8(W, block_rows=128)
    if scales == "f32":
        ws = ws.float() * (1 + torch.rand(ws.shape, generator=g, device=DEV))
    return W8, ws, *ok.quantize_fp8(X)


def wide(v, s, rows):
    n, m = v.shape
    return v.double() * s.double().repeat_interleave(128, 1)[:, :m].repeat_interleave(rows, 0)[:n]


def cuts(w, x):
    """What the cuts add to each block's sum [blocks, n, T] of e4m3 values."""
    def exponent(v):
        return torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))

    out = torch.zeros(w.shape[1] // 128, w.shape[0], x.shape[0], dtype=torch.float64, device=DEV)
    for k in range(0, w.shape[1], 8):
        p = w[:, None, k:k + 8] * x[None, :, k:k + 8]
        step = torch.exp2((exponent(w[:, k:k + 8])[:, None] + exponent(x[:, k:k + 8])[None]).amax(2, True) - 13)
        out[k // 128] += (torch.trunc(p / step) * step - p).sum(2)
    return out


def twice(t, order=None):
    b = t.view(torch.uint8) if t.dtype != torch.float32 else t
    return torch.cat([b, b if order is None else b[:, order]], 1).contiguous().view(t.dtype)


def rms(t):
    return float(t.square().mean().sqrt())


@pytest.mark.parametrize("n,T", [(2100, 1003), (4096, 4096)])
@pytest.mark.parametrize("scales", ["e8m0", "f32"])
@pytest.mark.parametrize("kind", ["gaussian", "channels"])
def test_cuts_of_products_in_tiles(kind, scales, n, T):
    m, part = 2048, 64
    W8, ws, X8, xs = operands(n, T, m, kind, scales, n)
    g = torch.Generator(device=DEV).manual_seed(1)
    order = torch.cat([torch.randperm(128, generator=g, device=DEV) + k for k in range(0, m, 128)])
    W2, X2 = twice(W8, order), twice(X8, order)
    W2[:, m:] = (-W2[:, m:].float()).to(F8)
    ws2, xs2 = twice(ws), twice(xs)
    half = rms(wide(W8, ws, 128) @ wide(X8, xs, 1).t())
    for r, t in ((slice(0, part), slice(0, part)), (slice(n - part, n), slice(T - part, T))):
        c = cuts(W2[r].double(), X2[t].double())
        s = wide(torch.ones_like(W2, dtype=torch.float32), ws2, 128)[r, ::128].t()[:, :, None] * xs2[t].double().t()[:, None, :]
        want = (c * s).sum(0)
        for y in (torch.float16, torch.bfloat16):
            got = ok.matmul_fp8(W2, ws2, X2, xs2, dtype=y)[r, t].double()
            step = 2.0 ** -11 if y == torch.float16 else 2.0 ** -8
            off = (got - want).abs() - step * want.abs() - (2.0 ** -25 if y == torch.float16 else 0.0)
            print(rms(want) / half, rms(got - want) / half)
            assert rms(off.clamp(min=0.0)) <= 32 * 2.0 ** -24 * half
    # float32 results have no cuts: the float32 sums alone
    got = ok.matmul_fp8(W2, ws2, X2, xs2, dtype=torch.float32).double()
    assert rms(got) <= 32 * 2.0 ** -24 * half


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("kind,most", [("gaussian", 1.5e-5), ("channels", 8e-5)])
def test_error_of_16_bit_results(kind, most, codes):
    # the documented figures, beside the rounding to 16 bits: within half again
    n, T, m = 4096, 4096, 4096
    W8, ws, X8, xs = operands(n, T, m, kind, "f32", 5)
    if codes:
        P, S, Z, (W, _) = products.codes(n, m, 4, 128, 6)
        W = torch.from_numpy(W).to(DEV)
        call = lambda y: ok.dequant_matmul_fp8(P, S, Z, m, 4, 128, X8, xs, dtype=y)  # noqa: E731
    else:
        W = wide(W8, ws, 128)
        call = lambda y: ok.matmul_fp8(W8, ws, X8, xs, dtype=y)  # noqa: E731
    exact = W @ wide(X8, xs, 1).t()
    for y in (torch.float16, torch.bfloat16):
        rounded = rms(exact.to(y).double() - exact)
        err = rms(call(y).double() - exact)
        print(err / rms(exact), rounded / rms(exact), max(err ** 2 - rounded ** 2, 0.0) ** 0.5 / rms(exact))
        assert err <= (rounded ** 2 + (1.5 * most * rms(exact)) ** 2) ** 0.5


@pytest.mark.parametrize("y", ["f16", "bf16"])
@pytest.mark.parametrize("n,T", [(4100, 400), (1900, 900), (33000, 32)])
def test_codes_below_their_tiles_are_exact(n, T, y, monkeypatch):
    # from 1280 to 1792 blocks of 32 x 32, where 8-bit weights are in tiles and
    # codes are not; and few tokens
    assert T <= 32 or 1280 < -(-n // 32) * -(-T // 32) <= 1792
    monkeypatch.setattr(products, "in_tiles", lambda n, T: False)
    m = 520
    P, S, Z, W = products.codes(n, m, 4, 128, 7)
    X8, xs, *X = products.eight_bits(T, m, 8)
    products.check(ok.dequant_matmul_fp8(P, S, Z, m, 4, 128, X8, xs, dtype=products.TYPES[y]), W, X)
