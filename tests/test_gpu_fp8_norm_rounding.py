"""The norm's y where it lies exactly on a border between two 8-bit numbers: one
division of h gain by the root, so that it goes to the even one."""

import numpy as np
import pytest
import torch

import paper_2602_08376_amd as ok
from oracle import fp8 as o8
from test_gpu_fp8_pack import TYPES, exponents, host, same

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ok.library()


def ties(m):
    """Gains between two numbers of the format each (and the largest in every
    block, whose scale they take)."""
    p = o8._POSITIVE[64:127]                          # 1.0 to 448
    mid = (p[1:] + p[:-1]) / 2
    g = mid[np.arange(m) % len(mid)]
    g[::128] = 448.0
    return g.astype(np.float32), g


@pytest.mark.parametrize("x", list(TYPES))
@pytest.mark.parametrize("T,m", [(130, 256), (600, 130), (130, 5000), (600, 5000), (600, 7000), (520, 9000), (520, 13000),
                                 (40, 40000)])
def test_rows_of_one_value(x, T, m):
    # h / sqrt(mean(h^2)) = 1 (the squares' sum and its root are exact), so y is
    # the gain; whole numbers h, most of which have no exact reciprocal
    h = torch.arange(1, T + 1, device=DEV).clamp(max=256).to(TYPES[x])     # (bfloat16 holds these)
    gain, g = ties(m)
    X = h[:, None].expand(T, m).contiguous()
    v, s = ok.rmsnorm_fp8(X, torch.from_numpy(gain).to(DEV), 0.0)
    want, e = o8.quantize(g[None, :])
    same(v, s, np.repeat(want, T, 0), np.repeat(e, T, 0))


@pytest.mark.parametrize("wide,m", [(16, 256), (16, 5008), (64, 4096), (9, 2304), (9, 18000)])
def test_quotients_on_a_border(wide, m):
    # c in every 16th, 64th or 9th feature and 0 in the others: the root is c / 4,
    # c / 8 or c / 3, and y = 4, 8 or 3 times the gain is on a border.  (c a
    # multiple of 3 for the last: no other third is a float64, and the root is
    # one, so y would not be on the border but 2^-53 beside it.)
    r = {16: 4, 64: 8, 9: 3}[wide]
    c = np.arange(1, 65, dtype=np.float32) * (3 if r == 3 else 1)
    h = np.zeros((64, m), dtype=np.float32)
    h[:, ::wide] = c[:, None]
    _, g = ties(m)
    if r == 3:                                         # 21 / 16 and 27 / 16 are borders
        g = np.where(np.arange(m) % 2 == 0, 7 / 16, 9 / 16) * np.exp2(np.arange(m) % 5)
    y = np.where(h > 0, r * g, 0.0)
    v, s = ok.rmsnorm_fp8(torch.from_numpy(h).to(DEV), torch.from_numpy(g.astype(np.float32)).to(DEV), 0.0)
    want, e = o8.quantize(y)
    same(v, s, want, e)


def test_largest_magnitudes_on_the_scales_border():
    # the largest y of a block is 448 2^k itself, for h with no exact reciprocal
    h = torch.tensor([3.0, 49.0, 98.0, 103.0, 1000.0, 7e-3], device=DEV)
    gain = torch.full((256,), 1.0, device=DEV)
    gain[128:] = 448.0
    v, s = ok.rmsnorm_fp8(h[:, None].expand(6, 256).contiguous(), gain, 0.0)
    assert (exponents(s) == [[-8, 0]]).all()
    assert (host(v) == [256.0] * 128 + [448.0] * 128).all()


@pytest.mark.parametrize("m", [4096, 8192])
def test_a_token_by_itself_and_among_many(m):
    # One square of 2^56 beside several of 8, of which float64 loses each that is
    # added to it by itself and keeps those that are added up before: the root is
    # 2^28 / sqrt(m) or two steps above, and a y of the second half on the border
    # of e4m3 or below it.  The order of the sum does not go by the number of
    # tokens, which chooses the threads to a token.
    h = np.zeros(m, dtype=np.float32)
    h[0] = 2.0 ** 28
    for run in [0, 1, 2, 4, 8, 16, 32] + list(range(64, m // 16, 64)):
        h[m // 2 + 8 * run:m // 2 + 8 * run + 2] = 2.0
    gain = torch.ones(m, device=DEV)
    gain[m // 2], gain[m // 2 + 1] = 19 / 16, 7 / 4
    x = torch.from_numpy(h).to(DEV)
    one = ok.rmsnorm_fp8(x[None], gain, 0.0)
    for T in (2, 512, 513, 2000):
        v, s = ok.rmsnorm_fp8(x.expand(T, m).contiguous(), gain, 0.0)
        same(v, s, np.repeat(host(one[0]), T, 0), np.repeat(exponents(one[1]), T, 0))
