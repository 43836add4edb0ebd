"""The 8-bit entry points at the ends of their ranges on the GPU: the most
tokens, arrays behind 32-bit offsets, long row strides, workspaces given by the
caller and shared, and what stands around the results.  What the kernels
compute is held against the oracle elsewhere; here a large call is held,
exactly, against calls on parts of it, or against whole numbers whose sums
float32 holds exactly."""

import numpy as np
import pytest
import torch

import paper_2602_08376_amd as ok
from oracle import fp8 as o8

pytestmark = pytest.mark.gpu
DEV = "cuda"
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
MOST = 1 << 24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ok.library()
    yield
    torch.cuda.empty_cache()


def bits(t):
    return t.view(torch.uint8)


def alike(a, b):
    return torch.equal(bits(a), bits(b))


def whole(rows, m, seed, most=4):
    """An 8-bit array of whole numbers up to `most`, scales 1."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    v = torch.randint(-most, most + 1, (rows, -(-m // 16) * 16), device=DEV, generator=g).float().to(F8)[:, :m]
    s = torch.full((rows, -(-m // 512) * 4), 127, dtype=torch.uint8, device=DEV).view(E8)[:, :-(-m // 128)]
    return v, s


def random_codes(n, m, b, group, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    P = torch.randint(-2 ** 31, 2 ** 31, (n, ok.packed_words(m, b)), device=DEV, generator=g, dtype=torch.int64).int()
    G = -(-m // group)
    Z = torch.randint(0, 1 << b, (n, G), device=DEV, generator=g).float()
    return P, torch.ones(n, G, device=DEV), Z


def test_the_most_tokens_norm():
    m, part = 3, 4096
    x = torch.randn(part, m, device=DEV).half().repeat(MOST // part, 1)
    r = torch.randn(part, m, device=DEV).repeat(MOST // part, 1)
    first = r[:part].clone()
    want = ok.rmsnorm_fp8(x[:part], None, 1e-5, residual=first)
    v, s = ok.rmsnorm_fp8(x, None, 1e-5, residual=r)
    assert bool((bits(v).reshape(-1, part, m) == bits(want[0])).all())
    assert bool((bits(s).reshape(-1, part, 1) == bits(want[1])).all())
    assert bool((r.view(-1, part, m) == first).all())


@pytest.mark.parametrize("form", ["rows", "features", "blocks"])
def test_the_most_rows_quantize(form):
    m, part = 3, 4096
    X = torch.randn(part, m, device=DEV).half()
    X = X * torch.exp2(torch.arange(part, device=DEV) % 7 - 3).half()[:, None]
    block = 128 if form == "blocks" else 1
    want = ok.quantize_fp8(X, block_rows=block)
    Y = X.repeat(MOST // part, 1)
    if form == "features":
        v, s = ok.quantize_fp8(Y.t().contiguous(), features_first=True)
    else:
        v, s = ok.quantize_fp8(Y, block_rows=block)
    assert bool((bits(v).reshape(-1, part, m) == bits(want[0])).all())
    assert bool((bits(s).reshape(-1, part // block, 1) == bits(want[1])).all())


@pytest.mark.parametrize("x", [torch.float32, torch.float16])
@pytest.mark.parametrize("T", [127, 128, 129, 255, 257])
def test_features_first_around_whole_groups_of_tokens(T, x):
    X = (torch.randn(300, T, device=DEV) * 3).to(x)
    v, s = ok.quantize_fp8(X, features_first=True)
    want = ok.quantize_fp8(X.t().contiguous())
    assert alike(v, want[0]) and alike(s, want[1])


def test_more_tokens_than_a_grids_second_dimension():
    # rows of weights longer than the tiles address: the kernel for few tokens
    n, m, T = 3, 16, 65535 * 32 + 33
    X8, xs = whole(T, m, 1)
    W8, ws = whole(n, m, 2)
    far = torch.empty(2 * ((1 << 23) + 16) + 16, dtype=torch.uint8, device=DEV)
    W = torch.as_strided(far, (n, m), ((1 << 23) + 16, 1)).view(F8)
    W.copy_(W8)
    Y = ok.matmul_fp8(W, ws, X8, xs)
    assert torch.equal(Y, W8.float() @ X8.float().t())


def test_rows_of_activations_behind_32_bits():
    n, m, T = 2100, 144, 1100          # in tiles
    W8, ws = whole(n, m, 3)
    X, xs = whole(T, m, 4)
    want = (W8.double() @ X.double().t()).float()
    for ld in ((1 << 22) + 16, (1 << 23) + 16):     # 4.6 GB; and beyond the tiles' rows
        far = torch.empty((T - 1) * ld + m, dtype=torch.uint8, device=DEV)
        X8 = torch.as_strided(far, (T, m), (ld, 1)).view(F8)
        X8.copy_(X)
        for y in (torch.float32, torch.bfloat16):
            # (products up to 16 add up exactly in any order, on the 8-bit path too)
            assert torch.equal(ok.matmul_fp8(W8, ws, X8, xs, dtype=y), want.to(y)), (ld, y)
        P, S, Z = random_codes(n, m, 4, 144, 5)
        got = ok.dequant_matmul_fp8(P, S, Z, m, 4, 0, X8, xs)
        assert torch.equal(got, ok.dequant_matmul_fp8(P, S, Z, m, 4, 0, X, xs)), ld
        del far, X8


def test_results_behind_32_bits():
    n, T, m = 65537, 65600, 16
    W8, ws = whole(n, m, 6)
    X8, xs = whole(T, m, 7)
    for first in (False, True):
        Y = ok.matmul_fp8(W8, ws, X8, xs, dtype=torch.bfloat16, tokens_first=first)
        for a, b in ((slice(0, 70), slice(0, 70)), (slice(n - 70, n), slice(T - 70, T)), (slice(n - 70, n), slice(0, 70))):
            got = Y[b, a].t() if first else Y[a, b]
            assert torch.equal(got, (W8[a].float() @ X8[b].float().t()).bfloat16())
        del Y


@pytest.mark.parametrize("T", [1, 40])
def test_codes_behind_32_bits(T):
    n, m, b = 1 << 20, 8448, 4          # 4.4 GB of codes
    P, S, Z = random_codes(n, m, b, 128, 8)
    X8, xs = whole(T, m, 9, most=1)
    Y = ok.dequant_matmul_fp8(P, S, Z, m, b, 128, X8, xs)
    for r in (slice(0, 300), slice(n - 300, n)):
        assert torch.equal(Y[r], ok.dequant_matmul_fp8(P[r], S[r], Z[r], m, b, 128, X8, xs))


def test_inputs_behind_32_bits():
    T, m = 70000, 32768
    X = torch.randn(T, m, device=DEV, dtype=torch.float16)
    for call in (ok.quantize_fp8, lambda x: ok.rmsnorm_fp8(x, None, 1e-5), lambda x: ok.quantize_fp8(x, block_rows=128)):
        got, want = call(X), call(X[69888:])         # (69888 = 128 x 546)
        assert alike(got[0][69888:], want[0]) and alike(got[1][-want[1].shape[0]:], want[1])
        del got
    got, want = ok.quantize_fp8(X, features_first=True), ok.quantize_fp8(X[69888:], features_first=True)
    assert alike(got[0][:, 69888:], want[0]) and alike(got[1][:, 546:], want[1])


def test_workspaces():
    n, m, T = 2100, 400, 1003
    lib = ok.library()
    P, S, Z = random_codes(n, m, 4, 128, 10)
    X8, xs = whole(T, m, 11)
    want = ok.dequant_matmul_fp8(P, S, Z, m, 4, 128, X8, xs, dtype=torch.float16)
    need = int(lib.ojbkq_dequant_matmul_fp8_workspace_bytes(n, m, T))
    assert need > 0 and lib.ojbkq_dequant_matmul_fp8_workspace_bytes(n, m, 32) == 0
    buf = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    call = lambda w, t=T: ok.dequant_matmul_fp8(P, S, Z, m, 4, 128, X8[:t], xs[:t], dtype=torch.float16, workspace=w)  # noqa: E731
    assert torch.equal(call(buf[16:16 + need]), want)
    assert bool((buf[:16] == 0xA5).all()) and bool((buf[16 + need:] == 0xA5).all())
    buf.fill_(0xA5)                                    # a few tokens leave it alone
    assert torch.equal(call(buf, 32), call(None, 32)) and bool((buf == 0xA5).all())
    for w, code in ((buf[:need - 1], -2), (buf[8:8 + need], -1)):
        with pytest.raises(ok.OjbkqError) as e:
            call(w)
        assert e.value.status == code
    with pytest.raises(ValueError):
        call(buf.float())
    with pytest.raises(ValueError):
        call(buf.cpu())


def test_two_graphs_on_one_workspace():
    n, m, T = 2100, 400, 1003
    X8, xs = whole(T, m, 12)
    need = int(ok.library().ojbkq_dequant_matmul_fp8_workspace_bytes(n, m, T))
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    layers = [random_codes(n, m, b, 128, b) for b in (3, 4)]
    call = lambda i: ok.dequant_matmul_fp8(*layers[i], m, 3 + i, 128, X8, xs, dtype=torch.bfloat16, workspace=ws)  # noqa: E731
    want = [call(0), call(1)]
    graphs, got = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(call(i))
        graphs.append(g)
    for turn in range(3):
        for i in (0, 1, 1, 0):
            got[i].zero_()
            graphs[i].replay()
        torch.cuda.synchronize()
        ws.fill_(turn)                                 # eager work of the program's own in between
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), turn


@pytest.mark.parametrize("ytype,y", [(0, torch.float32), (1, torch.float16), (2, torch.bfloat16)])
@pytest.mark.parametrize("n,m,T", [(37, 200, 19), (2101, 200, 1003)])
def test_what_stands_around_a_result(n, m, T, ytype, y):
    lib, stream = ok.library(), torch.cuda.current_stream().cuda_stream
    X8, xs = whole(T, m, 13)
    W8, ws = whole(n, m, 14)
    want = (W8.float() @ X8.float().t()).to(y)
    for first in (0, 1):
        rows, cols = (T, n) if first else (n, T)
        buf = torch.full((rows + 2, cols + 5), -7.0, dtype=y, device=DEV)
        assert lib.ojbkq_matmul_fp8(W8.data_ptr(), W8.stride(0), ws.data_ptr(), 1, 1, ws.stride(0), n, m, X8.data_ptr(),
                                    X8.stride(0), xs.data_ptr(), xs.stride(0), T, buf[1:].data_ptr(), ytype, first,
                                    cols + 5, stream) == 0
        assert torch.equal(buf[1:-1, :cols], want.t() if first else want)
        buf[1:-1, :cols] = -7.0
        assert bool((buf == -7.0).all())


@pytest.mark.parametrize("m", [5, 200, 640])
def test_what_stands_around_an_8_bit_array(m):
    lib, stream, T = ok.library(), torch.cuda.current_stream().cuda_stream, 33
    m16, G = -(-m // 16) * 16, -(-m // 128)
    x = torch.randn(T, m, device=DEV)
    want = ok.quantize_fp8(x)
    xt = x.t().contiguous()
    for call in ("rows", "features", "norm", "blocks"):
        v = torch.full((T + 2, m16 + 32), 0x55, dtype=torch.uint8, device=DEV)
        s = torch.full((T + 2, -(-G // 4) * 4 + 4), 0x55, dtype=torch.uint8, device=DEV)
        to = (v[1:].data_ptr(), v.stride(0), s[1:].data_ptr(), s.stride(0), stream)
        if call == "norm":
            rc = lib.ojbkq_rmsnorm_fp8(x.data_ptr(), 0, T, m, m, None, None, 0, m, None, 0.5, *to)
            want8 = ok.rmsnorm_fp8(x, None, 0.5)
        else:
            f, b = int(call == "features"), 128 if call == "blocks" else 1
            rc = lib.ojbkq_quantize_fp8((xt if f else x).data_ptr(), 0, T, m, T if f else m, f, b, *to)
            want8 = ok.quantize_fp8(x, block_rows=128) if b == 128 else want
        assert rc == 0
        R = want8[1].shape[0]
        assert torch.equal(v[1:-1, :m], bits(want8[0])) and not v[1:-1, m:m16].any()
        assert torch.equal(s[1:1 + R, :G], bits(want8[1]))
        v[1:-1, :m16] = 0x55
        s[1:1 + R, :G] = 0x55
        assert bool((v == 0x55).all()) and bool((s == 0x55).all()), call


def test_a_token_whose_features_are_all_masked():
    # tokens of zeros, as a padded batch has them: no scale, no product, no NaN
    x = torch.randn(70, 300, device=DEV)
    x[5], x[69] = 0.0, 0.0
    X8, xs = ok.quantize_fp8(x)
    assert bool((bits(xs)[5] == 127).all()) and not bits(X8)[5].any()
    N8, ns = ok.rmsnorm_fp8(x, None, 1e-6)
    assert not bits(N8)[5].any() and bool((bits(ns)[5] == 127).all())
    W8, ws = whole(90, 300, 15)
    Y = ok.matmul_fp8(W8, ws, X8, xs)
    assert not Y[:, 5].any() and not Y[:, 69].any() and not bool(Y.isnan().any())
    want, e = o8.quantize(x.double().cpu().numpy())
    assert np.array_equal(X8.double().cpu().numpy(), want)


def test_arguments_that_the_binding_refuses():
    X8, xs = whole(40, 256, 16)
    W8, ws = whole(30, 256, 17)
    P, S, Z = random_codes(30, 256, 4, 128, 18)
    x, gain = torch.randn(40, 256, device=DEV), torch.ones(256, device=DEV)
    mm = ok.matmul_fp8
    dq = lambda *a, **k: ok.dequant_matmul_fp8(*a, X8, xs, **k)  # noqa: E731
    bad = [lambda: mm(W8, [1.0], X8, xs), lambda: mm(W8, ws[0], X8, xs), lambda: mm(W8, ws[:7], X8, xs),
           lambda: mm(W8, ws.double(), X8, xs), lambda: mm(W8, ws.cpu(), X8, xs), lambda: mm(W8, ws, X8, xs[:39]),
           lambda: mm(W8[:, :128], ws[:, :1], X8, xs), lambda: mm(W8, ws, X8[:, 1:], xs), lambda: mm(W8.t(), ws, X8, xs),
           lambda: mm(W8, ws, X8, xs, dtype=torch.float64), lambda: mm(W8, ws, X8, ws), lambda: mm(W8, ws, x, xs),
           lambda: dq(P, S, Z, 255, 4, 128), lambda: dq(P, S, Z, 256, 3, 128), lambda: dq(P, S[:, :1], Z, 256, 4, 128),
           lambda: dq(P, S, Z.double(), 256, 4, 128), lambda: dq(P.t(), S, Z, 256, 4, 128), lambda: dq(P[0], S, Z, 256, 4, 128),
           lambda: ok.rmsnorm_fp8(x, gain[:255], 1e-5), lambda: ok.rmsnorm_fp8(x, gain.half(), 1e-5),
           lambda: ok.rmsnorm_fp8(x, gain, 1e-5, residual=x[:39]), lambda: ok.rmsnorm_fp8(x, gain, 1e-5, residual_out=x),
           lambda: ok.rmsnorm_fp8(x, gain, 1e-5, residual=x.double()),
           lambda: ok.rmsnorm_fp8(x, gain, 1e-5, residual=x, residual_out=torch.empty(40, 300, device=DEV)[:, :256]),
           lambda: ok.quantize_fp8(x, block_rows=64), lambda: ok.quantize_fp8(x[:, ::2]),
           lambda: ok.quantize_fp8(x[:1].expand(40, 256))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            print("call", i)
            call()
    for call in (lambda: dq([1], S, Z, 256, 4, 128), lambda: ok.rmsnorm_fp8(x, 1.0, 1e-5), lambda: ok.rmsnorm_fp8(None, gain, 1e-5)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ok.quantize_fp8(x, block_rows=128, features_first=True), lambda: ok.rmsnorm_fp8(x, gain, -1.0),
                 lambda: ok.rmsnorm_fp8(x, gain, float("nan")), lambda: ok.quantize_fp8(x[:0]),
                 lambda: dq(P, torch.ones(30, 4, device=DEV), torch.ones(30, 4, device=DEV), 256, 4, 64)):
        with pytest.raises(ok.OjbkqError):
            call()


def test_a_scale_that_is_no_number():
    # an e8m0 code 255 makes its token's or its channels' results infinite or NaN, no others
    for n, T in ((40, 20), (2100, 1003), (4096, 4096)):
        X8, xs = whole(T, 256, 19, most=3)
        W8, ws = whole(n, 256, 20, most=3)
        X8, W8 = (X8.float().abs() + 1).to(F8), (W8.float().abs() + 1).to(F8)
        bits(xs)[3, 1] = 255
        bits(ws)[5, 0] = 255
        for y in (torch.float32, torch.bfloat16):
            Y = ok.matmul_fp8(W8, ws, X8, xs, dtype=y)
            bad = torch.zeros(n, T, dtype=torch.bool, device=DEV)
            bad[5], bad[:, 3] = True, True
            assert torch.equal(~Y.isfinite(), bad), (n, T, y)
