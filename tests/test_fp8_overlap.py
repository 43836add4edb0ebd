"""What the norm's binding refuses of a residual stream that shares memory with
the call's other arrays, and what it takes."""

import itertools

import pytest
import torch

import paper_2602_08376_amd as ok


def touched(t):
    """The bytes of a matrix."""
    out = set()
    for i in range(t.shape[0]):
        p = t.data_ptr() + i * t.stride(0) * t.element_size()
        out.update(range(p, p + t.shape[1] * t.element_size()))
    return out


def test_overlap_is_that_of_the_bytes():
    buf = torch.zeros(400, dtype=torch.uint8)
    views = []
    for dtype, n, m, ld, shift in itertools.product((torch.float32, torch.float16), (1, 2, 5), (1, 3), (3, 4, 6),
                                                    (0, 1, 2, 3, 4, 7, 20)):
        v = buf.view(dtype)
        if shift + (n - 1) * ld + m <= v.numel():
            views.append(torch.as_strided(v, (n, m), (ld, 1), shift))
    checked = 0
    for a, b in itertools.product(views, views):
        if a.shape != b.shape:
            continue
        n, m = a.shape
        sizes = a.element_size(), b.element_size()
        pitch = lambda t: (t.stride(0) if n > 1 else m) * t.element_size()  # noqa: E731
        same = a.data_ptr() == b.data_ptr() and pitch(a) == pitch(b) and sizes[0] == sizes[1]
        want = not same and bool(touched(a) & touched(b))
        got = ok._overlap(a.data_ptr(), pitch(a), b.data_ptr(), pitch(b), n, m, sizes)
        assert got == want, (a.shape, a.stride(), a.storage_offset(), a.dtype, b.stride(), b.storage_offset(), b.dtype)
        checked += 1
    assert checked > 3000


gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("T,m", [(1, 300), (9, 2500), (600, 4096), (3, 20000)])
def test_streams_that_share_memory(T, m):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    buf = torch.randn(T + 1, 2 * m + 8, device="cuda", dtype=torch.float16)
    x, r = buf[:T, :m], buf[:T, m:2 * m]            # side by side: no overlap
    gain = torch.rand(m, device="cuda") + 0.5
    want = ok.rmsnorm_fp8(x.clone(), gain, 1e-5, residual=r.clone(), residual_out=(h := torch.empty_like(r.clone())))
    same = lambda got: all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))  # noqa: E731

    # the sum in place, and in x's place
    before = buf.clone()
    assert same(ok.rmsnorm_fp8(x, gain, 1e-5, residual=r)) and torch.equal(r, h) and torch.equal(x, before[:T, :m])
    buf.copy_(before)
    assert same(ok.rmsnorm_fp8(x, gain, 1e-5, residual=r, residual_out=x)) and torch.equal(x, h)
    assert torch.equal(r, before[:T, m:2 * m])
    # a stream added to itself
    buf.copy_(before)
    ok.rmsnorm_fp8(x, gain, 1e-5, residual=x)
    assert torch.equal(x, (2 * before[:T, :m].float()).half())

    buf.copy_(before)
    for out in (buf[:T, 8:m + 8], buf[:T, m - 8:2 * m - 8], buf[1:T + 1, :m] if T > 1 else buf[:T, 1:m + 1],
                buf[:T, m + 2:2 * m + 2]):
        with pytest.raises(ValueError, match="overlap"):
            ok.rmsnorm_fp8(x, gain, 1e-5, residual=r, residual_out=out)
    # the same place, wider elements
    wide = torch.zeros(T, m, device="cuda")
    half = wide.view(torch.float16)[:, :m]
    with pytest.raises(ValueError, match="overlap"):
        ok.rmsnorm_fp8(half, gain, 1e-5, residual=wide)
    assert torch.equal(buf, before)
