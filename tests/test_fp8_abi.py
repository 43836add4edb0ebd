"""CPU-only checks of the C ABI of the 8-bit side (include/ojbkq_fp8.h): every
declared function is exported and bound, and every documented argument error is
found before anything is enqueued (the pointers here are no memory)."""

import ctypes
import os
import re

import pytest
import torch

import paper_2602_08376_amd as ok
from conftest import ROOT

A = 4096          # an aligned address


def test_every_declared_function_is_bound():
    text = open(os.path.join(ROOT, "include", "ojbkq_fp8.h")).read()
    text = re.sub(r"/\*.*?\*/", " ", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(ojbkq_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(ok.FP8_FUNCTIONS)
    lib = ctypes.CDLL(ok.library_path)
    for name in names:
        assert hasattr(lib, name)
        assert getattr(ok.library(), name).argtypes is not None


def refused(name, good, word=None, status=-1, **bad):
    args = dict(good)
    assert set(bad) <= set(args)
    args.update(bad)
    lib = ok.library()
    assert getattr(lib, name)(*args.values()) == status, bad
    message = lib.ojbkq_last_error().decode()
    assert message and (word is None or word in message), (bad, message)


QUANT = dict(X=A, xtype=0, rows=10, m=200, ldx=200, features_first=0, block_rows=1, X8=A, ld8=208, scales=A, lds=4,
             stream=None)
NORM = dict(x=A, xtype=1, T=10, m=200, ldx=200, r_in=A, r_out=A, rtype=0, ldr=200, gain=A, eps=1e-5, X8=A, ld8=208,
            scales=A, lds=4, stream=None)
PRODUCT = dict(W8=A, ldw=208, ws=A, wtype=1, wrows=128, ldws=4, n=10, m=200, X8=A, ld8=208, scales=A, lds=4, T=10, Y=A,
               ytype=0, tokens_first=0, ldy=10, stream=None)
CODES = dict(packed=A, s=A, z=A, n=10, m=200, bits=4, group=128, X8=A, ld8=208, scales=A, lds=4, T=10, Y=A, ytype=0,
             tokens_first=0, ldy=10, workspace=None, bytes=0, stream=None)
BIG = 2 ** 62

EIGHT = [dict(X8=None), dict(X8=A + 8), dict(ld8=200), dict(ld8=192), dict(ld8=BIG), dict(scales=None), dict(scales=A + 2),
         dict(lds=2), dict(lds=0), dict(lds=6), dict(lds=BIG)]


@pytest.mark.parametrize("bad", EIGHT + [
    dict(X=None), dict(X=A + 2), dict(xtype=3), dict(xtype=-1), dict(rows=0), dict(rows=-5), dict(rows=2 ** 24 + 1), dict(m=0),
    dict(m=2 ** 20 + 1), dict(ldx=199), dict(ldx=BIG), dict(features_first=2), dict(block_rows=0), dict(block_rows=64),
    dict(features_first=1, block_rows=128), dict(features_first=1, ldx=9)])
def test_quantize(bad):
    refused("ojbkq_quantize_fp8", QUANT, **bad)


@pytest.mark.parametrize("bad", EIGHT + [
    dict(x=None), dict(x=A + 1), dict(xtype=3), dict(T=0), dict(m=0), dict(T=2 ** 24 + 1), dict(m=2 ** 20 + 1), dict(ldx=199),
    dict(ldx=BIG), dict(r_in=None), dict(r_out=None), dict(rtype=3), dict(ldr=199), dict(ldr=BIG), dict(r_in=A + 2),
    dict(r_out=A + 2), dict(gain=A + 2), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf"))])
def test_norm(bad):
    refused("ojbkq_rmsnorm_fp8", NORM, **bad)


SHARED = EIGHT + [dict(n=0), dict(m=0), dict(T=0), dict(n=2 ** 24 + 1), dict(m=2 ** 20 + 1), dict(T=2 ** 24 + 1), dict(Y=None),
                  dict(Y=A + 2), dict(ytype=3), dict(ytype=-1), dict(tokens_first=2), dict(ldy=9), dict(ldy=BIG),
                  dict(tokens_first=1, n=11)]


@pytest.mark.parametrize("bad", SHARED + [
    dict(W8=None), dict(W8=A + 4), dict(ldw=200), dict(ldw=BIG), dict(ws=None), dict(ws=A + 2), dict(wtype=2), dict(wtype=-1),
    dict(wrows=0), dict(wrows=2), dict(ldws=2), dict(wtype=0, ldws=1), dict(wtype=0, ldws=BIG)])
def test_product(bad):
    refused("ojbkq_matmul_fp8", PRODUCT, **bad)


@pytest.mark.parametrize("bad", SHARED + [
    dict(packed=None), dict(s=None), dict(z=None), dict(packed=A + 1), dict(s=A + 2), dict(z=A + 2), dict(bits=0), dict(bits=5),
    dict(bits=8), dict(group=64), dict(group=100), dict(group=130)])
def test_codes(bad):
    refused("ojbkq_dequant_matmul_fp8", CODES, **bad)


def test_more_than_four_bits_says_why():
    refused("ojbkq_dequant_matmul_fp8", CODES, word="exact", bits=5)


def test_tensors_that_the_binding_refuses():
    f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    v, s = torch.zeros(4, 128, dtype=torch.uint8).view(f8), torch.zeros(4, 4, dtype=torch.uint8).view(e8)[:, :1]
    x = torch.zeros(4, 128)
    for bad in (lambda: ok.quantize_fp8(x), lambda: ok.rmsnorm_fp8(x, None, 1e-5),          # not on the GPU
                lambda: ok.matmul_fp8(v, s, v, s), lambda: ok.quantize_fp8(x.double()), lambda: ok.quantize_fp8(x[0]),
                lambda: ok.quantize_fp8(x, block_rows=2), lambda: ok.matmul_fp8(x, s, v, s),
                lambda: ok.dequant_matmul_fp8(x, x, x, 128, 4, 128, v, s)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        ok.quantize_fp8([1.0])
