"""A layer as the package quantizes it, with and without a decode order, on
8-bit activations: codes packed with ``perm`` take activations in that order."""

import importlib.util
import json
import math
import os
import sys

import numpy as np
import pytest
import torch

import paper_2602_08376_amd as ok
from conftest import ROOT
from oracle import fp8 as o8
from synth import LayerConfig, make_layer
from test_gpu_fp8_pack import host
from test_gpu_fp8_products import check

pytestmark = pytest.mark.gpu
DEV = "cuda"
N, M, GROUP = 1030, 640, 128


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ok.library()


@pytest.fixture(scope="module", params=[False, True, "static"])
def layer(request):
    cfg = LayerConfig(key="act8", title="8-bit activations", n=N, m=M, T=2400, bits=4, group=GROUP, K=4, mus=(0.5,),
                      w_std=0.02, kind="heavy", data_seed=71, klein_seed=72)
    W, Xr, Xq = make_layer(cfg, device=DEV)
    q = ok.quantize_layer(W, Xr, Xq, 0.5, 4, GROUP, 4, 72, act_order=request.param)
    perm = q.perm if request.param is True else None
    order = np.arange(M) if perm is None else perm.cpu().numpy()
    assert request.param is not True or not np.array_equal(order, np.arange(M))
    # W_hat and its codes less zero points, in W's own order
    group_of = np.empty(M, dtype=np.int64)
    group_of[order] = np.arange(M) // GROUP
    w = host(q.codes) - host(q.zeros)[:, group_of]
    return q, perm, order, host(q.scales)[:, group_of] * w, w, Xq


# a token, a few, the kernel for few tokens, tiles for results in 16 bits and in float32
@pytest.mark.parametrize("T,y", [(1, torch.float32), (20, torch.float16), (300, torch.bfloat16), (2000, torch.bfloat16),
                                 (2400, torch.float32)])
def test_codes_in_decode_order(layer, T, y):
    q, perm, order, W, w, Xq = layer
    P = ok.pack_codes(q.codes, 4, perm)
    X = Xq[:, :T].contiguous()
    X8, xs = ok.quantize_fp8(X if perm is None else X.index_select(0, perm.long()), features_first=True)
    Y = ok.dequant_matmul_fp8(P, q.scales, q.zeros, M, 4, GROUP, X8, xs, dtype=y)
    v, e = host(X8), xs.view(torch.uint8).cpu().numpy().astype(np.int64) - 127
    X8 = o8.dequantize(v, e)
    check(Y, (W[:, order], w[:, order]), (X8, v))
    # and against the layer on the activations themselves, in W's order: a value
    # is off by half a step, 2^-4 of it or of the smallest normal number's scale
    X = host(X).T
    back = np.empty_like(X8)
    back[:, order] = X8
    least = np.empty_like(X8)
    least[:, order] = np.ldexp(1.0, np.repeat(e, 128, 1) - 10)
    off = np.abs(back - X)
    assert (off <= np.maximum(2.0 ** -4 * np.abs(X), least)).all()
    got, want = host(Y), W @ X.T
    half = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[y]
    # (the products' own sums, cut in tiles to 13 bits beside the largest of eight: below 2^-9 of the magnitudes)
    bound = np.abs(W) @ off.T + (2.0 ** -9 + 2.0 ** -14) * (np.abs(W) @ np.abs(X8[:, np.argsort(order)]).T)
    assert (np.abs(got - want) <= bound + half * (np.abs(want) + bound) + 1e-6 * (y == torch.float16)).all()


@pytest.mark.parametrize("order", [None, "positions", "static"])
def test_the_stacks_error_is_the_rounding_of_its_activations(order, capsys, monkeypatch):
    # Against the product of 16-bit activations on the same inputs, the error
    # grows by that of the activations' rounding, independent of it: at most
    # half a step, 2^-4 of a value.  Activations in another order than the codes
    # would be off by the whole result.
    spec = importlib.util.spec_from_file_location("bench", os.path.join(ROOT, "bench.py"))
    bench = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(bench)
    monkeypatch.setattr(sys, "argv", ["bench.py", "--mlp-stack", "--act8", "--stack-layers", "2", "--stack-dim", "512",
                                      "--stack-tokens", "2048"] + (["--act-order", order] if order else []))
    bench.main()
    lines = [json.loads(x) for x in capsys.readouterr().out.splitlines() if x.startswith("{")]
    assert len(lines) == 4
    for line in lines:
        for e8, e16 in zip(line["relative_output_error_act8"], line["relative_output_error"]):
            print(e8, e16)
            assert e8 <= math.hypot(e16, 2.0 ** -4)
