"""``bench.py --mlp-stack --act8``: the stack with 8-bit activations, run as the
command runs it, at a small size."""

import importlib.util
import json
import math
import os
import sys

import pytest
import torch

from conftest import ROOT


@pytest.mark.gpu
@pytest.mark.parametrize("order", [None, "positions", "static"])
def test_stack_of_layers_with_8_bit_activations(order, capsys, monkeypatch):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("bench", os.path.join(ROOT, "bench.py"))
    bench = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(bench)
    L = 2
    monkeypatch.setattr(sys, "argv", ["bench.py", "--mlp-stack", "--act8", "--stack-layers", str(L), "--stack-dim", "512",
                                      "--stack-tokens", "2048"] + (["--act-order", order] if order else []))
    bench.main()
    lines = [json.loads(x) for x in capsys.readouterr().out.splitlines() if x.startswith("{")]
    assert len(lines) == 4
    for line in lines:
        e8, e16 = line["relative_output_error_act8"], line["relative_output_error"]
        assert len(e8) == len(e16) == L
        assert all(len(line[k]) == L and min(line[k]) > 0 for k in ("quantize_fp8_ms", "dequant_matmul_fp8_ms"))
        assert all(0 < v < math.inf for v in e8 + e16)
    assert line["dequant_matmul_fp8_tflops"] > 0


def test_the_option_needs_the_stack(monkeypatch):
    spec = importlib.util.spec_from_file_location("bench", os.path.join(ROOT, "bench.py"))
    bench = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(bench)
    for argv in (["--act8"], ["--act8", "--mlp-stack", "--adaptive"]):
        monkeypatch.setattr(sys, "argv", ["bench.py"] + argv)
        with pytest.raises(SystemExit):
            bench.parse()
