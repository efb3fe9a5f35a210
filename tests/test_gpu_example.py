"""The example that quantizes an output head, runs it in integers and scores it."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA GPU")]


def test_score_quantized_head():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    from score_quantized_head import main
    r = main(vocab=1500, din=256, group=64, tokens=2048, steps=4)
    # the head that drew the tokens scores them best; refinement recovers part of
    # what quantization lost; the bias was fitted to these very tokens
    assert r["full"] > r["refined"] > r["host"]
    assert r["refined with a bias"] > r["refined"]
    assert 0 < r["host in top 5"] <= 1 and 0 < r["refined in top 5"] <= 1
