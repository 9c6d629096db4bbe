"""The example that runs the serving operators and the clustering together, as a program would."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("clustered_decode", os.path.join(ROOT, "examples", "clustered_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("tokens", [500, 4096])
def test_attention_over_the_nearest_clusters_carries_most_of_the_mass(tokens):
    r = load().main(tokens)
    assert r["read"] < 0.6 * r["tokens"]              # a part of the cache is read
    assert 0.5 < r["mass"] <= 1.001                   # and it holds most of what the full attention looks at
    assert torch.isfinite(r["result"].float()).all() and r["error"] < 0.5
