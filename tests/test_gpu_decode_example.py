"""The attention block of examples/decode_step.py, captured and replayed, against plain torch on what its cache holds."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_step.py")


@pytest.mark.parametrize("cache", ["nvfp4", "bf16"])
@pytest.mark.parametrize("seqs,steps,heads,kv_heads", [(3, 40, 8, 2), (5, 300, 4, 4)])
def test_steps_replayed_from_a_graph(cache, seqs, steps, heads, kv_heads):
    spec = importlib.util.spec_from_file_location("decode_step", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    r = module.run(seqs, steps, heads, kv_heads, cache)
    assert r["length"] == steps
    # bf16 results: half a unit in the last place of the largest value, and the sums'; log-sum-exp of scores of a few units in binary32
    assert r["error"] <= 2.0 ** -8 and r["lse_error"] <= 1e-5
