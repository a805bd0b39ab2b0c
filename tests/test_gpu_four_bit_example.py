"""The example of the table operators runs, and what it returns belongs together."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example_runs():
    spec = importlib.util.spec_from_file_location(
        "four_bit_step", os.path.join(ROOT, "examples", "four_bit_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    r = mod.run(V=5000, d=256, sessions=4, k=3, steps=3)
    again = mod.run(V=5000, d=256, sessions=4, k=3, steps=3)
    kept = set(r["keep"].tolist())
    for (n, t), (n2, t2) in zip(r["history"], again["history"]):
        assert ((n >= 0) & (n <= 3)).all() and set(t.tolist()) <= kept
        assert torch.equal(n, n2) and torch.equal(t, t2)
    # 4.5 bits a weight and 4 bytes a row, for 16 in bf16
    assert r["bits4"] < 0.3 * r["bf16"]
    touched = (r["grad"] != 0).any(1).nonzero()[:, 0]
    assert set(touched.tolist()) == set(torch.cat(r["seen"]).tolist())
    assert torch.equal(r["grad"], again["grad"])
