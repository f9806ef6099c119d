"""The paged conversation of examples/, run whole at a small size."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("paged_conversation", os.path.join(ROOT, "examples", "paged_conversation.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [dict(prompt=700, budget=128, generate=5, turn=70), dict(prompt=1025, budget=300, generate=2, turn=33, batch=1, heads=12, kv_heads=4, dim=64)])
def test_conversation(sizes):
    m = load()
    r = m.run(**sizes)
    n, b = sizes["prompt"], sizes["budget"]
    assert r["rows"] == [n, b, b + sizes["generate"], b + sizes["generate"] + sizes["turn"], b]
    want = m.reference(r["q"], r["K"], r["V"])
    # the rows were read back rounded to bf16: in the logits (d terms of sizes about 1) and in V; the output is rounded once more
    d = r["q"].shape[-1]
    size = float((r["q"].double().abs().amax() * r["K"].double().abs().amax())) * d ** 0.5
    top = float(r["V"].double().abs().amax())
    assert float((r["out"].double() - want).abs().max()) <= top * (2 * 2.0 ** -9 * size + 3 * 2.0 ** -8)
