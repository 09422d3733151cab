"""The example that learns an index's dense rows: embedding, loss, gradients, 8-bit scores and the index, together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
def test_learned_rows_find_their_documents(bf16):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "learn_rows.py")
    spec = importlib.util.spec_from_file_location("learn_rows", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.main(["--docs", "1000", "--dim", "64", "--steps", "40"] + (["--bf16"] if bf16 else []))
    assert r["losses"][-1] < 0.5 * r["losses"][0]        # ln(1000) = 6.9 to begin with
    assert r["found"] > 0.5                              # 0.001 by chance
    assert r["found8"] > r["found"] - 0.05
    assert r["found_ix"] > 0.9
