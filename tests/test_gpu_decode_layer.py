"""The example's decoding steps (examples/decode_layer.py) against the same
layer in fp64.  Each of the layer's nine 16-bit results (two norms, five
products, the turned queries, the attention) rounds by at most 2^-8 of itself,
2^-9 at random, and the errors of a step add like independent ones or better:
the norm of the error stays under 9 * 2^-8 of the result's."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("decode_layer", os.path.join(ROOT, "examples", "decode_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("batch,steps", [(1, 3), (8, 20), (33, 4)])
def test_decode_layer(batch, steps):
    assert load().main(["--batch", str(batch), "--steps", str(steps), "--check"]) < 9 * 2.0 ** -8
