"""The example's decoding steps in 4 bits (examples/decode_layer.py --bits 4):
products with 4-bit weights, append with head norms into the 4-bit cache and
its attention, one after the other.

Against fp64 on the weights, keys and values as they are held: each of the
layer's nine 16-bit results rounds by at most 2^-8 of itself, as in 16 bits,
and the norm of the error stays under 9 * 2^-8 of the result's.  A step in a
graph gives the bits of a step by itself."""
import importlib.util
import os
import sys

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
def test_decode_layer_in_4_bits(batch, steps):
    worst = load().main(["--batch", str(batch), "--steps", str(steps), "--bits", "4", "--check"])
    print(f"[decode layer] {batch} {steps}: {worst:.2e}", file=sys.stderr, flush=True)
    assert worst < 9 * 2.0 ** -8


@pytest.mark.parametrize("batch", [1, 33])
def test_steps_in_a_graph(batch):
    """The whole step, captured once and replayed over new tokens and
    positions, beside steps by themselves on another layer of the same weights."""
    print(f"[decode graph] {batch}", file=sys.stderr, flush=True)
    module = load()
    graphed, alone = (module.Layer(batch, bits=4) for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(5)
    tokens = [torch.randn(batch, alone.qkv.k, generator=gen, device="cuda").bfloat16() for _ in range(6)]
    x, pos = torch.empty_like(tokens[0]), torch.zeros(batch, dtype=torch.int32, device="cuda")
    x.copy_(tokens[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.step(x, pos)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = graphed.step(x, pos)
    for s, token in enumerate(tokens):
        x.copy_(token)
        pos.fill_(s)
        graph.replay()
        want = alone.step(token, torch.full_like(pos, s))
        torch.cuda.synchronize()
        assert torch.equal(y, want), f"step {s}"
