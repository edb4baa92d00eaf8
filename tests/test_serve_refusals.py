"""CPU tests: the binding of the decoding-step operators words what it refuses
where arguments are missing, go together, or are no tensors at all."""
import pytest

torch = pytest.importorskip("torch")

import paper_2503_01253_amd as nm  # noqa: E402


def test_arguments_that_go_together():
    x = torch.zeros(4, 32)
    for kw in (dict(cos=x), dict(sin=x)):
        with pytest.raises(ValueError, match="cos and sin"):
            nm.nmspmm_kv_append(None, x, x, x, x, **kw)
    with pytest.raises(ValueError, match="q_out without q"):
        nm.nmspmm_kv_append(None, x, x, x, x, q_out=x)


def test_handles_that_are_none():
    x = torch.zeros(4, 32)
    for bad in (None, x, "weight"):
        with pytest.raises(TypeError, match="weight must be a HalfWeight"):
            nm.nmspmm_half_run(x, bad, x)
        with pytest.raises(TypeError, match="cache must be a KvCache"):
            nm.nmspmm_kv_append(bad, x, x, x, x)
        with pytest.raises(TypeError, match="cache must be a KvCache"):
            nm.nmspmm_kv_attend(bad, x, x, x)
