"""What the binding of the decoding-step operators refuses of its tensors:
TypeError for what is no CUDA tensor of the type, ValueError for its shape."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import numpy as np  # noqa: E402

import paper_2503_01253_amd as nm  # noqa: E402

WRONG = (None, [1.0], 3, "x", np.zeros((4, 64), np.float32))


def new(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def test_half_run():
    k, n, N, M, V = 64, 64, 4, 32, 32
    weight = nm.nmspmm_half_pack(new(8, n), new(8, 2, dtype=torch.uint8), n, k, N, M, V)
    good = dict(A=new(4, k), C=new(4, n), bias=new(n, dtype=torch.float32), mul=new(4, n), residual=new(4, n))

    def run(**kw):
        a = {**good, **kw}
        return nm.nmspmm_half_run(a.pop("A"), weight, a.pop("C"), **a)

    assert run() is good["C"]
    for name in good:
        for x in WRONG + (good[name].cpu(), good[name].to(torch.int32)):
            if x is None and name not in ("A", "C"):
                continue
            with pytest.raises(TypeError, match=f"{name} must be a CUDA tensor"):
                run(**{name: x})
        for x in (good[name][:-1], good[name][None], torch.cat((good[name], good[name]), -1)[..., ::2]):
            with pytest.raises(ValueError):
                run(**{name: x})
    with pytest.raises(ValueError, match="act"):
        run(act="tanh")
    for x in (new(256), [0], "ws"):
        with pytest.raises(TypeError, match="workspace"):
            run(workspace=x)


@pytest.fixture
def cache():
    return nm.nmspmm_kv_cache(new(4, 16, 2, 64), new(4, 16, 2, 64), new(3, 2, dtype=torch.int32))


def test_append(cache):
    i32, f32 = dict(dtype=torch.int32), dict(dtype=torch.float32)
    good = dict(k=new(3, 2, 64), v=new(3, 2, 64), seq=new(3, **i32), pos=new(3, **i32), cos=new(8, 16, **f32),
                sin=new(8, 16, **f32), q=new(3, 4, 64), q_out=new(3, 4, 64))
    assert nm.nmspmm_kv_append(cache, **good) is good["q_out"]
    for name in good:
        for x in WRONG + (good[name].cpu(), good[name].to(torch.float64)):
            if x is None and name in ("cos", "sin", "q", "q_out"):
                continue
            with pytest.raises(TypeError, match=f"{name} must be a CUDA tensor"):
                nm.nmspmm_kv_append(cache, **{**good, name: x})
        for x in (good[name][:-1], good[name][None], torch.cat((good[name], good[name]), -1)[..., ::2]):
            with pytest.raises(ValueError):
                nm.nmspmm_kv_append(cache, **{**good, name: x})


def test_attend(cache):
    good = dict(q=new(3, 4, 64), lengths=new(3, dtype=torch.int32), out=new(3, 4, 64),
                lse=new(3, 4, dtype=torch.float32))
    assert nm.nmspmm_kv_attend(cache, **good) is good["out"]
    for name in good:
        for x in WRONG + (good[name].cpu(), good[name].to(torch.float64)):
            if x is None and name == "lse":
                continue
            with pytest.raises(TypeError, match=f"{name} must be a CUDA tensor"):
                nm.nmspmm_kv_attend(cache, **{**good, name: x})
        for x in (good[name][:-1], good[name][None], torch.cat((good[name], good[name]), -1)[..., ::2]):
            with pytest.raises(ValueError):
                nm.nmspmm_kv_attend(cache, **{**good, name: x})


def test_cache_sizes_beyond_32_bits():
    """The C structure holds a page's sizes in 32 bits: 2^32 + 16 would be 16."""
    table = new(1, 1, dtype=torch.int32)
    for shape in ((1, 2 ** 32 + 16, 1, 64), (1, 16, 2 ** 32 + 2, 64)):
        far = new(1, 1, 1, 64).expand(shape)
        with pytest.raises(ValueError, match="32-bit"):
            nm.nmspmm_kv_cache(far, far, table)
