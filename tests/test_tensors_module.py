"""The binding's host half (the module _tensors): what it allocates and what it refuses. No GPU is needed for either."""
import pytest
import torch

from paper_2606_12950_amd import _train


@pytest.fixture(scope="module")
def tensors():
    _train.load()
    return _train._tensors


def test_empties(tensors):
    a, none, b, c = tensors.empties(torch.zeros(2, dtype=torch.bfloat16), ((3,), False), None, ((2, 5), True), ((4, 0), False))
    assert none is None
    assert (a.shape, a.dtype) == ((3,), torch.float32) and (b.shape, b.dtype) == ((2, 5), torch.int32)
    assert (c.shape, c.dtype) == ((4, 0), torch.float32)
    assert all(t.is_contiguous() and t.device.type == "cpu" and not t.requires_grad for t in (a, b, c))
    assert tensors.empties(a) == ()


@pytest.mark.parametrize("args, error", [((), TypeError), ((3,), TypeError), ((torch.zeros(1), 3), TypeError),
                                         ((torch.zeros(1), ((1, 2, 3), False)), ValueError),
                                         ((torch.zeros(1), (("a",), False)), TypeError),
                                         ((torch.zeros(1), ((-1,), False)), RuntimeError)])
def test_empties_refusals(tensors, args, error):
    with pytest.raises(error):
        tensors.empties(*args)


def test_table_refusals(tensors):
    for bad in ([torch.zeros(1)], [None], [3]):
        with pytest.raises(TypeError, match="grads must be CUDA"):
            tensors.table(bad, "grads")
    with pytest.raises(TypeError):
        tensors.table((), "grads")
    assert tensors.table([], "grads") == (b"", b"", b"")


@pytest.mark.gpu
def test_table(tensors):
    a, b = torch.zeros(3, 5, device="cuda"), torch.zeros(7, dtype=torch.bfloat16, device="cuda")
    at, sizes, codes = tensors.table([a, b[1:], b[:0]], "grads")
    word = lambda x: int.from_bytes(x, "little")
    assert [word(at[i:i + 8]) for i in (0, 8)] == [a.data_ptr(), b.data_ptr() + 2]
    assert [word(sizes[i:i + 8]) for i in (0, 8, 16)] == [15, 6, 0]
    assert [word(codes[i:i + 4]) for i in (0, 4, 8)] == [0, 1, 1]
    with pytest.raises(ValueError, match="contiguous"):
        tensors.table([a.t()], "grads")
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        tensors.table([a.half()], "grads")


def test_missing_module_is_named(tmp_path, monkeypatch):
    monkeypatch.setattr(_train, "TENSORS_PATH", str(tmp_path / "missing.so"))
    monkeypatch.setattr(_train, "_lib", None)
    with pytest.raises(RuntimeError, match="missing.so"):
        _train.load()


def test_empties_types(tensors):
    like = torch.zeros(1, dtype=torch.bfloat16)
    assert [t.dtype for t in tensors.empties(like, ((1,), 0), ((1,), 1), ((1,), 2))] == [torch.float32, torch.int32, torch.bfloat16]
    for bad in (((1,), 3), ((1,), -1)):
        with pytest.raises(ValueError):
            tensors.empties(like, bad)
    with pytest.raises(TypeError):
        tensors.empties(like, ((1,),))
