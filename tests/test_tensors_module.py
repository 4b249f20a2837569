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


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_whole_calls_and_the_binding_agree(tensors, dtype):
    """What the native module takes whole gives the bits that the binding's own path (outputs given) gives."""
    import paper_2606_12950_amd as M
    r = torch.Generator().manual_seed(3)
    d = lambda *s: torch.randn(*s, generator=r).cuda()
    x, w, b, gz = d(37, 64).to(dtype), d(48, 64).to(dtype), d(48), d(37, 48).to(dtype)
    assert torch.equal(M.layer(x, w, b), M.layer(x, w, b, out=torch.empty_like(gz)))
    one = M.layer_grad(x, w, gz, relu_input=True)
    two = M.layer_grad(x, w, gz, relu_input=True, out=M.LayerGrad(torch.empty_like(x), torch.empty(48, 64, device="cuda"), torch.empty(48, device="cuda")))
    assert type(one) is M.LayerGrad and all(map(torch.equal, one, two))
    assert M.layer_grad(x, w, gz, want_x=False).x is None
    t = torch.arange(37, dtype=torch.int32, device="cuda")
    for k, token in ((0, None), (3, t), (16, t)):
        one = M.logprobs(gz, token, k=k)
        two = M.logprobs(gz, token, k=k, out=M.Logprobs(*(None if u is None else torch.full_like(u, 7) for u in one)))
        assert type(one) is M.Logprobs and (one.logprob is None) == (token is None)
        assert all(u is v is None or torch.equal(u, v) for u, v in zip(one, two))
    g = d(37)
    for token, gl, ge in ((t, g, g), (t, g, None), (None, None, g)):
        one = M.logprobs_grad(gz, token, two.stats, two.entropy, gl, ge)
        assert torch.equal(one, M.logprobs_grad(gz, token, two.stats, two.entropy, gl, ge, out=torch.empty_like(gz)))
    grads = [x, w, b]
    one, two = [torch.empty_like(u) for u in grads], [torch.empty_like(u) for u in grads]
    norms = M.clip_gradients(grads, 0.5, out=one), M.clip_gradients(grads, 0.5, out=two, norm=torch.empty(1, device="cuda"))
    assert torch.equal(*norms) and all(map(torch.equal, one, two))


@pytest.mark.gpu
def test_calls_that_are_not_plain_are_left_to_the_binding(tensors):
    x, w, b = torch.zeros(8, 32, device="cuda"), torch.zeros(16, 32, device="cuda"), torch.zeros(16, device="cuda")
    t = torch.zeros(8, dtype=torch.int32, device="cuda")
    for bad in ((x.cpu(), w, b), (x, w.bfloat16(), b), (x[:, ::2], w[:, ::2], b), (x, w, b[:8]), (x, w, b.double()), (x, w, None),
                (x[:, :24], w[:, :24].contiguous(), b), (3, w, b), (x, w.to_sparse(), b)):
        assert tensors.layer(*bad, True, 0) is None
    for bad in ((x, w, x), (x, w[:8], w), (x, None, x)):
        assert tensors.layer_grad(*bad, True, True, 0) is None
    for bad in ((x.t(), None, 0), (x, t[:7], 0), (x, t.long(), 0), (x, t, 17), (x, t, -1), (x, t, "2"), (x[0], None, 0), (x.half(), t, 0)):
        assert tensors.logprobs(*bad, True, True, 0) is None
    s, e = torch.zeros(8, 2, device="cuda"), torch.zeros(8, device="cuda")
    for bad in ((x, t, s, e, None, e), (x, None, s, e, None, None), (x, None, s, None, None, e), (x, t, s[:4], e, e, e), (x, t, None, e, e, e)):
        assert tensors.logprobs_grad(*bad, 0) is None
    for bad in (([], 1.0, None), ([x.cpu()], 1.0, None), ([x], 1, None), ([x], 1.0, []), ([x], 1.0, [x[:4]]), ([x], -1.0, None), ((x,), 1.0, None)):
        assert tensors.clip(*bad, 0) is None
