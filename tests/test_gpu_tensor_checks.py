"""The native checks of tensors give what their Python forms give, and refuse
what those refuse in the same words."""
import pytest
import torch

from gpu_util import need_gpu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _tensors():
    c = "cuda"
    a = torch.zeros(6, 40, device=c)
    yield from [a, a[:, 8:24], a[2:5], a[::2], a[3:4, 8:24], a[:1, ::2], a[:, :1], a[:, 4:5], a.t(), a[0], a[:0],
                a[:, :0], a[0, 0], a.expand(2, 6, 40), a[:1].expand(6, 40), a.bfloat16(), a.half(), a.double(),
                a.int(), a.to(torch.uint8), a.long(), a.cpu(), torch.nn.Parameter(a), a.clone().requires_grad_(),
                a.view(2, 3, 40), a.view(6, 1, 40), a.as_strided((1, 40), (7, 1)), a.as_strided((6, 1), (40, 7)),
                a.as_strided((3, 40), (20, 1)), None]


def _result(f, *args):
    try:
        return f(*args)
    except (ValueError, AttributeError, TypeError) as e:
        return type(e), str(e)


def test_native_checks_equal_pythons():
    P = need_gpu()
    _, _, at, rows_at = P._native()
    assert at is not P._at and rows_at is not P._rows_at
    found = refused = 0
    for t in _tensors():
        shapes = {(6, 40), (6, 16), (1, 40), (40,), (), (2, 6, 40)} | ({tuple(t.shape)} if t is not None else set())
        for shape in shapes:
            for dtype in (F32, BF16, torch.int32, torch.uint8, torch.float16):
                for dev in (0, 1):
                    for fast, slow in ((at, P._at), (rows_at, P._rows_at)):
                        if fast is rows_at and (t is None or len(shape) != 2):
                            continue
                        got, want = (_result(f, dev, "it", t, shape, dtype) for f in (fast, slow))
                        assert got == want, (t if t is None else (t.shape, t.stride(), t.dtype), shape, dtype)
                        refused += isinstance(got, tuple) and isinstance(got[0], type)
                        found += not (isinstance(got, tuple) and isinstance(got[0], type))
    assert found > 30 and refused > 300


def test_what_is_no_tensor_is_refused():
    P = need_gpu()
    _, _, at, rows_at = P._native()
    for f in (at, rows_at):
        for thing in (5, "tensor", [1.0], object()):
            with pytest.raises((AttributeError, TypeError)):
                f(0, "it", thing, (1,), F32)
        with pytest.raises(TypeError):
            f(0, "it")
