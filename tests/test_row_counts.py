"""Numbers of rows and columns that the library's 32-bit counts do not hold are refused by the calls on tensors: counts from 2^32 on would
come out as small ones, and a part of the work be done.  On the CPU: tensors of one element's memory that say that they lie on a GPU."""
import pytest

torch = pytest.importorskip("torch")
B = pytest.importorskip("paper_2306_02272_amd.binding")


class Far(torch.Tensor):
    """A tensor of one element's memory that passes for a packed one on GPU 0."""
    __torch_function__ = torch._C._disabled_torch_function_impl
    is_cuda = True

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def stride(self):
        return (self.shape[1], 1)

    def new_empty(self, shape, dtype=None):
        return far(shape if isinstance(shape, tuple) else (shape,), dtype or self.dtype)


def far(shape, dtype):
    return torch.zeros(1, dtype=dtype).expand(shape).as_subclass(Far)


class Library:
    def __init__(self):
        self.called = []

    def __getattr__(self, name):
        def call(*args):
            self.called.append(name)
            return B.OWQ_OK
        return call


@pytest.fixture
def library(monkeypatch):
    library = Library()
    monkeypatch.setattr(B, "lib", lambda: library)
    monkeypatch.setattr(B, "_current_stream", lambda torch: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    return library


def dropout(rows, width):
    B.dropout(far((rows, width), torch.float16), far((2,), torch.int64), 0.5)


def logprobs(rows, width):
    B.token_logprobs(far((rows, width), torch.float16), far((rows,), torch.int32))


def logprobs_backward(rows, width):
    f = lambda *s: far(s, torch.float32)  # noqa: E731
    B.token_logprobs_backward(f(rows), f(rows), far((rows, width), torch.float16), far((rows,), torch.int32), f(3, rows))


def sample(rows, width):
    B.sample(far((rows, width), torch.float16), far((rows, width), torch.float32))


CALLS = {"dropout": dropout, "token_logprobs": logprobs, "token_logprobs_backward": logprobs_backward, "sample": sample}


@pytest.mark.parametrize("call", CALLS)
def test_the_largest_reach_the_library(library, call):
    for shape in ((2 ** 31 - 1, 1), (3, 2 ** 31 - 1)):
        CALLS[call](*shape)
    assert len(library.called) == 2


@pytest.mark.parametrize("shape", [(2 ** 31, 1), (2 ** 32 + 2, 1), (3, 2 ** 31), (3, 2 ** 32 + 5), (2 ** 33, 7)], ids=str)
@pytest.mark.parametrize("call", CALLS)
def test_larger_ones_do_not(library, call, shape):
    with pytest.raises(AssertionError):
        CALLS[call](*shape)
    assert not library.called
