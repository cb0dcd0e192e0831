"""Workspaces that a caller brings: refused where they are not on the call's device, or not packed.  On the CPU: tensors that say where
they lie, and a library that only notes what it was called with."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
B = pytest.importorskip("paper_2306_02272_amd.binding")


class Placed(torch.Tensor):
    """A tensor that says that it lies on GPU `place`."""
    __torch_function__ = torch._C._disabled_torch_function_impl
    is_cuda = True

    def get_device(self):
        return self.place


def placed(x, place=0):
    x = x.as_subclass(Placed)
    x.place = place
    return x


class Library:
    def __init__(self):
        self.called = []

    def __getattr__(self, name):
        def call(*args):
            self.called.append((name, args))
            return B.OWQ_OK
        return call


@pytest.fixture
def library(monkeypatch):
    library = Library()
    monkeypatch.setattr(B, "lib", lambda: library)
    monkeypatch.setattr(B, "_current_stream", lambda torch: 0)
    return library


half = lambda *s: placed(torch.zeros(*s, dtype=torch.float16))  # noqa: E731
ints = lambda *s: placed(torch.zeros(*s, dtype=torch.int32))  # noqa: E731
table = lambda *s: placed(torch.zeros(*s))  # noqa: E731


def rope(work):
    q, k = half(3, 2, 32), half(3, 1, 32)
    return B.qk_norm_rope_backward(q, k, q, k, table(8, 16), table(8, 16), ints(3), half(32), half(32), workspace=work)


def attention(work):
    pages = placed(torch.zeros(4, 1, 1, 32 * 32 + 256, dtype=torch.uint8))
    return B.cache_attention(half(3, 2, 32), pages, ints(2, 2), ints(3), ints(2), workspace=work)


def linear(work):
    layer = object.__new__(B.OwqLinear)
    layer.torch, layer.handle, layer.d_in, layer.d_out, layer.desc = torch, None, 64, 32, B.LayerDesc()
    layer.desc.k = 4
    dy, x = (placed(torch.zeros(3, n, dtype=torch.float16)) for n in (32, 64))
    # its outputs are made on dy's device, which is the host here
    return layer.backward(dy, x, workspace=work)


CALLS = {"owq_qk_norm_rope_backward": rope, "owq_cache_attention": attention, "owq_linear_backward": linear}
BYTES = torch.zeros(1 << 12, dtype=torch.uint8)
plain = lambda v: v.value if isinstance(v, C._SimpleCData) else v  # noqa: E731


@pytest.mark.parametrize("call", CALLS)
def test_bytes_are_counted_in_any_type(library, call):
    for work in (placed(BYTES), placed(torch.zeros(1 << 10))):
        CALLS[call](work)
        name, args = library.called.pop()
        args = [plain(v) for v in args]
        assert name == call and args[args.index(work.data_ptr()) + 1] == 1 << 12


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("work", [BYTES, placed(BYTES, 1), placed(BYTES[::2]), placed(BYTES[:1].expand(1 << 12))],
                         ids=["the host", "another GPU", "every other byte", "one byte many times"])
def test_refused(library, call, work):
    with pytest.raises(AssertionError):
        CALLS[call](work)
    assert not library.called


def test_linear_backward_needs_its_input_beside_the_gradient(library):
    layer = object.__new__(B.OwqLinear)
    layer.torch, layer.handle, layer.d_in, layer.d_out, layer.desc = torch, None, 64, 32, B.LayerDesc()
    layer.desc.k = 4
    for x in (torch.zeros(3, 64, dtype=torch.float16), placed(torch.zeros(3, 64, dtype=torch.float16), 1)):
        with pytest.raises(AssertionError):
            layer.backward(placed(torch.zeros(3, 32, dtype=torch.float16)), x, workspace=placed(BYTES))
    assert not library.called
