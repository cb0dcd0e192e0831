"""Every tensor that a call at the ends of a block is given has to lie on the current device.  On the CPU: tensors that say where they
lie, and a library that only notes that it was called."""
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


half = lambda *s: torch.zeros(*s, dtype=torch.float16)  # noqa: E731
f32 = lambda *s: torch.zeros(*s)  # noqa: E731
KEY = torch.zeros(2, dtype=torch.int64)
BYTES = torch.zeros(1 << 16, dtype=torch.uint8)
INTS = torch.zeros(3, dtype=torch.int32)

CALLS = {
    "dropout": (B.dropout, dict(x=half(3, 16), rng=KEY, residual=half(3, 16), out=half(3, 16)), dict(p=0.5)),
    "residual_norm": (B.residual_norm, dict(h=half(3, 16), branch=half(3, 16), gate=half(16), post_weight=half(16), post_bias=half(16), weight=half(16),
                                            bias=half(16), rng=KEY, total=half(3, 16), y=half(3, 16)), dict(post="rms", p=0.5)),
    "residual_norm, gate of every token": (B.residual_norm, dict(h=half(3, 16), branch=half(3, 16), gate=half(3, 16)), {}),
    "residual_norm_backward": (B.residual_norm_backward, dict(dy=half(3, 16), dtotal=half(3, 16), total=half(3, 16), branch=half(3, 16), gate=half(16),
                                                              post_weight=half(16), post_bias=half(16), weight=half(16), bias=half(16), rng=KEY,
                                                              workspace=BYTES), dict(post="rms", p=0.5)),
    "token_logprobs": (B.token_logprobs, dict(logits=half(3, 16), targets=INTS), dict(top=2)),
    "token_logprobs_backward": (B.token_logprobs_backward, dict(dlogprob=f32(3), dentropy=f32(3), logits=half(3, 16), targets=INTS, stats=f32(3, 3),
                                                                out=half(3, 16)), {}),
}
EVERY = [(call, name) for call, (_, tensors, _) in CALLS.items() for name in tensors]


def run(call, tensors, options):
    if "total" in tensors and "y" in tensors:
        tensors = dict(tensors)
        tensors["out"] = tensors.pop("total"), tensors.pop("y")
    return call(**tensors, **options)


@pytest.mark.parametrize("call", CALLS)
def test_all_on_the_current_device(library, call):
    f, tensors, options = CALLS[call]
    run(f, {k: placed(v) for k, v in tensors.items()}, options)
    assert len(library.called) == 1


@pytest.mark.parametrize("where", ["another GPU", "the host"])
@pytest.mark.parametrize("call,name", EVERY)
def test_one_that_is_not(library, call, name, where):
    f, tensors, options = CALLS[call]
    tensors = {k: v if k == name and where == "the host" else placed(v, 1 if k == name else 0) for k, v in tensors.items()}
    with pytest.raises(AssertionError):
        run(f, tensors, options)
    assert not library.called


def test_workspaces_are_packed(library):
    # a view's bytes are not all its own, or not there at all
    f, tensors, options = CALLS["residual_norm_backward"]
    for work in (BYTES[::2], BYTES[:1].expand(1 << 16)):
        with pytest.raises(AssertionError):
            f(**{k: placed(work if k == "workspace" else v) for k, v in tensors.items()}, **options)
    assert not library.called
