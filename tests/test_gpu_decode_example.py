"""examples/decode.py: the operators between two layers as a user strings them together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode.py")
    spec = importlib.util.spec_from_file_location("decode", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return torch, module, module.Decoder()


def test_a_prompt_and_its_tokens_one_by_one_agree(env):
    # the same tokens through the cache at once, in two pieces, and singly: the same keys and values are quantised, so the last
    # logits differ by fp16 roundings only.  Ten of them per block and a residual of 4 to 10 times a branch: 2 % of the logits' size.
    torch, D, model = env
    prompt = [(37 * i) % 1000 for i in range(90)]
    table = D.int32([[3, 1]])

    def run(pieces):
        at = 0
        for n in pieces:
            logits = model.forward(D.int32(prompt[at:at + n]), torch.arange(at, at + n, dtype=torch.int32, device="cuda"), table, D.int32([0, n]),
                                   D.int32([at + n]), n, at + n)
            at += n
        return logits.double()
    whole = run([90])
    for pieces in ([40, 50], [1] * 90, [33, 3, 1, 53]):
        got = run(pieces)
        assert (got - whole).norm() <= 0.02 * whole.norm(), pieces


def test_generates_and_greedy_is_the_sharpest(env):
    torch, D, model = env
    prompts = [list(range(5, 45)), [7], list(range(100, 230))]
    out = D.generate(model, prompts, 6)
    assert [len(o) for o in out] == [46, 7, 136] and all(o[:len(p)] == p for o, p in zip(out, prompts))
    assert all(0 <= t < 1000 for o in out for t in o)
    assert out == D.generate(model, prompts, 6)                                       # the same random numbers, the same tokens
    greedy = D.generate(model, prompts, 6, temperature=0.0)
    assert greedy == D.generate(model, prompts, 6, temperature=1.0, top_k=1, top_p=1.0, seed=5)
