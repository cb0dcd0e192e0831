"""examples/tune.py: norms, dropout, log-probabilities, their gradients and the low-bit layers' as a user strings them together."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import ends

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tune.py")
    spec = importlib.util.spec_from_file_location("tune", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return torch, module, module.Model()


def reference(torch, model, tokens, targets, key):
    """The same loss by torch in binary64 on the CPU, with the activations rounded where the library rounds them, and its gradients
    by differentiation (of each rounding as of the identity)."""
    half = lambda x: x + (x.detach().half().double() - x.detach())  # noqa: E731
    leaf = lambda t: t.detach().double().cpu().requires_grad_(True)  # noqa: E731

    def dense(low):
        L = low.layer
        groups = np.arange(L.d_in) // 128
        w = L.scale.view(np.float16).astype(np.float64)[:, groups] * (L.codes.astype(np.float64) - L.zero.view(np.float16).astype(np.float64)[:, groups])
        w[:, L.weak_idx] = 0
        return torch.from_numpy(w), leaf(low.weak), torch.from_numpy(L.weak_idx).long()
    weights = [dense(low) for low in model.layers()]
    vectors = {i: {k: leaf(b[k]) for k in ("gate", "post", "norm")} for i, b in enumerate(model.blocks)}
    vectors["first"] = leaf(model.first)
    h = leaf(model.embed[tokens.long()])
    norm = lambda x, w: x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * w  # noqa: E731
    linear = lambda x, w: half(x @ w[0].t() + x[:, w[2]] @ w[1].t())  # noqa: E731
    total, y = h, half(norm(h, vectors["first"]))
    for i in range(len(model.blocks)):
        o = linear(torch.relu(linear(y, weights[2 * i])), weights[2 * i + 1])
        factor = torch.from_numpy(ends.factor(key, model.p, i, *o.shape))
        total = total + vectors[i]["gate"] * factor * norm(o, vectors[i]["post"])
        y = half(norm(total, vectors[i]["norm"]))
    lp = torch.log_softmax(linear(y, weights[-1]), -1)
    t = targets.long().cpu()
    counted = t >= 0
    loss = -lp[torch.arange(len(t))[counted], t[counted]].mean()
    loss.backward()
    return loss.item(), [w[1].grad for w in weights], vectors, h.grad


def test_gradients_against_differentiation(env):
    # The activations are the reference's up to a last bit here and there, the gradients are rounded to fp16 eight times on the way
    # (2^-11 of an element each) and pass five low-bit products whose scales are (2^-11): as independent errors 0.2 % of a gradient's size.
    # An activation within a last bit of 0 (one in a thousand) may lie on the relu's other side, for sqrt(0.001) = 3 % of its
    # gradient at most where that is not as small as the others'; weak columns see 4 activations a row.  2 % is allowed.
    torch, T, model = env
    tokens, targets = T.batch(model)
    rng = torch.tensor([11, 3], dtype=torch.int64, device="cuda")
    loss, weak, vectors, dh = model.gradients(tokens, targets, rng)
    want_loss, want_weak, want_vectors, want_dh = reference(torch, model, tokens, targets, (11, 3))
    assert abs(loss - want_loss) < 0.002 * want_loss

    def near(got, want, what):
        want = want.to(got.device)
        off = ((got.double() - want).norm() / want.norm()).item()
        assert off <= 0.02, (what, off)
    for i, (g, w) in enumerate(zip(weak, want_weak)):
        near(g, w, i)
    for i in range(len(model.blocks)):
        for k in ("gate", "post", "norm"):
            near(vectors[i][k], want_vectors[i][k].grad, (i, k))
    near(vectors["first"], want_vectors["first"].grad, "first")
    near(dh, want_dh, "embedding")


def test_the_loss_moves_along_a_gradient(env):
    # a central difference along one layer's gradient, of a length that moves weak weights of 1/16 by hundredths
    torch, T, model = env
    tokens, targets = T.batch(model)
    rng = torch.tensor([5, 0], dtype=torch.int64, device="cuda")
    _, weak, _, _ = model.gradients(tokens, targets, rng)
    low, g = model.layers()[-1], weak[-1]
    old = low.weak.clone()
    step = (0.5 * g / g.norm()).float()
    low.update(old.float() + step)
    up, upper = model.loss(tokens, targets, rng), low.weak.float()
    low.update(old.float() - step)
    down, lower = model.loss(tokens, targets, rng), low.weak.float()
    low.update(old)
    slope = (g * (upper - lower)).sum().item()
    # logits are rounded to fp16 (2^-11 of about 4, of 96 rows' mean); the third derivative's share of the step: a percent
    assert abs((up - down) - slope) < 0.02 * slope + 2 * 4 * 2.0 ** -11 / np.sqrt(96)


def test_trains_and_repeats(env):
    torch, T, _ = env
    losses = T.train(T.Model(seed=3), 3)
    assert len(losses) == 3 and np.isfinite(losses).all()
    assert losses == T.train(T.Model(seed=3), 3)             # the same random bits: the same bits
