"""A whole tuning step of examples/tune.py in a graph: forward, log-probabilities and all gradients, with the step of the random bits moved
between replays.  Every replay gives the bits that the eager calls give at the same step."""
import pytest

from test_gpu_tune_example import env  # noqa: F401

pytestmark = pytest.mark.gpu


def test_replays_with_a_step_that_moves(env):  # noqa: F811
    torch, T, model = env
    tokens, targets = T.batch(model)
    count = int((targets >= 0).sum())
    rng = torch.tensor([21, 0], dtype=torch.int64, device="cuda")

    def flat(lp, weak, vectors, dh):
        return [lp, *weak, *(v for i in range(len(model.blocks)) for v in vectors[i].values()), vectors["first"], dh]
    eager = []
    for step in range(4):
        rng[1] = step
        eager.append([t.clone() for t in flat(*model.step(tokens, targets, count, rng))])
    assert not torch.equal(eager[0][0], eager[1][0])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            captured = flat(*model.step(tokens, targets, count, rng))
        for step in (0, 1, 2, 3, 1):
            for t in captured:
                t.fill_(7)                               # eager work between the replays
            rng[1] = step
            other = model.loss(tokens, targets, rng)
            stream.synchronize()
            graph.replay()
            stream.synchronize()
            for i, (a, b) in enumerate(zip(captured, eager[step])):
                assert torch.equal(a, b), (step, i)
            assert abs(other + eager[step][0].sum().item() / count) < 1e-5 * abs(other)
