"""Gradients of the residual norm written over what they are made of, and calls that want some of them: in every kernel (one, two and three
pieces of a row to a thread, rolled), several rows to a workgroup, bit for bit what separate outputs get.  And rows that are not finite
beside others of the same workgroup."""
import pytest

import test_gpu_norm as N
from test_gpu_norm import EPS, env, host  # noqa: F401

pytestmark = pytest.mark.gpu
WIDTHS = [(2003, 72), (1031, 2000), (777, 5003), (601, 6001), (601, 9217), (601, 12000), (601, 12289)]
PAIRS = [(None, None), ("rms", None), (None, "row"), ("layer", "row"), ("rms", "token")]


class Call:
    """owq_residual_norm_backward with packed tensors and outputs of the caller's choice."""
    NAMES = ("dh", "dbranch", "dgate", "dpost_weight", "dpost_bias", "dweight", "dbias")

    def __init__(self, env, rows, width, post, gate, wide, seed=1):  # noqa: F811
        self.torch, self.B = torch, B = env
        g = torch.Generator("cuda").manual_seed(seed)
        rand = lambda *s, about=0.0: (about + torch.randn(*s, generator=g, device="cuda")).half()  # noqa: E731
        self.shape = rows, width
        self.post, self.gate = post, gate
        self.h_dtype = torch.float32 if wide else torch.float16
        self.x = {"dy": rand(rows, width), "dtotal": rand(rows, width).to(self.h_dtype), "total": rand(rows, width, about=0.5).to(self.h_dtype),
                  "branch": rand(rows, width, about=-0.3),
                  "gate": None if gate is None else rand(width, about=1) if gate == "row" else rand(rows, width, about=1)}
        self.vectors = [rand(width, about=1) if post else None, rand(width) if post else None, rand(width, about=1)]
        self.key = torch.tensor([seed, 3], dtype=torch.int64, device="cuda")
        kinds = {None: 0, "rms": 1, "layer": 2}
        self.desc = B.NormDesc(n_tokens=rows, width=width, type=0, h_type=2 if wide else 0, post=kinds[post], norm=2,
                               gate=kinds[None] if gate is None else 1 if gate == "row" else 2, site=4, eps=EPS, h_scale=1.25, branch_scale=0.6, p=0.1,
                               h_row=width, branch_row=width, gate_row=width, total_row=width, dy_row=width, dtotal_row=width)

    def outputs(self):
        torch, (rows, width) = self.torch, self.shape
        vector = lambda there=True: torch.empty(width, device="cuda") if there else None  # noqa: E731
        matrix = lambda dtype: torch.empty(rows, width, dtype=dtype, device="cuda")  # noqa: E731
        return {"dh": matrix(self.h_dtype), "dbranch": matrix(torch.float16),
                "dgate": None if self.gate is None else vector() if self.gate == "row" else matrix(torch.float16),
                "dpost_weight": vector(self.post), "dpost_bias": vector(self.post), "dweight": vector(), "dbias": vector()}

    def run(self, x, out, workspace=True):
        at = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
        need = self.B.owq_residual_norm_backward_workspace_bytes(self.desc) if workspace else 0
        work = self.torch.empty(need, dtype=self.torch.uint8, device="cuda") if need else None
        self.B.owq_residual_norm_backward(self.desc, at(x["dy"]), at(x["dtotal"]), at(x["total"]), at(x["branch"]), at(x["gate"]),
                                          *(at(v) for v in self.vectors), at(self.key), *(at(out[k]) for k in self.NAMES), at(work), need,
                                          self.torch.cuda.current_stream().cuda_stream)
        self.torch.cuda.synchronize()
        return out


def same(torch, got, want):
    return all((got[k] is None) == (want[k] is None) and (got[k] is None or torch.equal(got[k], want[k])) for k in want)


@pytest.mark.parametrize("wide", [False, True], ids=["16 bits", "fp32 residual"])
@pytest.mark.parametrize("post,gate", PAIRS)
@pytest.mark.parametrize("shape", WIDTHS, ids=str)
def test_over_the_inputs(env, shape, post, gate, wide):  # noqa: F811
    c = Call(env, *shape, post, gate, wide)
    want = c.run(c.x, c.outputs())
    for h, o in (("dtotal", None), ("total", None), (None, "branch"), (None, "dy"), ("dtotal", "dy"), ("total", "branch"), ("dtotal", "branch"), ("total", "dy")):
        x = {k: None if v is None else v.clone() for k, v in c.x.items()}
        out = c.outputs()
        if h:
            out["dh"] = x[h]
        if o:
            out["dbranch"] = x[o]
        assert same(c.torch, c.run(x, out), want), (h, o)


@pytest.mark.parametrize("post,gate", PAIRS)
@pytest.mark.parametrize("shape", WIDTHS, ids=str)
def test_some_gradients(env, shape, post, gate):  # noqa: F811
    c = Call(env, *shape, post, gate, False)
    torch = c.torch
    want = c.run(c.x, c.outputs())

    def part(*names, workspace=True):
        out = {k: v if k in names else None for k, v in c.outputs().items()}
        return c.run(c.x, out, workspace)
    # those of the rows alone need no workspace, a sum alone no rows
    for names in (("dh", "dbranch"), ("dbranch",)) + ((("dgate",),) if gate == "token" else ()):
        got = part(*names, workspace=False)
        assert all(torch.equal(got[k], want[k]) for k in names), names
    for name in ("dweight", "dbias") + (("dpost_weight", "dpost_bias") if post else ()) + (("dgate",) if gate == "row" else ()):
        got = part("dbranch", name)
        assert torch.equal(got[name], want[name]) and torch.equal(got["dbranch"], want["dbranch"]), name
    # nothing of the branch's: another kernel, whose roundings of the same steps are the compiler's
    got = part("dh", "dweight", "dbias")
    size = want["dh"].double().abs().amax(-1, keepdim=True)
    assert ((got["dh"].double() - want["dh"].double()).abs() <= 2.0 ** -10 * want["dh"].double().abs() + 1.2e-5 * size).all()
    rows = shape[0]
    x = (c.x["total"].double() - c.x["total"].double().mean(-1, keepdim=True))
    x = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
    for name, terms in (("dweight", c.x["dy"].double() * x), ("dbias", c.x["dy"].double())):
        # 64 additions and 4e-6 of a row's largest number in each term
        off = 4e-6 * terms.abs().sum(0) + (8e-6 * c.x["dy"].double().abs() * (1 + x.abs().amax(-1, keepdim=True))).sum(0)
        assert ((got[name].double() - terms.sum(0)).abs() <= off).all(), (name, rows)


@pytest.mark.parametrize("post,gate", PAIRS)
@pytest.mark.parametrize("shape", WIDTHS, ids=str)
def test_rows_that_are_not_finite(env, shape, post, gate):  # noqa: F811
    # first, middle and last rows of workgroups; the others get the bits that they get without them
    rows, width = shape
    c = Call(env, *shape, post, gate, False)
    torch, B = env
    want = c.run(c.x, c.outputs())
    options = dict(gate=c.x["gate"], post=post, post_weight=c.vectors[0], post_bias=c.vectors[1], norm="layer", weight=c.vectors[2], rng=c.key, p=0.1)
    fine = B.residual_norm(c.x["total"], c.x["branch"], **options)
    bad = torch.tensor([0, 3, rows // 3, rows // 2, rows - 200, rows - 1], device="cuda")
    at = torch.tensor([0, width - 1, width // 2, 7, 64, width // 3], device="cuda")
    x = {k: None if v is None else v.clone() for k, v in c.x.items()}
    x["total"][bad[:4], at[:4]] = float("nan")
    x["branch"][bad[4], :] = float("inf")                   # some of it stays
    x["dy"][bad[5], at[5]] = float("inf")
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[bad] = False
    got = c.run(x, c.outputs())
    for k in ("dh", "dbranch") + (("dgate",) if gate == "token" else ()):
        assert torch.equal(got[k][keep], want[k][keep]), k
    assert torch.isnan(got["dh"][bad[:4]]).all() and not torch.isfinite(got["dh"][bad[5]]).any()
    total, y = B.residual_norm(x["total"], x["branch"], **options)
    assert torch.equal(total[keep], fine[0][keep]) and torch.equal(y[keep], fine[1][keep])
    assert torch.isnan(y[bad[:5]]).all() and torch.equal(y[bad[5]], fine[1][bad[5]])
