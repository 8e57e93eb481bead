"""The example that walks, trains and answers with the row-wise choices, and its module's gradients."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("walk_experts", os.path.join(ROOT, "examples", "walk_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_it_learns_to_step_along_edges(example):
    r = example.main(steps=60, walkers=512)
    # log(400) = 6.0 without knowledge of the graph; a walk step has at most log(max degree) < 3.5
    assert r["losses"][-1] < 0.7 * r["losses"][0]
    assert r["on_an_edge"] > 0.5  # a uniform draw meets a neighbour in about 10 of 400 cases
    assert (r["ids"] >= 0).all() and (r["kept"] <= 20).all() and torch.isfinite(r["logp"]).all()


def test_walks_stay_on_edges_and_repeat(example):
    from paper_2609_27209_gb300 import synth

    dev = torch.device("cuda:0")
    table = example.neighbour_scores(*synth.random_connected(300, 900, seed=3, weighted=True), dev)
    runs = []
    for _ in range(2):
        g = torch.Generator(device=dev).manual_seed(5)
        runs.append(example.walk(table, torch.arange(300, device=dev), 6, g))
    assert torch.equal(*runs)
    ids = torch.where(table[1] > -torch.inf, table[0].long(), -1)
    for a, b in zip(runs[0].t()[:-1], runs[0].t()[1:]):
        assert (ids[a] == b[:, None]).any(1).all()


@pytest.mark.parametrize("score", [0, 1])
def test_module_gradients_against_torch(example, score):
    """The same experts in plain float64 torch operations, with the module's own choices."""
    torch.manual_seed(score)
    dev = torch.device("cuda:0")
    m = example.Experts(32, 6, 3, score).to(dev).eval()
    m.b.data.normal_()
    x = torch.randn(50, 32, device=dev, requires_grad=True)
    g = torch.randn(50, 32, device=dev)
    m(x).backward(g)
    got = [x.grad, m.router.grad, m.A.grad, m.b.grad]

    x64, router, A, b = (t.detach().double().requires_grad_() for t in (x, m.router, m.A, m.b))
    logits = x64 @ router
    s = torch.sigmoid(logits) if score == 1 else torch.softmax(logits, 1)
    top = s.topk(3, 1)
    w = top.values / top.values.sum(1, keepdim=True)
    y = torch.relu(torch.einsum("td,edf->tef", x64, A) + b)
    out = (w[:, :, None] * y.gather(1, top.indices[:, :, None].expand(-1, -1, 32))).sum(1)
    out.backward(g.double())
    for have, want in zip(got, (x64.grad, router.grad, A.grad, b.grad)):
        # float32 products of depth 32 and 50, a chain of three: 1e-5 of the largest entry is far above
        assert (have.double() - want).abs().max() <= 1e-5 * want.abs().max()
