"""The operators of training and answering used together: a step of the gated experts against plain torch
operators in float64, captured and replayed, from several threads, and the example that trains them."""
import importlib.util
import os
import threading

import numpy as np
import pytest
import torch

from oracle import expert_oracle as X
from paper_2609_27209_gb300 import erc

from ._gpu import dev

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("walk_experts", os.path.join(ROOT, "examples", "walk_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("act", [0, 1])
def test_a_training_step_against_torch(example, act):
    """The whole step in float32 against float64 with the step's own experts and dropped entries."""
    torch.manual_seed(act)
    rows, width, E, k, n = 70, 24, 6, 2, 301
    m = example.GatedExperts(width, E, k, inner=36, p=0.25, act=act).to(dev())
    head = torch.randn(width, n, device=dev(), requires_grad=True)
    x = torch.randn(rows, width, device=dev(), requires_grad=True)
    ids = torch.randint(-1, n, (rows,), device=dev(), dtype=torch.int32)
    g, h = torch.randn(2, rows, device=dev())

    out = m(x)
    logp, entropy = example.Scored.apply(out @ head, ids)
    (logp * g + entropy * h).sum().backward()
    got = [x.grad, head.grad, m.router.grad, m.w_in.grad, m.w_out.grad]

    x64, head64, router, w_in, w_out = (t.detach().double().requires_grad_() for t in (x, head, m.router, m.w_in, m.w_out))
    s = torch.softmax(x64 @ router, 1)
    top = s.topk(k, 1)
    weights = top.values / top.values.sum(1, keepdim=True)
    gate, up = torch.einsum("td,efd->tef", x64, w_in).split(36, 2)
    inner = (torch.nn.functional.silu(gate) if act == 0 else torch.nn.functional.gelu(gate)) * up
    y = torch.einsum("tef,edf->ted", inner, w_out)
    mixed = (weights[:, :, None] * y.gather(1, top.indices[:, :, None].expand(-1, -1, width))).sum(1)
    keep = torch.from_numpy(X.dropout_keep(rows * width, 0.25, 1)).view(rows, width).to(dev())
    out64 = x64 + torch.where(keep, mixed / 0.75, 0.0)
    log_p = torch.log_softmax(out64 @ head64, 1)
    picked = torch.where(ids >= 0, log_p.gather(1, ids.clamp(min=0).long()[:, None])[:, 0], 0.0)
    entropy64 = -(log_p.exp() * log_p).sum(1)
    (picked * g.double() + entropy64 * h.double()).sum().backward()
    # a chain of products of depth 24, 36 and 24 and a softmax over 301 entries, each within some 300 U of its
    # magnitudes' sum: 1e-4 of the largest entry is above
    assert (logp.double() - picked).abs().max() <= 1e-4 * picked.abs().max()
    assert (entropy.double() - entropy64).abs().max() <= 1e-4 * entropy64.abs().max()
    for have, want in zip(got, (x64.grad, head64.grad, router.grad, w_in.grad, w_out.grad)):
        assert (have.double() - want).abs().max() <= 1e-4 * want.abs().max()


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_a_captured_step_replays_as_the_eager_one(kind):
    g = torch.Generator(device=dev()).manual_seed(3)
    rows, width, inner, E, k, n = 200, 64, 96, 8, 2, 1000
    mk = lambda *s, scale=1.0: (scale * torch.randn(*s, generator=g, device=dev())).to(kind)  # noqa: E731
    router, w_in, w_out = mk(width, E), mk(E, 2 * inner, width, scale=0.1), mk(E, width, inner, scale=0.1)
    head, x, key = mk(width, n), mk(rows, width), torch.tensor([7], device=dev())
    ids = torch.arange(rows, dtype=torch.int32, device=dev())
    words = torch.randint(-(2**62), 2**62, (rows,), generator=g, device=dev())
    ones = torch.ones(rows, device=dev())

    def step():
        logits = x @ router
        experts, weights = erc.erc_route(logits, k)
        offsets, _, slot = erc.erc_expert_plan(experts, E)
        xs = erc.erc_expert_gather(x, slot, offsets)
        y, pre = erc.erc_expert_ffn(xs, offsets, w_in, w_out, keep=True)
        out = erc.erc_dropout(erc.erc_expert_combine(y, slot, weights), 0.2, key, residual=x)
        scores = out @ head
        logp, entropy, norm, top, _ = erc.erc_score_rows(scores, ids, k=5)
        drawn, _, _ = erc.erc_sample_rows(scores, words, top_k=20)
        dscores = erc.erc_score_rows_backward(scores, ids, norm, ones, entropy, ones)
        dout = (dscores @ head.t()).contiguous()
        dy, dweights = erc.erc_expert_combine_backward(erc.erc_dropout(dout, 0.2, key), y, slot, offsets, weights)
        dxs, dw_in, dw_out = erc.erc_expert_ffn_backward(dy, xs, pre, offsets, w_in, w_out)
        dx = erc.erc_expert_combine(dxs, slot)
        dlogits = erc.erc_route_backward(logits, experts, dweights)
        return logp, entropy, top, drawn, dx, dw_in, dw_out, dlogits

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in range(3):
        x.copy_(torch.randn(rows, width, generator=torch.Generator().manual_seed(seed)))
        key.fill_(100 + seed)
        graph.replay()
        for a, b in zip(held, step()):
            assert torch.equal(a, b)


def test_two_captured_graphs_with_workspaces_of_their_own_run_at_once():
    offsets = torch.tensor([0, 90, 90, 300], device=dev())
    w_in, w_out = torch.randn(3, 64, 40, device=dev()).half() * 0.1, torch.randn(3, 40, 32, device=dev()).half() * 0.1
    scores = torch.randn(5, 700001, device=dev())
    graphs, held, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    xs = [torch.randn(300, 40, device=dev()).half() for _ in range(2)]

    def step(i):
        y, pre = erc.erc_expert_ffn(xs[i], offsets, w_in, w_out, keep=True)
        return (y, *erc.erc_expert_ffn_backward(y, xs[i], pre, offsets, w_in, w_out), *erc.erc_score_rows(scores * (i + 1), k=9)[1:])

    want = [step(i) for i in range(2)]
    torch.cuda.synchronize()
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=streams[i]):
            held.append(step(i))
        graphs.append(graph)
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(held[i], want[i]))


def test_calls_from_several_threads():
    offsets = torch.tensor([0, 40, 130], device=dev())
    w_in, w_out = torch.randn(2, 48, 64, device=dev()).bfloat16(), torch.randn(2, 64, 24, device=dev()).bfloat16()
    xs = torch.randn(130, 64, device=dev()).bfloat16()
    rows = {n: torch.randn(6, n, device=dev()) for n in (200, 9000, 30000, 150000)}
    calls = [lambda: erc.erc_expert_ffn(xs, offsets, w_in, w_out, keep=True), lambda: (erc.erc_dropout(xs, 0.3, 5),)]
    calls += [lambda n=n, k=k: [t for t in erc.erc_score_rows(rows[n], k=k) if t is not None] for n in rows for k in (0, 32)]
    want = [call() for call in calls]
    torch.cuda.synchronize()
    bad = []

    def work(seed):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for at in np.random.default_rng(seed).permutation(len(calls) * 4):
                    got = calls[at % len(calls)]()
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[at % len(calls)])):
                        bad.append(at % len(calls))
        except Exception as e:  # noqa: BLE001
            bad.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for thread in threads:
        thread.start()
    for thread in threads:
        thread.join()
    assert not bad


def test_the_gated_example_runs(example):
    r = example.main(steps=3, walkers=64, gated=True)
    assert len(r["losses"]) == 3 and np.isfinite(r["losses"]).all()
    assert (r["ids"] >= 0).all() and torch.isfinite(r["logp"]).all()


def every_call():
    x = torch.randn(8, 16, device=dev())
    ids = torch.zeros(8, dtype=torch.int32, device=dev())
    at = torch.tensor([0, 5, 8], device=dev())
    w_in, w_out = torch.randn(2, 24, 16, device=dev()), torch.randn(2, 16, 12, device=dev())
    pre = torch.randn(8, 24, device=dev())
    norm, one = torch.zeros(8, 2, device=dev()), torch.ones(8, device=dev())
    return [lambda **kw: erc.erc_score_rows(x, ids, k=2, **kw), lambda **kw: erc.erc_expert_ffn(x, at, w_in, w_out, **kw),
            lambda **kw: erc.erc_expert_ffn_backward(x, x, pre, at, w_in, w_out, **kw),
            lambda: erc.erc_score_rows_backward(x, ids, norm, one), lambda: erc.erc_dropout(x, 0.5, 3)]


def refused(call, **kw):
    with pytest.raises(erc.ErcError) as e:
        call(**kw)
    assert e.value.status == erc.ERC_ERR_INVALID_ARG


def test_tensors_of_a_device_that_is_not_current_are_refused(monkeypatch):
    calls = every_call()
    for call in calls:
        call()
    torch.cuda.synchronize()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in calls:
        refused(call)


def test_workspaces_of_another_type_device_or_layout_are_refused():
    for call in every_call()[:3]:
        call(ws=torch.empty(1 << 20, dtype=torch.uint8, device=dev()))
        for ws in (torch.empty(1 << 20, dtype=torch.uint8), torch.empty(1 << 20, device=dev()),
                   torch.empty(1 << 20, dtype=torch.uint8, device=dev())[::2], 1 << 20):
            refused(call, ws=ws)


def test_a_workspace_may_start_anywhere_and_says_that_the_work_ended_well():
    offsets = torch.tensor([0, 100, 260], device=dev())
    w_in, w_out = torch.randn(2, 64, 48, device=dev()).half(), torch.randn(2, 48, 32, device=dev()).half()
    x = torch.randn(260, 48, device=dev()).half()
    want, _ = erc.erc_expert_ffn(x, offsets, w_in, w_out)
    need = erc.lib().erc_expert_ffn_workspace_size(erc.ctypes.byref(erc._ffn_shape(x, "xs", offsets, w_in, w_out, 0)))
    for lead in (0, 1, 8, 255):
        buffer = torch.full((need + 256,), 77, dtype=torch.uint8, device=dev())
        ws = buffer[lead:lead + need]
        got, _ = erc.erc_expert_ffn(x, offsets, w_in, w_out, ws=ws)
        assert torch.equal(got, want)
        first = -ws.data_ptr() % 256 + lead  # the first 256-byte boundary
        assert not buffer[first:first + 4].any()
        assert (buffer[:lead] == 77).all() and (buffer[lead + need:] == 77).all()


def test_numbers_that_do_not_fit_are_refused():
    x = torch.randn(4, 16, device=dev())
    ids = torch.zeros(4, dtype=torch.int32, device=dev())
    at = torch.tensor([0, 4], device=dev())
    w_in, w_out = torch.randn(1, 24, 16, device=dev()), torch.randn(1, 16, 12, device=dev())
    for call in (lambda: erc.erc_score_rows(x, ids, k=2**32), lambda: erc.erc_expert_ffn(x, at, w_in, w_out, act=2**32),
                 lambda: erc.erc_dropout(x, 0.5, 1, first=2**62), lambda: erc.erc_dropout(x, 0.5, 1, first=0.5)):
        refused(call)
