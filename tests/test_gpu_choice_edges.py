"""The row-wise choices at the ends of their ranges: scores below 2^-126, sums that cancel or overflow,
calls from several threads, and arguments that do not fit."""
import ctypes
import threading

import numpy as np
import pytest
import torch

from oracle import choice_oracle as C
from paper_2609_27209_gb300 import erc

from ._gpu import dev, host
from .test_gpu_choice import TYPES, U, check_route, check_sample, f32, refused, words_of

pytestmark = pytest.mark.gpu

# a row in 8 and in 16 lanes, in shared memory (groups of 15), and in a warp with 8, 16 and 32 experts a lane
KERNELS = [(8, 1), (64, 1), (128, 1), (60, 4), (256, 1), (512, 1), (1024, 1)]


@pytest.mark.parametrize("E,groups", KERNELS)
@pytest.mark.parametrize("renorm", [True, False])
def test_sigmoid_scores_around_the_smallest_normal_float(E, groups, renorm):
    # e = 2^(-|l| log2(e)) is kept down to rint(t) = -126, where it is subnormal for t < -126: |l| of
    # 87.34 to 87.68.  More than 32 candidates of a warp's row look alike to its approximate scores.
    rng = np.random.default_rng(E)
    x = rng.uniform(-87.75, -87.25, (40, E)).astype(np.float32)
    x[0] = -87.5
    x[1] = np.resize(np.float32([-87.375, -87.5, -87.625]), E)
    for t in TYPES.values():
        check_route(torch.from_numpy(x).to(dev()).to(t), min(8, E), kind="sigmoid", groups=groups,
                    top_groups=max(1, groups // 2), renorm=renorm)


def just_below(points):
    """float32 logits whose float32 sigmoids are the largest below `points` that 65 neighbours hold."""
    l = np.log(points / (1 - points)).astype(np.float32)[:, None]
    near = (l.view(np.int32) + np.arange(-32, 33, dtype=np.int32)).view(np.float32)
    s, _ = C.route_scores(near, "sigmoid")
    s = np.where(s.astype(np.float64) < points[:, None], s, -1)
    best = s.argmax(1)[:, None]
    return np.take_along_axis(near, best, 1)[:, 0], np.take_along_axis(s, best, 1)[:, 0].astype(np.float64)


@pytest.mark.parametrize("E,big", [(256, 512.0), (256, 1024.0), (512, 1024.0), (1024, 65536.0)])
def test_groups_whose_two_best_cancel(E, big):
    # One expert of a group has the bias `big`, the others -big: the choices are rounded to steps of
    # ulp(big), a group's score is near 1.  The last group's best score lies just below the middle of
    # such a step, the first group's well inside it: they tie, so the first is taken.
    rows, size = 4096, 32
    step = np.spacing(np.float32(big)).astype(np.float64)
    j = np.floor(np.linspace(0.5, 0.9, rows) / step)
    x = np.full((rows, E), -np.inf, np.float32)
    x[:, :size] = x[:, -size:] = -1.0
    x[:, 0], low = just_below((j + 0.25) * step)
    x[:, E - size], high = just_below((j + 0.5) * step)
    keep = (low > 0) & (high > 0) & ((j + 0.5) * step < 0.95)
    x = x[keep]
    assert len(x) > 4
    bias = np.full(E, -big, np.float32)
    bias[::size] = big
    experts, _ = check_route(torch.from_numpy(x).to(dev()), 2, kind="sigmoid", bias=bias, groups=E // size,
                             top_groups=1)
    assert (host(experts) == [0, 1]).all()


@pytest.mark.parametrize("E", [64, 128, 60, 256, 1024])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_groups_whose_sum_overflows_are_not_empty_groups(E, kind):
    x = np.random.default_rng(E).normal(size=(9, E)).astype(np.float32)
    x[:, : E // 4] = -np.inf  # a group with nothing to choose comes first, groups of -inf = -3e38 - 3e38 follow
    x[4, : 3 * E // 4] = -np.inf
    bias = np.full(E, -3e38, np.float32)
    for top in (1, 2, 3):
        with np.errstate(over="ignore"):  # the oracle's sums
            experts, _ = check_route(torch.from_numpy(x).to(dev()), 3, kind=kind, bias=bias, groups=4, top_groups=top)
        assert (host(experts) >= E // 4).all()


@pytest.mark.parametrize("E", [2, 64, 128, 200, 1024])
def test_sigmoid_gradient_where_the_chosen_scores_are_tiny(E):
    # (g - mean) / D alone overflows for D below 1e-35; times s it is an ordinary number
    rng = np.random.default_rng(E)
    k = min(4, E)
    x = rng.uniform(-87.2, -84, (20, E)).astype(np.float32)
    e, _ = C.route(x, k, "sigmoid")
    for size in (1.0, 1e3, 1e6):
        g = (rng.normal(size=e.shape) * size).astype(np.float32)
        got = erc.erc_route_backward(torch.from_numpy(x).to(dev()), torch.from_numpy(e.astype(np.int32)).to(dev()),
                                     torch.from_numpy(g).to(dev()), score=erc.ERC_SCORE_SIGMOID)
        assert np.isfinite(f32(got)).all()
        s = C.scores64(x, "sigmoid")
        v = np.take_along_axis(s, e, 1)
        want = C.route_gradient(x, e, g, "sigmoid", True, 1.0)
        # scores within delta of themselves (|t| <= 126 moved by 2.5 U |t| ln 2, the rest 5 U, and half of
        # 2^-149 against at least 2^-126), in five factors; k terms are summed
        delta = 126 * 2.5 * U * np.log(2) + 5 * U + 2.0**-24
        bound = s / v.sum(1, keepdims=True) * 2 * np.abs(g).sum(1, keepdims=True) * (5 * delta + (k + 8) * U)
        assert np.all(np.abs(f32(got) - want) <= bound)


@pytest.mark.parametrize("E,groups", KERNELS)
def test_softmax_orders_experts_far_below_the_best(E, groups):
    # the scores of whole-number logits within 80 of the best are distinct normal floats: the order of the
    # experts is the order of the logits, and nothing of them is lost
    rng = np.random.default_rng(E)
    x = np.stack([rng.permutation(np.resize(-rng.permutation(81), E)) for _ in range(30)]).astype(np.float32)
    x[:, 0] = 0
    x[0, 1:8] = [-40, -30, -50, -35, -60, -45, -70]
    x[0, 8:] = -np.inf
    k = min(6, E)
    for renorm in (True, False):
        experts, weights = erc.erc_route(torch.from_numpy(x).to(dev()), k, groups=groups, top_groups=groups, renorm=renorm)
        want = np.argsort(-x, 1, kind="stable")[:, :k]
        np.testing.assert_array_equal(host(experts), want)
        w = C.weights64(x, want, "softmax", renorm, 1.0)
        # |t| <= 116 moved by 2.5 U |t| ln 2; the polynomial, the sum, its reciprocal, a product and a quotient
        np.testing.assert_allclose(host(weights), w, rtol=116 * 2.5 * U * np.log(2) + (k + 12) * U, atol=0)


@pytest.mark.parametrize("E", [8, 64, 128, 200, 1024])
@pytest.mark.parametrize("renorm", [True, False])
def test_softmax_gradient_of_experts_far_below_the_best(E, renorm):
    # experts that a bias chose: their scores are down to e^-86 of the best one's
    rng = np.random.default_rng(E)
    k = min(4, E - 1)
    x = rng.uniform(-86, -60, (20, E)).astype(np.float32)
    x[:, -1] = 0
    x[::2, :k] = rng.uniform(-86, -85, (10, k))
    e = np.tile(np.arange(k), (20, 1))
    g = (rng.normal(size=e.shape) * 1e4).astype(np.float32)
    got = f32(erc.erc_route_backward(torch.from_numpy(x).to(dev()), torch.from_numpy(e.astype(np.int32)).to(dev()),
                                     torch.from_numpy(g).to(dev()), renorm=renorm))
    s = C.scores64(x, "softmax")
    want = C.route_gradient(x, e, g, "softmax", renorm, 1.0)
    d = np.take_along_axis(s, e, 1).sum(1, keepdims=True) if renorm else 1.0
    delta = 126 * 2.5 * U * np.log(2) + 5 * U
    bound = s / d * 2 * np.abs(g).sum(1, keepdims=True) * (5 * delta + (k + 8) * U)
    # renormalised weights do not depend on the other logits at all; results below 2^-126 may be rounded to 0
    assert np.all(np.abs(got - want) <= bound + 2.0**-126)


@pytest.mark.parametrize("rows,n", [(3, 4100), (200, 4100), (400, 1500), (2, 70001)])
@pytest.mark.parametrize("kind", list(TYPES))
def test_top_p_counts_what_a_small_min_p_keeps(rows, n, kind):
    # One entry of weight 1, 2000 (or half the row) of 2^-12, the rest far lighter, each below an eighth of
    # (1 - top_p) / n but well above min_p: together they move top_p's target by tens of the second kind.
    rng = np.random.default_rng(n)
    p = 0.8
    light = np.log2((1 - p) / n) - 3.6
    x = np.full((rows, n), light * np.log(2), np.float32)
    for row in x:
        at = rng.permutation(n)
        row[at[: min(2000, n // 2)]] = -12 * np.log(2)
        row[at[0]] = 0
    check_sample(torch.from_numpy(x).to(dev()).to(TYPES[kind]), words_of(rng, rows), every=max(1, rows // 4),
                 top_p=p, min_p=1e-9)


def test_calls_from_several_threads():
    # Rows of 1249 entries and more need more shared memory for top-p than a kernel has without asking.
    # The library's calls alone, without the binding's work around them, meet most often.
    rng = np.random.default_rng(3)
    rows, jobs, errors = 320, [], []
    rule = erc.ErcSampleRuleC(1.0, 0, 0.9, 0.0)
    for n in (1536, 1300, 1249, 1400):
        x = torch.from_numpy(rng.normal(size=(rows, n)).astype(np.float32)).to(dev())
        w = torch.from_numpy(words_of(rng, rows)).to(dev())
        jobs.append((x, w, erc.erc_sample_rows(x, w, top_p=0.9), torch.cuda.Stream()))
    torch.cuda.synchronize()
    call = erc.lib().erc_sample_rows

    def work(x, w, want, stream):
        got = [torch.empty_like(t) for t in want]
        torch.cuda.synchronize()
        args = (rows, x.shape[1], x.data_ptr(), erc.ERC_F32, x.shape[1], w.data_ptr(), ctypes.byref(rule),
                *(t.data_ptr() for t in got), stream.cuda_stream)
        failed = sum(call(*args) != erc.ERC_OK for _ in range(5000))
        stream.synchronize()
        if failed or not all(torch.equal(a, b) for a, b in zip(got, want)):
            errors.append(failed)

    threads = [threading.Thread(target=work, args=job) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors


def every_call():
    """Each operator with arguments that fit: (its name, the call)."""
    x, w = torch.zeros(4, 8, device=dev()), torch.zeros(4, dtype=torch.int64, device=dev())
    experts, weights = erc.erc_route(x, 2)
    offsets, _, slot = erc.erc_expert_plan(experts, 8)
    y = torch.zeros(8, 8, device=dev())
    return [("sample_rows", lambda: erc.erc_sample_rows(x, w)),
            ("route", lambda: erc.erc_route(x, 2)),
            ("route_backward", lambda: erc.erc_route_backward(x, experts, weights)),
            ("plan", lambda: erc.erc_expert_plan(experts, 8)),
            ("gather", lambda: erc.erc_expert_gather(x, slot, offsets)),
            ("combine", lambda: erc.erc_expert_combine(y, slot)),
            ("combine_backward", lambda: erc.erc_expert_combine_backward(x, y, slot, offsets, weights))]


def test_tensors_of_a_device_that_is_not_current_are_refused(monkeypatch):
    calls = every_call()
    for _, call in calls:
        call()
    torch.cuda.synchronize()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for _, call in calls:
        refused(call)


def test_plan_workspaces_that_do_not_fit_are_refused():
    e = torch.zeros(4, 2, dtype=torch.int32, device=dev())  # so few pairs need no workspace: none is touched
    erc.erc_expert_plan(e, 3, ws=torch.empty(64, dtype=torch.uint8, device=dev()))
    for ws in (torch.empty(64, dtype=torch.uint8), torch.empty(64, device=dev()),
               torch.empty(64, dtype=torch.uint8, device=dev())[::2], 64):
        refused(lambda: erc.erc_expert_plan(e, 3, ws=ws))


def test_whole_numbers_that_do_not_fit_are_refused():
    x, w = torch.zeros(4, 8, device=dev()), torch.zeros(4, dtype=torch.int64, device=dev())
    for top_k in (-1, -(2**31), -(2**32), -(2**32) + 5, 0.5, float("nan")):
        refused(lambda: erc.erc_sample_rows(x, w, top_k=top_k))
    assert host(erc.erc_sample_rows(x, w, top_k=2**40)[2]).tolist() == [8] * 4  # more than there are: all
    assert host(erc.erc_sample_rows(x, w, top_k=3.0)[2]).tolist() == [3] * 4
    for bad in (dict(score=2**32), dict(groups=2**32 + 1), dict(groups=2, top_groups=2**32 + 1),
                dict(group_best=2**32 + 1), dict(groups=1.5)):
        refused(lambda: erc.erc_route(x, 2, **bad))
    refused(lambda: erc.erc_route(x[:0], 2**32 + 2))
    experts, weights = erc.erc_route(x, 2)
    refused(lambda: erc.erc_route_backward(x, experts, weights, score=2**32 + 1))
