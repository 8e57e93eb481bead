"""GPU parity of the row-wise choices (erc_sample_rows, erc_route, erc_expert_*): whole-number results
bit-exact against the oracle, real ones within bounds derived from float32 rounding."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import choice_oracle as C
from paper_2609_27209_gb300 import erc

from ._gpu import dev, host

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0**-24, "bf16": 2.0**-8, "f16": 2.0**-11}  # half a unit of 24, 8, 11 bits
U = 2.0**-24


def f32(t):
    return t.detach().float().cpu().numpy()


def words_of(rng, rows):
    w = rng.integers(-(2**63), 2**63, rows, dtype=np.int64)
    w[: min(2, rows)] = [-1, 0][: min(2, rows)]  # both ends of the words
    return w


def per_row(v, i):
    return v[i].item() if isinstance(v, np.ndarray) else v


def check_sample(logits, words, every=1, **rule):
    """Draws of a device matrix against the oracle, `every`-th row by row."""
    given = {k: torch.from_numpy(v).to(dev()) if isinstance(v, np.ndarray) else v for k, v in rule.items()}
    ids, logp, kept = erc.erc_sample_rows(logits, torch.from_numpy(words).to(dev()), **given)
    assert ids.dtype == torch.int32 and logp.dtype == torch.float32 and kept.dtype == torch.int32
    ids, logp, kept = host(ids), host(logp).astype(np.float64), host(kept)
    x = f32(logits)
    for i in range(0, x.shape[0], every):
        want = C.sample_row(x[i], words[i], **{k: per_row(v, i) for k, v in rule.items()})
        assert (ids[i], kept[i]) == (want[0], len(want[2])), (i, ids[i], kept[i], want[0], len(want[2]))
        if want[0] < 0:
            assert logp[i] == -math.inf
        else:
            # two conversions and a quotient (3 U in the ratio, so in its logarithm) and an ulp or
            # two of the logarithm itself
            assert abs(logp[i] - want[1]) <= 4 * U * (1 + abs(want[1])), (i, logp[i], want[1])


RULES = [dict(), dict(temperature=0.7), dict(top_k=5), dict(top_k=1000), dict(top_p=0.9),
         dict(temperature=1.5, top_p=0.999), dict(min_p=0.05), dict(temperature=0.0),
         dict(temperature=0.8, top_k=50, top_p=0.95), dict(top_k=300, top_p=0.5, min_p=0.001),
         dict(temperature=2.0, top_p=0.3, min_p=0.9), dict(top_p=1e-9), dict(min_p=1.0)]


@pytest.mark.parametrize("n", [0, 1, 2, 31, 33, 257, 1000, 4099])
@pytest.mark.parametrize("rule", RULES, ids=str)
def test_sample_matches_oracle(n, rule):
    rng = np.random.default_rng(n * 100 + len(rule))
    rows = 7
    x = rng.normal(size=(rows, n)).astype(np.float32) * np.linspace(0.2, 4, rows, dtype=np.float32)[:, None]
    x[rng.random((rows, n)) < 0.1] = -np.inf
    x[3] = -np.inf
    for kind in TYPES.values():
        check_sample(torch.from_numpy(x).to(dev()).to(kind), words_of(rng, rows), **rule)


@pytest.mark.parametrize("rule", RULES, ids=str)
@pytest.mark.parametrize("n", [1025, 4099, 16384])
def test_sample_many_rows_of_middling_length(n, rule):
    rng = np.random.default_rng(n)
    rows = 320
    x = rng.normal(size=(rows, n)).astype(np.float32) * np.linspace(0.3, 3, rows, dtype=np.float32)[:, None]
    x[::5] = np.round(x[::5] * 2) / 2  # ties
    x[15::40, n // 3:] = -np.inf
    x[30] = -np.inf
    x[45] = 0.0
    for kind in TYPES.values():
        check_sample(torch.from_numpy(x).to(dev()).to(kind), words_of(rng, rows), every=15, **rule)


@pytest.mark.parametrize("n,rows", [(20000, 3), (70001, 3), (169343, 2), (400003, 2)])
@pytest.mark.parametrize("rule", [dict(), dict(temperature=0.8, top_k=50, top_p=0.95), dict(top_p=0.9),
                                  dict(top_k=5000, top_p=0.97), dict(min_p=0.02), dict(top_k=9000)], ids=str)
def test_sample_long_rows(n, rows, rule):
    rng = np.random.default_rng(n)
    x = rng.normal(size=(rows, n)).astype(np.float32) * np.linspace(0.6, 2.5, rows, dtype=np.float32)[:, None]
    for kind in ("f32", "bf16"):
        check_sample(torch.from_numpy(x).to(dev()).to(TYPES[kind]), words_of(rng, rows), **rule)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n", [60001, 250007])
def test_sample_top_p_that_ends_inside_a_long_flat_tail(kind, n):
    rng = np.random.default_rng(n)
    rows = 4
    x = rng.uniform(-0.3, 0.3, (rows, n)).astype(np.float32)  # a tail of nearly equal weights
    x[np.arange(rows), rng.integers(0, n, rows)] = np.log(n) + np.array([2, 3, 1, 0], np.float32)  # 0.88, 0.95, ..
    for p in (0.9, 0.96, 0.999):
        check_sample(torch.from_numpy(x).to(dev()).to(TYPES[kind]), words_of(rng, rows), top_p=p)
        check_sample(torch.from_numpy(x).to(dev()).to(TYPES[kind]), words_of(rng, rows), top_p=p, min_p=1e-6)


@pytest.mark.parametrize("rule", RULES, ids=str)
@pytest.mark.parametrize("n", [8193, 20011, 300007])
def test_sample_long_bfloat16_rows_of_every_kind(n, rule):
    rng = np.random.default_rng(n)
    x = rng.normal(size=(10, n)).astype(np.float32) * 2
    x[1] = rng.integers(-3, 4, n) * 0.25  # seven values, zeros of both signs
    x[1][x[1] == 0] *= np.where(rng.random((x[1] == 0).sum()) < 0.5, -1, 1)
    x[2] = -np.inf
    x[3] = np.where(rng.random(n) < 0.7, -np.inf, x[3])
    x[3, ::97] = np.nan
    x[4, 5] = 300.0  # magnitudes that a table of codes may not hold
    x[5, ::1001] = 1e-9
    x[6, 77], x[6, 78] = np.inf, -np.inf
    x[7] = x[7] * 1e-3 + 100
    x[8] = -np.abs(x[8]) - 1
    x[9] = np.finfo(np.float32).min / 2
    check_sample(torch.from_numpy(x).to(dev()).to(torch.bfloat16), words_of(rng, 10), **rule)


@pytest.mark.parametrize("top", [3.0, 1.0, 0.0])
@pytest.mark.parametrize("rule", [dict(top_p=0.3), dict(top_p=0.999), dict(top_k=7000), dict(top_k=4000, top_p=0.9), dict(top_p=0.5)], ids=str)
def test_sample_bfloat16_rows_of_zeros_and_tiny_magnitudes(top, rule):
    rng = np.random.default_rng(int(top))
    n = 9001
    x = rng.choice(np.array([0.0, -0.0, 1e-9, -1e-9, 2e-8, -3e-8, 2.0**-24, -(2.0**-24)], np.float32), (6, n))
    x[:, ::300] = top
    x[3, 1::2] = -1.0
    x[4] = np.where(rng.random(n) < 0.5, x[4], 1.0)
    x[5] = rng.choice(np.array([0.0, -0.0], np.float32), n)
    check_sample(torch.from_numpy(x).to(dev()).to(torch.bfloat16), words_of(rng, 6), **rule)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_sample_the_largest_rows(kind):
    n = 1 << 22  # ERC_SAMPLE_ROWS_MAX_N
    rng = np.random.default_rng(5)
    flat = torch.zeros(2, n, dtype=TYPES[kind], device=dev())
    w = words_of(rng, 2)
    ids, logp, kept = erc.erc_sample_rows(flat, torch.from_numpy(w).to(dev()))
    # every weight is 2^40: the draw is floor(x n / 2^64), all n are kept
    assert host(ids).tolist() == [(int(v) & (2**64 - 1)) * n >> 64 for v in w]
    assert host(kept).tolist() == [n, n]
    np.testing.assert_allclose(host(logp), -math.log(n), rtol=4 * U)
    ids, _, kept = erc.erc_sample_rows(flat, torch.from_numpy(w).to(dev()), top_k=100001, top_p=0.5)
    want = math.ceil(100001 * 2**40 // 2 / 2**40)  # target floor(W / 2) over equal weights
    assert host(kept).tolist() == [want, want]
    assert host(ids).tolist() == [(int(v) & (2**64 - 1)) * want >> 64 for v in w]


@pytest.mark.parametrize("rule", [dict(top_k=5), dict(top_p=0.5), dict(top_k=40, top_p=0.7), dict(min_p=0.5)], ids=str)
def test_sample_ties(rule):
    rng = np.random.default_rng(2)
    for n, levels in [(100, 1), (1000, 2), (5000, 3), (9001, 40)]:
        x = rng.integers(0, levels, (5, n)).astype(np.float32) * 0.25
        x[x == 0] *= np.where(rng.random((x == 0).sum()) < 0.5, -1, 1)  # both zeros
        check_sample(torch.from_numpy(x).to(dev()), words_of(rng, 5), **rule)


@pytest.mark.parametrize("high", [127, 128, 129, 255, 256, 257])
@pytest.mark.parametrize("rule", [dict(top_k=100), dict(top_k=60, top_p=0.6), dict(top_k=120, min_p=0.7)], ids=str)
def test_sample_few_candidates_with_ties_among_them(high, rule):
    rng = np.random.default_rng(high)
    for rows, n in [(3, 20001), (200, 5001)]:  # a cluster, and a small block, a row
        x = rng.normal(size=(rows, n)).astype(np.float32) - 20
        for row in x:
            row[rng.choice(n, high, replace=False)] = np.repeat([1.0, 0.75, 0.5], (30, 40, high - 70))
        for kind in TYPES.values():
            check_sample(torch.from_numpy(x).to(dev()).to(kind), words_of(rng, rows), every=max(1, rows // 8), **rule)


def test_sample_infinities_nan_and_lowest_values():
    low = float(np.finfo(np.float32).min)
    x = np.array([[np.nan] * 5, [np.inf, 1, np.inf, np.nan, -np.inf], [low] * 5, [low, low, 3, -np.inf, 2],
                  [np.nan, -np.inf, -np.inf, 7, -np.inf], [-np.inf] * 5, [3e38, -3e38, low, 3e38, 0]], np.float32)
    rng = np.random.default_rng(4)
    for rule in RULES:
        check_sample(torch.from_numpy(x).to(dev()), words_of(rng, 7), **rule)
    for kind in ("bf16", "f16"):
        lowest = torch.finfo(TYPES[kind]).min
        y = torch.full((3, 50), lowest, dtype=TYPES[kind], device=dev())
        y[1, 7] = 1.0
        check_sample(y, words_of(rng, 3))
        check_sample(y, words_of(rng, 3), top_p=0.5)


def test_sample_settings_of_each_row_and_out_of_range_ones():
    rng = np.random.default_rng(8)
    rows, n = 64, 3001
    x = rng.normal(size=(rows, n), scale=2).astype(np.float32)
    pick = lambda v, t: rng.choice(np.array(v, t), rows)  # noqa: E731
    rule = dict(temperature=pick([0, -1, np.nan, 1e-30, 0.5, 1, 1.4, 3e38, np.inf], np.float32),
                top_k=pick([-3, 0, 1, 2, 40, 2999, 5000, 2**31 - 1], np.int32),
                top_p=pick([-1, 0, 0.1, 0.9, 1, 2, np.nan], np.float32),
                min_p=pick([-1, 0, 0.01, 1, 5, np.nan], np.float32))
    check_sample(torch.from_numpy(x).to(dev()), words_of(rng, rows), **rule)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_sample_strides_and_alignment(kind):
    rng = np.random.default_rng(6)
    base = torch.from_numpy(rng.normal(size=40 * 1100).astype(np.float32)).to(dev()).to(TYPES[kind])
    for n, stride, start in [(1000, 1003, 1), (999, 1024, 3), (17, 20, 5), (1, 7, 2), (1000, 0, 3), (64, 13, 0)]:
        x = base.as_strided((9, n), (stride, 1), start)
        check_sample(x, words_of(rng, 9), top_k=20)
        check_sample(x, words_of(rng, 9), temperature=0.9)


def test_sample_offsets_past_32_bits():
    n, stride = 300, (1 << 31) + 11
    buffer = torch.empty(2 * stride, dtype=torch.bfloat16, device=dev())
    x = buffer.as_strided((2, n), (stride, 1), 5)
    rng = np.random.default_rng(9)
    x.copy_(torch.from_numpy(rng.normal(size=(2, n)).astype(np.float32)))
    check_sample(x, words_of(rng, 2), top_p=0.8)


def test_sample_on_another_stream_and_twice():
    rng = np.random.default_rng(10)
    x = torch.from_numpy(rng.normal(size=(50, 30011)).astype(np.float32)).to(dev())
    w = torch.from_numpy(words_of(rng, 50)).to(dev())
    a = erc.erc_sample_rows(x, w, top_p=0.9)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = erc.erc_sample_rows(x * 1, w, top_p=0.9)
    s.synchronize()
    for u, v in zip(a, b):
        assert torch.equal(u, v)


def test_sample_more_rows_than_a_grid():
    rng = np.random.default_rng(13)
    n, rows = 2100, 70001
    base = torch.from_numpy(rng.normal(size=n + rows).astype(np.float32)).to(dev()).to(torch.bfloat16)
    x = base.as_strided((rows, n), (1, 1))  # row i starts at entry i
    check_sample(x, words_of(rng, rows), every=7777, top_p=0.9)


def test_sample_draws_follow_the_probabilities():
    x = np.array([0.0, 1.0, 2.0, -1.0], np.float32)
    rows = 1 << 16
    words = torch.from_numpy(np.random.default_rng(12).integers(-(2**63), 2**63, rows, dtype=np.int64)).to(dev())
    ids, _, _ = erc.erc_sample_rows(torch.from_numpy(x).to(dev()).expand(rows, 4), words)
    freq = np.bincount(host(ids), minlength=4) / rows
    q = C.sample_probs(x, 1.0, np.arange(4))
    assert np.all(np.abs(freq - q) < 6 * np.sqrt(q * (1 - q) / rows))  # six standard deviations


def refused(call):
    with pytest.raises(erc.ErcError) as e:
        call()
    assert e.value.status == erc.ERC_ERR_INVALID_ARG


def test_sample_refusals():
    x = torch.zeros(2, 5, device=dev())
    w = torch.zeros(2, dtype=torch.int64, device=dev())
    for bad in (dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf), dict(top_k=-1),
                dict(top_p=0.0), dict(top_p=1.5), dict(top_p=math.nan), dict(min_p=-0.1), dict(min_p=1.1),
                dict(temperature=torch.ones(3, device=dev())), dict(top_k=torch.ones(2, device=dev())),
                dict(top_p=torch.ones(2))):
        refused(lambda: erc.erc_sample_rows(x, w, **bad))
    refused(lambda: erc.erc_sample_rows(x.double(), w))
    refused(lambda: erc.erc_sample_rows(x.cpu(), w))
    refused(lambda: erc.erc_sample_rows(x[0], w))
    refused(lambda: erc.erc_sample_rows(torch.zeros(5, 2, device=dev()).t(), w))
    refused(lambda: erc.erc_sample_rows(x, w[:1]))
    refused(lambda: erc.erc_sample_rows(x, w.int()))
    refused(lambda: erc.erc_sample_rows(torch.zeros(1, (1 << 22) + 1, device=dev()), w[:1]))
    ids, logp, kept = erc.erc_sample_rows(x[:0], w[:0])
    assert ids.numel() == logp.numel() == kept.numel() == 0


# ------------------------------------------------------------------------------------------------ routing


def check_route(logits, k, **rule):
    given = dict(rule)
    if rule.get("bias") is not None:
        given["bias"] = torch.from_numpy(rule["bias"]).to(dev())
    kind = given.pop("kind")
    given["score"] = erc.ERC_SCORE_SOFTMAX if kind == "softmax" else erc.ERC_SCORE_SIGMOID
    experts, weights = erc.erc_route(logits, k, **given)
    assert experts.dtype == torch.int32 and weights.dtype == torch.float32
    e, w = C.route(f32(logits), k, **rule)
    np.testing.assert_array_equal(host(experts), e)
    # the scores have the oracle's bits; a sum of k of them, a quotient and a product are rounded
    np.testing.assert_allclose(host(weights), w, rtol=(k + 3) * U, atol=1e-44)
    return experts, weights


@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (7, 3), (32, 8), (33, 33 - 1), (64, 2), (100, 32), (256, 8), (1000, 6), (1024, 9)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_route_matches_oracle(E, k, kind):
    rng = np.random.default_rng(E * 7 + k)
    x = rng.normal(size=(37, E), scale=2).astype(np.float32)
    x[rng.random(x.shape) < 0.05] = -np.inf
    x[5] = -np.inf
    x[6, 1:] = np.nan
    bias = rng.normal(size=E, scale=0.2).astype(np.float32)
    for t in TYPES.values():
        for b in (None, bias):
            check_route(torch.from_numpy(x).to(dev()).to(t), k, kind=kind, bias=b, renorm=b is None, scale=2.5)


@pytest.mark.parametrize("E,groups,top,k", [(8, 4, 1, 2), (8, 8, 3, 3), (60, 4, 2, 6), (256, 8, 4, 8), (256, 32, 5, 8),
                                            (1024, 2, 1, 32), (96, 3, 3, 4), (1024, 1024, 40, 32), (35, 5, 2, 14)])
@pytest.mark.parametrize("best", [1, 2])
def test_route_groups(E, groups, top, k, best):
    rng = np.random.default_rng(E + groups)
    x = rng.normal(size=(29, E)).astype(np.float32)
    x[3, : E // 2] = -np.inf  # whole groups masked: fewer than k may be left
    x[4] = -np.inf
    x[4, -1] = 0.5
    bias = rng.normal(size=E, scale=0.1).astype(np.float32)
    for kind in ("softmax", "sigmoid"):
        check_route(torch.from_numpy(x).to(dev()), k, kind=kind, bias=bias, groups=groups, top_groups=top,
                    group_best=best)


def test_route_ties_infinities_and_extremes():
    low = float(np.finfo(np.float32).min)
    x = np.array([[1, 1, 1, 1, 1, 1], [0.0, -0.0, 0.0, -0.0, 0, 0], [np.inf, 0, np.inf, 1, 2, np.nan],
                  [low, low, low, 0, low, low], [3e38, 3e38, -3e38, 0, 1, 2], [-200, -201, -1e30, -np.inf, -300, -200]], np.float32)
    for kind in ("softmax", "sigmoid"):
        for bias in (None, np.array([0, 0.5, 0, np.inf, np.nan, -np.inf], np.float32)):
            for renorm in (True, False):
                check_route(torch.from_numpy(x).to(dev()), 5, kind=kind, bias=bias, renorm=renorm)
                check_route(torch.from_numpy(x).to(dev()), 3, kind=kind, bias=bias, renorm=renorm, groups=3, top_groups=2)


@pytest.mark.parametrize("rows", [0, 1, 2, 5, 1000])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_route_rows_strides_and_both_directions(rows, kind):
    rng = np.random.default_rng(rows)
    for t, half in ((torch.float32, 0.0), (torch.bfloat16, 2.0**-8), (torch.float16, 2.0**-11)):
        for E, stride, start, k in [(64, 64, 0, 4), (60, 67, 1, 7), (9, 9, 3, 1), (130, 0, 1, 2)]:
            base = torch.from_numpy(rng.normal(size=rows * max(stride, 1) + E + 8, scale=2).astype(np.float32)).to(dev()).to(t)
            x = base.as_strided((rows, E), (stride, 1), start)
            for renorm in (True, False):
                experts, _ = check_route(x, k, kind=kind, renorm=renorm, scale=1.5)
                g = rng.normal(size=(rows, k)).astype(np.float32)
                score = erc.ERC_SCORE_SOFTMAX if kind == "softmax" else erc.ERC_SCORE_SIGMOID
                got = erc.erc_route_backward(x, experts, torch.from_numpy(g).to(dev()), score=score, renorm=renorm, scale=1.5)
                assert got.dtype == t and got.shape == x.shape
                check_gradient(got, f32(x), host(experts), g, kind, renorm, 1.5, half)


def check_gradient(got, x, e, g, kind, renorm, scale, half):
    if not x.size:
        return
    want = C.route_gradient(x, e, g, kind, renorm, scale)
    s = C.scores64(x, kind)
    v = np.where(e >= 0, np.take_along_axis(s, np.maximum(e, 0), 1), 0.0)
    d = v.sum(1, keepdims=True) if renorm else np.ones((len(x), 1))
    # a score is off by at most delta of itself (|t| <= 40 moved by 2.5 U |t| ln 2, the rest 5 U), and
    # each of the handful of factors built from them; k terms are summed
    delta = 40 * 2.5 * U + 5 * U
    size = scale * np.abs(g).sum(1, keepdims=True) * 2 / np.where(d > 0, d, 1)
    bound = s * size * (5 * delta + (e.shape[1] + 8) * U) + half * np.abs(want) * 1.01 + 2.0**-25 * (half > 0)
    assert np.all(np.abs(f32(got) - want) <= bound + 1e-30)


@pytest.mark.parametrize("E,k", [(1, 1), (3, 2), (33, 5), (256, 8), (1024, 32)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_route_backward_with_empty_choices(E, k, kind):
    rng = np.random.default_rng(E)
    x = rng.normal(size=(21, E)).astype(np.float32)
    x[2] = -np.inf
    x[3, 0] = np.nan
    e, _ = C.route(x, k, kind)
    e[rng.random(e.shape) < 0.3] = -1
    e[4] = -1
    g = rng.normal(size=e.shape).astype(np.float32)
    score = erc.ERC_SCORE_SOFTMAX if kind == "softmax" else erc.ERC_SCORE_SIGMOID
    for renorm in (True, False):
        got = erc.erc_route_backward(torch.from_numpy(x).to(dev()), torch.from_numpy(e.astype(np.int32)).to(dev()),
                                     torch.from_numpy(g).to(dev()), score=score, renorm=renorm, scale=0.5)
        check_gradient(got, x, e, g, kind, renorm, 0.5, 0.0)
        assert not f32(got)[4].any() and not f32(got)[2].any()


def test_route_gradient_against_differences_of_the_kernel():
    rng = np.random.default_rng(31)
    x = rng.normal(size=(6, 12)).astype(np.float32)
    g = torch.from_numpy(rng.normal(size=(6, 3)).astype(np.float32)).to(dev())
    h = 2.0**-6
    for score in (erc.ERC_SCORE_SOFTMAX, erc.ERC_SCORE_SIGMOID):
        xd = torch.from_numpy(x).to(dev())
        e, _ = erc.erc_route(xd, 3, score=score)
        got = f32(erc.erc_route_backward(xd, e, g, score=score))
        for i in range(12):
            side = []
            for sign in (1, -1):
                y = x.copy()
                y[:, i] += sign * h
                es, ws = erc.erc_route(torch.from_numpy(y).to(dev()), 3, score=score)
                side.append((host(es), f32(ws)))
            same = (side[0][0] == host(e)).all(1) & (side[1][0] == host(e)).all(1)  # choices unchanged
            d = ((side[0][1] - side[1][1]) * f32(g)).sum(1) / (2 * h)
            # rounding 2 U sum|g| / (2 h) < 1e-4, and h^2/6 times a third derivative of order sum|g|
            assert np.all(np.abs(d - got[:, i])[same] < 1e-3)


def test_route_offsets_past_32_bits():
    stride = (1 << 31) + 3
    buffer = torch.empty(stride + 64, dtype=torch.bfloat16, device=dev())
    x = buffer.as_strided((2, 40), (stride, 1), 1)
    rng = np.random.default_rng(1)
    x.copy_(torch.from_numpy(rng.normal(size=(2, 40)).astype(np.float32)))
    check_route(x, 4, kind="softmax")


def test_route_refusals():
    x = torch.zeros(3, 8, device=dev())
    for bad in (dict(k=0), dict(k=9), dict(k=33), dict(score=2), dict(groups=3), dict(groups=0), dict(groups=2, top_groups=3),
                dict(groups=2, top_groups=0), dict(group_best=3), dict(scale=math.inf), dict(scale=math.nan),
                dict(bias=torch.zeros(7, device=dev())), dict(bias=torch.zeros(8))):
        refused(lambda: erc.erc_route(x, **{"k": 2, **bad}))
    refused(lambda: erc.erc_route(torch.zeros(2, 1025, device=dev()), 2))
    refused(lambda: erc.erc_route(torch.zeros(2, 0, device=dev()), 1))
    refused(lambda: erc.erc_route(x.long(), 2))
    refused(lambda: erc.erc_route(x.t(), 2))
    e = torch.zeros(3, 2, dtype=torch.int32, device=dev())
    g = torch.zeros(3, 2, device=dev())
    refused(lambda: erc.erc_route_backward(x, e.long(), g))
    refused(lambda: erc.erc_route_backward(x, e, g[:2]))
    refused(lambda: erc.erc_route_backward(x, e, g.double()))


# ------------------------------------------------------------------------------------------------ experts


@pytest.mark.parametrize("rows,k", [(0, 2), (1, 1), (3, 2), (130, 4), (1023, 1), (5000, 3), (700, 32)])
@pytest.mark.parametrize("E", [1, 5, 64, 256, 1024])
def test_plan_matches_oracle(rows, k, E):
    rng = np.random.default_rng(rows * 31 + E)
    for kind in ("even", "one", "gaps"):
        e = rng.integers(0, E, (rows, k))
        if kind == "one":
            e[:] = E // 2
        if kind == "gaps":
            e = np.where(rng.random((rows, k)) < 0.5, rng.choice([-1, -(2**31), E, 2**31 - 1], (rows, k)), e // 2)
        offsets, order, slot = erc.erc_expert_plan(torch.from_numpy(e.astype(np.int32)).to(dev()), E)
        o, r, s = C.plan(e, E)
        np.testing.assert_array_equal(host(offsets), o)
        np.testing.assert_array_equal(host(order), r)
        np.testing.assert_array_equal(host(slot), s)


def test_plan_of_a_large_step():
    rng = np.random.default_rng(3)
    rows, k, E = 169343, 8, 200
    e = rng.integers(-1, E, (rows, k)).astype(np.int32)
    offsets, order, slot = (host(t) for t in erc.erc_expert_plan(torch.from_numpy(e).to(dev()), E))
    flat = np.where(e.reshape(-1) < 0, E, e.reshape(-1))
    want = np.argsort(flat, kind="stable")
    placed = int((flat < E).sum())
    np.testing.assert_array_equal(offsets, np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E + 1)[:E])]))
    np.testing.assert_array_equal(order[:placed], want[:placed])
    assert (order[placed:] == -1).all()
    back = np.full(flat.size, -1)
    back[want[:placed]] = np.arange(placed)
    np.testing.assert_array_equal(slot.reshape(-1), back)


@pytest.mark.parametrize("width", [0, 1, 3, 8, 33, 64, 520, 1030, 4096])
@pytest.mark.parametrize("k", [1, 2, 8, 32])
@pytest.mark.parametrize("kind", list(TYPES))
def test_gather_combine_and_gradient_match_oracle(width, k, kind):
    rng = np.random.default_rng(width * 3 + k)
    t, half = TYPES[kind], HALF_ULP[kind]
    for rows in (1, 41):
        e = rng.integers(0, 40, (rows, k))
        e[rng.random(e.shape) < 0.2] = -1
        _, _, s = C.plan(e, 40)
        offsets, _, slot = erc.erc_expert_plan(torch.from_numpy(e.astype(np.int32)).to(dev()), 40)
        make = lambda n: torch.from_numpy(rng.normal(size=(n, width)).astype(np.float32)).to(dev()).to(t)  # noqa: E731
        x, y, dout = make(rows), make(rows * k), make(rows)
        w = rng.normal(size=(rows, k)).astype(np.float32)
        wd = torch.from_numpy(w).to(dev())
        xs = erc.erc_expert_gather(x, slot, offsets)
        want = np.zeros((rows * k, width))
        for i, j in np.argwhere(s >= 0):
            want[s[i, j]] = f32(x)[i]
        np.testing.assert_array_equal(f32(xs), want)
        for weights in (w, None):
            out = erc.erc_expert_combine(y, slot, None if weights is None else wd)
            assert out.dtype == t
            ww = np.where(s >= 0, np.ones_like(w) if weights is None else w, 0)
            size = C.combine(np.abs(f32(y)), s, np.abs(ww))
            want = C.combine(f32(y), s, weights)
            # k products and k sums in float32, then one rounding to the type
            assert np.all(np.abs(f32(out) - want) <= (k + 1) * U * size + half * np.abs(want) * 1.01 + 2.0**-25 * (kind == "f16"))
        dy, dw = erc.erc_expert_combine_backward(dout, y, slot, offsets, wd)
        want_y, want_w = C.combine_gradient(f32(dout), f32(y), s, w)
        assert np.all(np.abs(f32(dy) - want_y) <= (U + half) * np.abs(want_y) * 1.01 + 2.0**-25 * (kind == "f16"))
        size = np.where(s >= 0, (np.abs(f32(dout))[:, None] * np.abs(f32(y))[np.maximum(s, 0)]).sum(2), 0)
        assert np.all(np.abs(f32(dw) - want_w) <= (width + 1) * U * size)


def test_gather_and_combine_are_adjoint():
    rng = np.random.default_rng(17)
    rows, k, width = 300, 4, 96
    e = torch.from_numpy(rng.integers(-1, 16, (rows, k)).astype(np.int32)).to(dev())
    offsets, _, slot = erc.erc_expert_plan(e, 16)
    x = torch.randn(rows, width, device=dev())
    y = torch.randn(rows * k, width, device=dev())
    a = (erc.erc_expert_gather(x, slot, offsets).double() * y.double()).sum().item()
    out = erc.erc_expert_combine(y, slot)
    b = (x.double() * out.double()).sum().item()
    size = (x.double().abs() * erc.erc_expert_combine(y.abs(), slot).double()).sum().item()
    assert abs(a - b) <= (k + 1) * U * size


def test_experts_ignore_slots_out_of_range():
    x = torch.ones(4, 8, device=dev())
    slot = torch.tensor([[0], [99], [-5], [2]], dtype=torch.int32, device=dev())
    offsets = torch.tensor([0, 3], dtype=torch.int64, device=dev())
    xs = erc.erc_expert_gather(x, slot, offsets)
    assert f32(xs)[[0, 2]].all() and not f32(xs)[3].any()
    y = torch.arange(32.0, device=dev()).view(4, 8)
    out = erc.erc_expert_combine(y, slot)
    assert torch.equal(out[0], y[0]) and torch.equal(out[3], y[2]) and not out[1].any() and not out[2].any()


def test_expert_refusals():
    e = torch.zeros(4, 2, dtype=torch.int32, device=dev())
    offsets, order, slot = erc.erc_expert_plan(e, 3)
    x, y, w = torch.zeros(4, 8, device=dev()), torch.zeros(8, 8, device=dev()), torch.zeros(4, 2, device=dev())
    refused(lambda: erc.erc_expert_plan(e.long(), 3))
    refused(lambda: erc.erc_expert_plan(e, 0))
    refused(lambda: erc.erc_expert_plan(e, 1025))
    refused(lambda: erc.erc_expert_plan(torch.zeros(4, 33, dtype=torch.int32, device=dev()), 3))
    refused(lambda: erc.erc_expert_plan(e.t(), 3))
    refused(lambda: erc.erc_expert_gather(x[:3], slot, offsets))
    refused(lambda: erc.erc_expert_gather(x.t(), slot, offsets))
    refused(lambda: erc.erc_expert_gather(x, slot, offsets.int()))
    refused(lambda: erc.erc_expert_combine(y[:7], slot))
    refused(lambda: erc.erc_expert_combine(y, slot, w.half()))
    refused(lambda: erc.erc_expert_combine(y.double(), slot))
    refused(lambda: erc.erc_expert_combine_backward(x, y.half(), slot, offsets, w))
    refused(lambda: erc.erc_expert_combine_backward(x, y, slot, offsets, w[:3]))
    with pytest.raises(erc.ErcError) as err:
        erc.erc_expert_plan(torch.zeros(4000, 2, dtype=torch.int32, device=dev()), 300,
                            ws=torch.empty(8, dtype=torch.uint8, device=dev()))
    assert err.value.status == erc.ERC_ERR_CAPACITY


def test_struct_layouts_of_the_rules():
    # natural alignment of 4-byte fields, then 8-byte pointers
    assert ctypes.sizeof(erc.ErcSampleRuleC) == 48 and erc.ErcSampleRuleC.temperature_rows.offset == 16
    assert ctypes.sizeof(erc.ErcRouteRuleC) == 32 and erc.ErcRouteRuleC.scale.offset == 28
