"""GPU parity of erc_score_rows and its gradient: indices exact, real results within bounds derived from
float32 rounding."""
import math

import numpy as np
import pytest
import torch

from oracle import expert_oracle as X
from paper_2609_27209_gb300 import erc

from ._gpu import dev, host

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0**-24


def half_ulp(t):
    return torch.finfo(t).eps / 2


def f32(t):
    return t.detach().float().cpu().numpy()


# A sum Z of float32 terms: a thread adds at most 256 segments / 8 warps x 32 vectors x 8 / 32 lanes < 600 terms one by
# one, and some 30 joins follow; the exponential (2^-22) and the scalings of a changed maximum add a few U each.
SUM = 640 * U


def spread(l, temperature):
    """E |t| of a row: an error of |t| 3U in t moves Z by 3U E|t|."""
    l = l[l > -np.inf]
    if not l.size or l.max() == np.inf:
        return 0.0
    t = (l.max() - l) / temperature
    return float((np.exp(-t) * t).sum() / np.exp(-t).sum())


def check(logits, ids, temperature=1.0, k=0, every=1):
    """Forward and gradient of a device matrix against the oracle, every `every`-th row."""
    rows, n = logits.shape
    logp, entropy, norm, top_ids, top_logp = erc.erc_score_rows(logits, torch.from_numpy(ids).to(dev()), temperature, k)
    if k:
        assert top_ids.shape == top_logp.shape == (rows, k) and top_ids.dtype == torch.int32
    else:
        assert top_ids is None and top_logp is None
        top_ids, top_logp = torch.empty(rows, 0, dtype=torch.int32), torch.empty(rows, 0)
    rng = np.random.default_rng(rows * 1000 + n)
    dlogp, dentropy = (rng.normal(size=rows).astype(np.float32) for _ in range(2))
    grad = erc.erc_score_rows_backward(logits, torch.from_numpy(ids).to(dev()), norm, torch.from_numpy(dlogp).to(dev()),
                                       entropy, torch.from_numpy(dentropy).to(dev()), temperature)
    assert grad.shape == logits.shape and grad.dtype == logits.dtype
    x = f32(logits).astype(np.float64)
    logp, entropy, norm, top_ids, top_logp, grad = (host(v.float() if v.dtype != torch.int32 else v)
                                                    for v in (logp, entropy, norm, top_ids, top_logp, grad))
    for r in range(0, rows, every):
        want = X.score_row(x[r], ids[r], temperature, k)
        ex = spread(x[r], temperature)
        lnz = want[2][1] if want[2][1] > -np.inf else 0.0
        base = SUM + 4 * U * (ex + abs(lnz))

        def near(got, value, extra=0.0):
            if math.isinf(value) or math.isinf(got):
                assert got == value or (value < -3e38 and got == -math.inf), (r, got, value)
            else:
                assert abs(got - value) <= base + 4 * U * abs(value) + extra, (r, got, value)

        near(logp[r], want[0])
        near(entropy[r], want[1], SUM * ex)
        assert norm[r, 0] == want[2][0]
        near(norm[r, 1], want[2][1])
        np.testing.assert_array_equal(top_ids[r], want[3])
        for got, value in zip(top_logp[r], want[4]):
            near(got, value)
        if n == 0:
            continue
        back = X.score_row_backward(x[r], ids[r], dlogp[r], dentropy[r], temperature)
        l = np.where(np.isnan(x[r]), -np.inf, x[r])
        m = l.max()
        if m == -np.inf:
            assert not grad[r].any()
            continue
        with np.errstate(invalid="ignore"):
            t = np.where(l == m, 0.0, (l - m) / temperature)
        # 2^-126 and below is flushed; with t that far down every product is 0 within that
        t = np.maximum(t, -700.0)
        p = np.exp(t - lnz)
        gh, g = abs(dentropy[r]), abs(dlogp[r])
        inside = gh * (np.abs(t) + abs(lnz) + want[1]) + g
        err = p * inside * (base + U * (4 * np.abs(t) + 16)) + p * gh * (2 * base + SUM * ex)
        err = (err + 4 * U * g * (np.arange(n) == ids[r])) / temperature
        tiny = {torch.float32: 2.0**-126, torch.bfloat16: 2.0**-126, torch.float16: 2.0**-24}[logits.dtype]
        bound = err + half_ulp(logits.dtype) * (np.abs(back) + err) + 2 * U * np.abs(back) + tiny * (1 + inside / temperature)
        assert np.all(np.abs(grad[r] - back) <= bound), (r, np.max(np.abs(grad[r] - back) - bound))


def rows_of(rng, rows, n):
    x = rng.normal(size=(rows, n)).astype(np.float32) * np.linspace(0.2, 4, max(rows, 1), dtype=np.float32)[:rows, None]
    x[rng.random((rows, n)) < 0.1] = -np.inf
    return x


def ids_of(rng, rows, n):
    ids = rng.integers(0, max(n, 1), rows).astype(np.int32)
    ids[::5] = [-1, n, 2**31 - 1, -(2**31)][rows % 4]
    return ids


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n", [0, 1, 2, 31, 33, 257, 1000, 1016, 1030, 2033, 2050, 4099])
@pytest.mark.parametrize("k", [0, 1, 5, 32])
def test_against_the_oracle(kind, n, k):
    rng = np.random.default_rng(n + k)
    rows = 9
    x = rows_of(rng, rows, n)
    x[3] = -np.inf
    x[4] = np.round(x[4])  # ties
    x[5] = 1.5
    if n:
        x[6, n // 2] = np.nan
        x[7, :: max(n // 3, 1)] = np.inf
        x[8] = np.finfo(np.float16).min if kind == "f16" else np.float32(-3.3e38)  # a type's lowest is a score
        x[8, n // 3] = -np.inf
    check(torch.from_numpy(x).to(dev()).to(TYPES[kind]), ids_of(rng, rows, n), [0.7, 1.0, 2.5][n % 3], k)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,n", [(3, 20000), (2, 70001), (1, 400003), (2, 169343), (700, 9001)])
@pytest.mark.parametrize("k", [0, 20, 32])
def test_long_rows(kind, rows, n, k):
    rng = np.random.default_rng(n)
    x = torch.from_numpy(rows_of(rng, rows, n)).to(dev()).to(TYPES[kind])
    check(x, ids_of(rng, rows, n), 1.0, k, every=max(1, rows // 5))


def test_the_longest_row():
    n = 4194304
    rng = np.random.default_rng(1)
    x = rng.normal(size=(1, n)).astype(np.float32)
    x[0, [7, n - 1]] = 9.0
    logits = torch.from_numpy(x).to(dev())
    logp, entropy, norm, ids, top = erc.erc_score_rows(logits, torch.tensor([n - 1], dtype=torch.int32, device=dev()), k=3)
    want = X.score_row(x[0].astype(np.float64), n - 1, 1.0, 3)
    assert ids[0].tolist() == want[3].tolist()
    assert abs(logp.item() - want[0]) <= 2 * SUM + 32 * U * 20 and abs(entropy.item() - want[1]) <= 2 * SUM * 16 + 32 * U * 20


@pytest.mark.parametrize("rows,n", [(3, 50), (3, 260), (3, 1000), (3, 9001), (3, 120001), (3000, 3001)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_with_one_sure_entry_keep_their_relative_accuracy(rows, n, kind):
    """ln Z and 1 - p come from the sum without the largest entry, not from a number next to 1."""
    rng = np.random.default_rng(n)
    lead = rng.choice([5.0, 15.0, 25.0], rows)
    x = torch.from_numpy(rng.normal(size=(rows, n)).astype(np.float32)).to(TYPES[kind])
    best = torch.from_numpy(rng.integers(0, n, rows))
    x[torch.arange(rows), best] = x.amax(1) + torch.from_numpy(lead).to(TYPES[kind])
    logits, ids = x.to(dev()), best.to(torch.int32).to(dev())
    logp, entropy, norm, _, top = erc.erc_score_rows(logits, ids, k=0 if rows > 100 else 1)
    one, zero = torch.ones(rows, device=dev()), torch.zeros(rows, device=dev())
    grad = erc.erc_score_rows_backward(logits, ids, norm, one, entropy, zero)
    for r in range(0, rows, max(1, rows // 5)):
        l = f32(logits[r]).astype(np.float64)
        t = np.delete(l, best[r].item()) - l.max()
        rest = np.exp(t).sum()
        # as SUM, and every t within 4 U |t| of its value
        bound = SUM + 4 * U * np.abs(t).max() + 16 * U
        assert abs(logp[r].item() + np.log1p(rest)) <= bound * rest
        assert top is None or top[r, 0].item() == logp[r].item()
        want = np.log1p(rest) - (np.exp(t) * t).sum() / (1 + rest)
        assert abs(entropy[r].item() - want) <= 2 * bound * want
        g = grad[r].double().cpu().numpy()
        half = half_ulp(TYPES[kind])
        assert abs(g[best[r].item()] - rest / (1 + rest)) <= (bound + half) * rest
        others = -np.exp(t) / (1 + rest)
        assert np.all(np.abs(np.delete(g, best[r].item()) - others) <= (bound + half) * np.abs(others))


@pytest.mark.parametrize("n", [300, 5000, 40000])
def test_all_equal_rows_give_the_first_entries(n):
    for value in (0.0, -0.0, 7.0, -3e38):
        x = torch.full((3, n), value, device=dev())
        x[1, ::2] = -x[1, ::2] if value == 0 else x[1, ::2]  # zeros of both signs are equal
        logp, entropy, _, ids, top = erc.erc_score_rows(x, torch.full((3,), n - 1, dtype=torch.int32, device=dev()), k=32)
        assert (ids == torch.arange(32, device=dev(), dtype=torch.int32)).all()
        assert (top + math.log(n)).abs().max() <= SUM + 8 * U * math.log(n)
        assert (logp + math.log(n)).abs().max() <= SUM + 8 * U * math.log(n)
        assert (entropy - math.log(n)).abs().max() <= SUM + 8 * U * math.log(n)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n", [200, 3001, 30001])
def test_strides_and_offsets_that_are_not_aligned(kind, n):
    rng = np.random.default_rng(n)
    for pad, lead in ((0, 1), (1, 0), (3, 2), (8, 3)):
        buffer = torch.full((5 * (n + pad) + lead,), float("nan"), device=dev()).to(TYPES[kind])
        view = buffer[lead:].as_strided((5, n), (n + pad, 1))
        x = rows_of(rng, 5, n)
        view.copy_(torch.from_numpy(x))
        check(view, ids_of(rng, 5, n), 1.0, 7)


def test_rows_that_share_memory():
    x = torch.randn(1, 5000, device=dev()).expand(4, 5000)  # stride 0
    ids = torch.arange(4, dtype=torch.int32, device=dev())
    logp, entropy, norm, top, _ = erc.erc_score_rows(x, ids, k=4)
    assert (entropy == entropy[0]).all() and (top == top[0]).all()
    grad = erc.erc_score_rows_backward(x, ids, norm, torch.ones(4, device=dev()))
    assert grad.is_contiguous() and (grad.sum(1).abs() < 1e-4).all()


def test_optional_parts():
    x = torch.randn(4, 300, device=dev())
    ids = torch.tensor([3, 4, -1, 299], dtype=torch.int32, device=dev())
    logp, entropy, norm, top, _ = erc.erc_score_rows(x, ids)
    none, entropy2, norm2, _, _ = erc.erc_score_rows(x)
    assert none is None and torch.equal(entropy, entropy2) and torch.equal(norm, norm2) and top is None
    g, h = torch.randn(2, 4, device=dev())
    zero = torch.zeros(4, device=dev())
    a = erc.erc_score_rows_backward(x, ids, norm, g)
    assert torch.equal(a, erc.erc_score_rows_backward(x, ids, norm, g, entropy, zero))
    b = erc.erc_score_rows_backward(x, None, norm, None, entropy, h)
    assert torch.equal(b, erc.erc_score_rows_backward(x, ids, norm, zero, entropy, h))
    assert not erc.erc_score_rows_backward(x, None, norm).any()
    # the loss of torch's own operators, in float64
    x64 = x.double().requires_grad_()
    loss = torch.nn.functional.cross_entropy(x64, ids.long(), ignore_index=-1, reduction="sum")
    loss.backward()
    got = erc.erc_score_rows_backward(x, ids, norm, torch.full((4,), -1.0, device=dev()))
    assert (logp.double().sum() + loss).abs() <= 4 * (SUM + 40 * U)
    assert (got - x64.grad).abs().max() <= SUM + 64 * U


@pytest.mark.parametrize("temperature", [2.0**-126, 1e-6, 1e30])
def test_extreme_temperatures(temperature):
    x = torch.tensor([[1.0, 2.0, 2.0, -5.0, -math.inf]], device=dev())
    logp, entropy, norm, ids, top = erc.erc_score_rows(x, torch.zeros(1, dtype=torch.int32, device=dev()), temperature, 5)
    assert ids[0].tolist() == [1, 2, 0, 3, -1]
    live = 2 if temperature < 1 else 4
    assert abs(entropy.item() - math.log(live)) < 1e-6 and abs(top[0, 0].item() + math.log(live)) < 1e-6
    grad = erc.erc_score_rows_backward(x, torch.ones(1, dtype=torch.int32, device=dev()), norm, torch.ones(1, device=dev()),
                                       entropy, torch.zeros(1, device=dev()), temperature)
    assert not torch.isnan(grad).any() and grad[0, 4] == 0


def test_results_repeat_and_calls_on_two_streams_agree():
    x = torch.randn(40, 60001, device=dev()).to(torch.bfloat16)
    ids = torch.arange(40, dtype=torch.int32, device=dev())
    first = erc.erc_score_rows(x, ids, k=20)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    runs = []
    for s in streams:
        with torch.cuda.stream(s):
            runs.append([erc.erc_score_rows(x, ids, k=20) for _ in range(3)])
    torch.cuda.synchronize()
    for run in runs:
        for out in run:
            assert all(torch.equal(a, b) for a, b in zip(first, out))


def test_a_captured_call_replays_on_new_scores():
    x = torch.randn(6, 50001, device=dev())
    ids = torch.zeros(6, dtype=torch.int32, device=dev())
    g = torch.randn(6, device=dev())

    def step():
        out = erc.erc_score_rows(x, ids, k=8)
        return (*out, erc.erc_score_rows_backward(x, ids, out[2], g, out[1], g))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in range(2):
        x.copy_(torch.randn(6, 50001, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))


def test_refusals():
    x = torch.randn(4, 300, device=dev())
    ids = torch.zeros(4, dtype=torch.int32, device=dev())
    norm = torch.zeros(4, 2, device=dev())
    bad = [lambda: erc.erc_score_rows(x.double(), ids), lambda: erc.erc_score_rows(x.t()), lambda: erc.erc_score_rows(x[0]),
           lambda: erc.erc_score_rows(x, ids.long()), lambda: erc.erc_score_rows(x, ids[:3]), lambda: erc.erc_score_rows(x, ids.cpu()),
           lambda: erc.erc_score_rows(x, ids, k=33), lambda: erc.erc_score_rows(x, ids, k=-1), lambda: erc.erc_score_rows(x, ids, k=1.5),
           lambda: erc.erc_score_rows(x, ids, 0.0), lambda: erc.erc_score_rows(x, ids, ws=torch.zeros(9, device=dev())),
           lambda: erc.erc_score_rows_backward(x, ids, norm[:, :1]), lambda: erc.erc_score_rows_backward(x, None, norm, norm[:, 0].contiguous()),
           lambda: erc.erc_score_rows_backward(x, ids, norm, dentropy=norm[:, 0].contiguous())]
    for call in bad:
        with pytest.raises(erc.ErcError) as e:
            call()
        assert e.value.status == erc.ERC_ERR_INVALID_ARG
    with pytest.raises(erc.ErcError) as e:
        erc.erc_score_rows(torch.randn(2, 60000, device=dev()), ws=torch.empty(8, dtype=torch.uint8, device=dev()))
    assert e.value.status == erc.ERC_ERR_CAPACITY
