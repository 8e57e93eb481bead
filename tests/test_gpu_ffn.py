"""GPU parity of the gated feed-forward block of experts and its gradients, within bounds derived from the
roundings that the header states."""
import numpy as np
import pytest
import torch

from oracle import expert_oracle as X
from paper_2609_27209_gb300 import erc

from ._gpu import dev

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0**-24
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0**-25}  # half the spacing of subnormal values


def f64(t):
    return t.detach().double().cpu().numpy()


def per_expert(f, offsets, rows, experts):
    """f(e, slice) for each expert with rows"""
    for e in range(experts):
        s = slice(int(offsets[e]), int(offsets[e + 1]))
        if s.start < s.stop:
            f(e, s)


def inputs(seed, counts, behind, width, inner, kind):
    g = torch.Generator().manual_seed(seed)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
    slots = int(offsets[-1]) + behind
    E = len(counts)
    mk = lambda *s, scale=1.0: (scale * torch.randn(*s, generator=g)).to(TYPES[kind]).to(dev())  # noqa: E731
    x, dy = mk(slots, width), mk(slots, width)
    x[offsets[-1]:] = float("nan")
    dy[offsets[-1]:] = float("nan")
    return offsets, x, dy, mk(E, 2 * inner, width, scale=width**-0.5), mk(E, width, inner, scale=inner**-0.5)


def check(offsets, x, dy, w_in, w_out, act):
    kind, E, inner, width = x.dtype, w_in.shape[0], w_out.shape[2], x.shape[1]
    half, tiny, used = torch.finfo(kind).eps / 2, TINY[kind], int(offsets[-1])
    at = torch.from_numpy(offsets).to(dev())
    y, pre = erc.erc_expert_ffn(x, at, w_in, w_out, act=act, keep=True)
    y2, none = erc.erc_expert_ffn(x, at, w_in, w_out, act=act)
    assert none is None and torch.equal(y, y2) and y.dtype == pre.dtype == kind
    assert not y[used:].any() and not pre[used:].any()
    X64, W1, W2 = f64(x), f64(w_in), f64(w_out)
    X64[used:] = 0
    want_y, want_pre = X.ffn(X64, offsets, W1, W2, act)
    got_y, got_pre = f64(y), f64(pre)
    assert np.isfinite(got_y).all() and np.isfinite(got_pre).all()

    def forward(e, s):
        # a sum of D products in float32, in any order: (D + 2) U of the sum of magnitudes, twice that where the adder
        # of the tensor cores cuts instead of rounding
        dpre = 2 * (width + 2) * U * (np.abs(X64[s]) @ np.abs(W1[e]).T)
        bound = dpre + half * (np.abs(want_pre[s]) + dpre) + tiny
        assert np.all(np.abs(got_pre[s] - want_pre[s]) <= bound), np.max(np.abs(got_pre[s] - want_pre[s]) / bound)
        a, b = want_pre[s, :inner], want_pre[s, inner:]
        da, db = dpre[:, :inner], dpre[:, inner:]
        value = np.abs(X.act_both(a, act)[0])
        h = value * np.abs(b)
        # |act'| <= 1.13; the activation's own evaluation costs some 8 U of its argument's size
        dh = 1.13 * da * (np.abs(b) + db) + value * db + 8 * U * (np.abs(a) + 1) * np.abs(b)
        dh = dh + half * (h + dh) + tiny
        bound = (dh + 2 * (inner + 2) * U * (h + dh)) @ np.abs(W2[e]).T
        bound = bound + half * (np.abs(want_y[s]) + bound) + tiny
        assert np.all(np.abs(got_y[s] - want_y[s]) <= bound), np.max(np.abs(got_y[s] - want_y[s]) / bound)

    per_expert(forward, offsets, x.shape[0], E)

    # the gradient, from the stored pre; what lies behind the last expert's rows must not matter
    pre_behind = pre.clone()
    pre_behind[used:] = float("nan")
    dx, dw_in, dw_out = erc.erc_expert_ffn_backward(dy, x, pre_behind, at, w_in, w_out, act=act)
    assert not dx[used:].any() and dx.dtype == dw_in.dtype == dw_out.dtype == kind
    DY = f64(dy)
    DY[used:] = 0
    want = X.ffn_backward(DY, X64, got_pre, offsets, W1, W2, act)
    got = [f64(t) for t in (dx, dw_in, dw_out)]

    def backward(e, s):
        a, b = got_pre[s, :inner], got_pre[s, inner:]
        value, slope = X.act_both(a, act)
        dh = DY[s] @ W2[e]
        ddh = 2 * (width + 2) * U * (np.abs(DY[s]) @ np.abs(W2[e]))
        g = np.concatenate([dh * b * slope, dh * value], 1)
        size = np.concatenate([(np.abs(dh) + ddh) * np.abs(b), (np.abs(dh) + ddh) * (np.abs(value) + np.abs(a) * 2.0**-10)], 1)
        dg = np.concatenate([ddh * np.abs(b * slope), ddh * np.abs(value)], 1) + 16 * U * (1 + np.abs(a).max()) * size
        dg = dg + half * (np.abs(g) + dg) + tiny
        h = np.abs(value * b)
        dhh = 8 * U * (np.abs(a) + 1) * np.abs(b)
        dhh = dhh + half * (h + dhh) + tiny
        rows = s.stop - s.start
        bounds = [(dg + 2 * (2 * inner + 2) * U * (np.abs(g) + dg)) @ np.abs(W1[e]),
                  (dg + 2 * (rows + 2) * U * (np.abs(g) + dg)).T @ np.abs(X64[s]),
                  np.abs(DY[s]).T @ (dhh + 2 * (rows + 2) * U * (h + dhh))]
        for have, ref, bound in zip((got[0][s], got[1][e], got[2][e]), (want[0][s], want[1][e], want[2][e]), bounds):
            bound = bound + half * (np.abs(ref) + bound) + tiny
            assert np.all(np.abs(have - ref) <= bound), np.max(np.abs(have - ref) / bound)

    per_expert(backward, offsets, x.shape[0], E)
    for e in range(E):
        if offsets[e] == offsets[e + 1]:
            assert not got[1][e].any() and not got[2][e].any()


COUNTS = {"one": [1], "tail": [65, 0, 1, 0], "empty": [0, 0], "ragged": [3, 130, 0, 257, 8, 16, 1], "even": [128, 128], "long": [700]}


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("width,inner", [(8, 8), (1, 1), (7, 13), (64, 64), (72, 40), (136, 264), (520, 200), (100, 67)])
@pytest.mark.parametrize("counts", COUNTS)
def test_against_the_oracle(kind, width, inner, counts):
    seed = width * 100 + inner
    check(*inputs(seed, COUNTS[counts], 5 if counts != "one" else 0, width, inner, kind), act=seed % 3)


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_every_activation(kind, act):
    check(*inputs(act, [40, 300], 0, 256, 128, kind), act=act)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_many_experts(kind):
    counts = np.random.default_rng(4).integers(0, 9, 1024)
    counts[::3] = 0
    check(*inputs(2, counts.tolist(), 3, 16, 24, kind), act=0)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_wide_and_deep(kind):
    check(*inputs(5, [300, 20], 0, 1032, 520, kind), act=0)


def test_a_dense_block_of_many_rows():
    check(*inputs(6, [3001], 0, 128, 192, "bf16"), act=1)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("width,inner", [(24, 16), (17, 40), (264, 8), (264, 136)])
@pytest.mark.parametrize("counts", [[9000], [4001, 0, 5003]], ids=str)
def test_long_sums_of_small_weights(kind, width, inner, counts):
    """The weights' gradients are few tiles over many slots: summed in parts, which are then added."""
    check(*inputs(13, counts, 4, width, inner, kind), act=0)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("width,inner", [(201, 203), (200, 203), (203, 200)])
def test_odd_widths_of_many_rows(kind, width, inner):
    """16-bit rows that are not whole 16-byte pieces are copied into rows that are."""
    check(*inputs(14, [2500, 0, 131], 7, width, inner, kind), act=1)
    offsets, x, dy, w_in, w_out = inputs(15, [2900], 3, width, inner, kind)
    at = torch.from_numpy(offsets).to(dev())
    y, pre = erc.erc_expert_ffn(x, at, w_in, w_out, keep=True)
    full = erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out)
    rows = erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out, dw=False)
    weights = erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out, dxs=False)
    assert torch.equal(rows[0], full[0]) and torch.equal(weights[1], full[1]) and torch.equal(weights[2], full[2])
    assert torch.equal(erc.erc_expert_ffn(x, at, w_in, w_out)[0], y)


def test_rows_that_hold_infinities_stay_by_themselves():
    offsets, x, dy, w_in, w_out = inputs(7, [70, 60], 0, 64, 64, "bf16")
    at = torch.from_numpy(offsets).to(dev())
    y, pre = erc.erc_expert_ffn(x, at, w_in, w_out, keep=True)
    dx, dw_in, dw_out = erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out)
    for value in (float("nan"), float("inf")):
        x2, dy2 = x.clone(), dy.clone()
        x2[70], dy2[71] = value, value  # rows of the second expert, next to the first one's last
        y2, pre2 = erc.erc_expert_ffn(x2, at, w_in, w_out, keep=True)
        dx2, dw_in2, dw_out2 = erc.erc_expert_ffn_backward(dy2, x2, pre2, at, w_in, w_out)
        assert torch.equal(y2[:70], y[:70]) and torch.equal(y2[71:], y[71:]) and torch.equal(dx2[:70], dx[:70])
        assert torch.equal(dw_in2[0], dw_in[0]) and torch.equal(dw_out2[0], dw_out[0])


def test_large_gates_saturate_without_nan():
    for act in (0, 1, 2):
        w_in = torch.ones(1, 16, 8, device=dev(), dtype=torch.bfloat16)
        w_out = torch.ones(1, 8, 8, device=dev(), dtype=torch.bfloat16)
        x = torch.tensor([[200.0], [-200.0], [1e30], [-1e30]], device=dev()).expand(4, 8).contiguous().to(torch.bfloat16)
        at = torch.tensor([0, 4], device=dev())
        y, pre = erc.erc_expert_ffn(x, at, w_in, w_out, act=act, keep=True)
        dx, _, _ = erc.erc_expert_ffn_backward(torch.full_like(x, 1e-30), x, pre, at, w_in, w_out, act=act)
        assert not torch.isnan(y).any() and not torch.isnan(dx).any()
        assert (y[1].float().abs() < 1e-30).all()


def test_parts_of_the_gradient():
    offsets, x, dy, w_in, w_out = inputs(8, [33, 0, 70], 2, 64, 72, "bf16")
    at = torch.from_numpy(offsets).to(dev())
    x[103:] = 0
    _, pre = erc.erc_expert_ffn(x, at, w_in, w_out, keep=True)
    full = erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out)
    rows = erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out, dw=False)
    weights = erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out, dxs=False)
    assert rows[1] is None and rows[2] is None and weights[0] is None
    assert torch.equal(rows[0], full[0]) and torch.equal(weights[1], full[1]) and torch.equal(weights[2], full[2])
    assert erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out, dxs=False, dw=False) == (None, None, None)


def test_no_slots():
    w_in, w_out = torch.randn(3, 32, 8, device=dev()), torch.randn(3, 8, 16, device=dev())
    x, at = torch.empty(0, 8, device=dev()), torch.zeros(4, dtype=torch.int64, device=dev())
    y, pre = erc.erc_expert_ffn(x, at, w_in, w_out, keep=True)
    assert y.shape == (0, 8) and pre.shape == (0, 32)
    dx, dw_in, dw_out = erc.erc_expert_ffn_backward(y, x, pre, at, w_in, w_out)
    assert dx.shape == (0, 8) and not dw_in.any() and not dw_out.any()


def test_misaligned_arrays_take_another_path_to_the_same_answer():
    offsets, x, dy, w_in, w_out = inputs(9, [50, 30], 0, 64, 64, "bf16")

    def moved(t):
        buffer = torch.empty(t.numel() + 1, dtype=t.dtype, device=dev())
        buffer[1:] = t.reshape(-1)
        return buffer[1:].view(t.shape)

    check(offsets, moved(x), dy, w_in, w_out, 0)
    check(offsets, x, moved(dy), w_in, moved(w_out), 0)


def test_results_repeat_and_calls_on_two_streams_agree():
    offsets, x, dy, w_in, w_out = inputs(10, [300, 41, 0, 500], 0, 256, 320, "bf16")
    at = torch.from_numpy(offsets).to(dev())

    def step():
        y, pre = erc.erc_expert_ffn(x, at, w_in, w_out, keep=True)
        return (y, pre, *erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out))

    first = step()
    torch.cuda.synchronize()
    runs = []
    for s in [torch.cuda.Stream() for _ in range(3)]:
        with torch.cuda.stream(s):
            runs += [step(), step()]
    torch.cuda.synchronize()
    for out in runs:
        assert all(torch.equal(a, b) for a, b in zip(first, out))


def test_a_captured_step_replays_on_new_rows_and_loads():
    offsets, x, dy, w_in, w_out = inputs(11, [100, 28, 72], 0, 128, 64, "bf16")
    at = torch.from_numpy(offsets).to(dev())

    def step():
        y, pre = erc.erc_expert_ffn(x, at, w_in, w_out, keep=True)
        return (y, pre, *erc.erc_expert_ffn_backward(dy, x, pre, at, w_in, w_out))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for counts in ([100, 28, 72], [0, 200, 0], [1, 1, 1]):
        x.copy_(torch.randn(200, 128, generator=torch.Generator().manual_seed(counts[0])))
        at.copy_(torch.tensor([0, *np.cumsum(counts)]))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))


def test_refusals():
    offsets, x, dy, w_in, w_out = inputs(12, [4, 4], 0, 16, 8, "bf16")
    at = torch.from_numpy(offsets).to(dev())
    pre = torch.zeros(8, 16, device=dev(), dtype=torch.bfloat16)
    bad = [lambda: erc.erc_expert_ffn(x.t(), at, w_in, w_out), lambda: erc.erc_expert_ffn(x, at.int(), w_in, w_out),
           lambda: erc.erc_expert_ffn(x, at[:2], w_in, w_out), lambda: erc.erc_expert_ffn(x, at, w_in[:, :15], w_out),
           lambda: erc.erc_expert_ffn(x, at, w_in.half(), w_out), lambda: erc.erc_expert_ffn(x, at, w_in, w_out.transpose(1, 2)),
           lambda: erc.erc_expert_ffn(x, at, w_in, w_out, act=3), lambda: erc.erc_expert_ffn(x, at, w_in, w_out, act=0.5),
           lambda: erc.erc_expert_ffn(x, at.cpu(), w_in, w_out), lambda: erc.erc_expert_ffn(x, at, w_in, w_out[0]),
           lambda: erc.erc_expert_ffn_backward(dy[:4], x, pre, at, w_in, w_out),
           lambda: erc.erc_expert_ffn_backward(dy, x, pre[:, :8], at, w_in, w_out),
           lambda: erc.erc_expert_ffn_backward(dy, x, None, at, w_in, w_out)]
    for call in bad:
        with pytest.raises(erc.ErcError) as e:
            call()
        assert e.value.status == erc.ERC_ERR_INVALID_ARG
    for call in (erc.erc_expert_ffn, lambda *a, ws: erc.erc_expert_ffn_backward(dy, a[0], pre, *a[1:], ws=ws)):
        with pytest.raises(erc.ErcError) as e:
            call(x, at, w_in, w_out, ws=torch.empty(16, dtype=torch.uint8, device=dev()))
        assert e.value.status == erc.ERC_ERR_CAPACITY


@pytest.mark.parametrize("slots,width,inner", [(300, 8192, 64), (2000, 4096, 640)])
def test_long_float32_sums_keep_their_last_bits(slots, width, inner):
    """n terms of mixed signs, summed 256 at a time: the k-th partial sum's square is k of a term's, its rounding's at
    most U^2 / 3 of that, so the sums of 256 add 256 U^2 / 6 and the sum of those n / 256 U^2 / 6 to the squared error.
    A single sum in order would add n U^2 / 6."""
    offsets, x, _, w_in, w_out = inputs(31, [slots], 0, width, inner, "f32")
    at = torch.from_numpy(offsets).to(dev())
    _, pre = erc.erc_expert_ffn(x, at, w_in, w_out, act=erc.ERC_ACT_SILU, keep=True)
    want = f64(x) @ f64(w_in[0]).T
    error = np.linalg.norm(f64(pre) - want) / np.linalg.norm(want)
    assert error <= U * np.sqrt((256 + width / 256) / 6), error / U
