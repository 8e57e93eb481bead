"""Pins of the oracle of training and answering against closed forms and differences, and the refusals
that need no GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import expert_oracle as X


def test_score_of_equal_entries_is_uniform():
    logp, entropy, norm, ids, top = X.score_row(np.full(7, 3.5), 2, 0.7, 3)
    assert logp == pytest.approx(-math.log(7)) and entropy == pytest.approx(math.log(7))
    assert norm == (3.5, pytest.approx(math.log(7))) and ids.tolist() == [0, 1, 2]
    assert top == pytest.approx([-math.log(7)] * 3)


def test_score_masks_infinities_and_missing_ids():
    row = [np.nan, 1.0, -np.inf, 1.0 + math.log(3)]
    logp, entropy, _, ids, _ = X.score_row(row, 1, 1.0, 4)
    assert logp == pytest.approx(math.log(0.25)) and ids.tolist() == [3, 1, -1, -1]
    assert entropy == pytest.approx(-(0.25 * math.log(0.25) + 0.75 * math.log(0.75)))
    assert X.score_row(row, 0)[0] == -math.inf and X.score_row(row, -1)[0] == 0.0 and X.score_row(row, 4)[0] == 0.0
    assert X.score_row([-np.inf] * 3, 1)[:3] == (-math.inf, 0.0, (-math.inf, -math.inf))
    assert X.score_row([np.inf, 2.0, np.inf], 0)[0] == pytest.approx(-math.log(2))
    assert X.score_row([np.inf, 2.0, np.inf], 1)[0] == -math.inf
    assert X.score_row([], 0)[0] == 0.0  # no id lies in an empty row


@pytest.mark.parametrize("temperature", [0.5, 1.0, 2.0])
def test_score_gradient_is_the_difference_quotient(temperature):
    rng = np.random.default_rng(3)
    l = rng.normal(size=9)
    l[4] = -np.inf
    dlogp, dentropy, i, h = 0.7, -1.3, 6, 1e-6
    want = np.zeros(9)
    for j in range(9):
        if j == 4:
            continue
        up, down = l.copy(), l.copy()
        up[j] += h
        down[j] -= h
        a, b = X.score_row(up, i, temperature), X.score_row(down, i, temperature)
        want[j] = (dlogp * (a[0] - b[0]) + dentropy * (a[1] - b[1])) / (2 * h)
    # second derivatives are below 10 here: h^2 10 / 6 and 2^-52 10 / h
    np.testing.assert_allclose(X.score_row_backward(l, i, dlogp, dentropy, temperature), want, atol=1e-8)
    assert not X.score_row_backward(l, 4, dlogp, 0.0, temperature).any()  # a masked entry
    assert not X.score_row_backward(l, -1, dlogp, 0.0, temperature).any()


@pytest.mark.parametrize("act", [0, 1, 2])
def test_block_gradient_is_the_difference_quotient(act):
    rng = np.random.default_rng(act)
    offsets = np.array([0, 3, 3, 5])
    x, dy = rng.normal(size=(6, 4)), rng.normal(size=(6, 4))
    w = [x, rng.normal(size=(3, 10, 4)), rng.normal(size=(3, 4, 5))]
    _, pre = X.ffn(*w[:1], offsets, *w[1:], act)
    assert np.abs(pre).min(initial=1, where=pre != 0) > 1e-4  # no kink of relu within a step
    got = X.ffn_backward(dy, x, pre, offsets, *w[1:], act)
    h = 1e-6
    for n in range(3):
        flat = rng.choice(w[n].size, 20, replace=False)
        for at in flat:
            value = []
            for step in (h, -h):
                moved = [v.copy() for v in w]
                moved[n].ravel()[at] += step
                value.append((X.ffn(moved[0], offsets, *moved[1:], act)[0] * dy).sum())
            # third derivatives times h^2, and 2^-52 of values up to about 100 over h
            assert got[n].ravel()[at] == pytest.approx((value[0] - value[1]) / (2 * h), abs=1e-7)
    assert not got[0][5].any() and not got[1][1].any() and not got[2][1].any()


def test_activations_against_torch():
    a = np.linspace(-20, 20, 801)
    t = torch.from_numpy(a)
    for act, f in enumerate((torch.nn.functional.silu, torch.nn.functional.gelu, torch.relu)):
        np.testing.assert_allclose(X.act_both(a, act)[0], f(t).numpy(), rtol=1e-13, atol=1e-14)
        live = t.clone().requires_grad_()
        f(live).sum().backward()
        np.testing.assert_allclose(X.act_both(a, act)[1], live.grad.numpy(), rtol=1e-11, atol=1e-13)


def test_dropout_keeps_its_share_and_follows_the_stream():
    keep = X.dropout_keep(40000, 0.3, 12345)
    assert abs(keep.mean() - 0.7) < 5 * math.sqrt(0.21 / 40000)
    np.testing.assert_array_equal(X.dropout_keep(1003, 0.3, 12345, 400), keep[400:1403])
    assert not (X.dropout_keep(40000, 0.3, 12346) == keep).all()
    assert X.dropout_keep(100, 0.0, 1).all() and not X.dropout_keep(100, 1.0, 1).any()
    x = np.arange(8, dtype=np.float32)
    np.testing.assert_array_equal(X.dropout(x, 0.0, 5), x)
    np.testing.assert_array_equal(X.dropout(np.full(8, np.nan, np.float32), 1.0, 5, x), x)


# ---- refusals by the C entry points: sizes, types, values and pointers, before any GPU call
F32, INVALID, CAPACITY = 0, 1, 3
P = ctypes.c_void_p(4096)  # never dereferenced


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2609_27209_gb300 import erc

    return erc.lib()


def score(lib, rows=2, n=8, logits=P, kind=F32, stride=8, ids=P, heat=1.0, k=0, logp=P, top=None):
    return lib.erc_score_rows(rows, n, logits, kind, stride, ids, heat, k, logp, None, None, top, top, None, 0, None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=2**31), dict(n=-1), dict(n=4194305), dict(kind=3), dict(stride=-1),
                                 dict(heat=0.0), dict(heat=-1.0), dict(heat=math.inf), dict(heat=math.nan), dict(heat=1e-40),
                                 dict(k=-1), dict(k=33), dict(k=1), dict(logits=None), dict(ids=None), dict(logp=None),
                                 dict(logits=ctypes.c_void_p(4097))], ids=str)
def test_score_refusals(lib, bad):
    assert score(lib, **bad) == INVALID
    assert lib.erc_last_error()


def test_score_of_no_rows_does_nothing(lib):
    assert score(lib, rows=0, logits=None) == 0


@pytest.mark.parametrize("bad", [dict(n=-1), dict(kind=-1), dict(heat=0.0), dict(norm=None), dict(out=None), dict(logits=None),
                                 dict(ids=None), dict(entropy=None), dict(out=ctypes.c_void_p(4098))], ids=str)
def test_score_backward_refusals(lib, bad):
    a = dict(rows=2, n=8, logits=P, kind=F32, stride=8, ids=P, heat=1.0, norm=P, entropy=P, dlogp=P, dentropy=P, out=P, s=None)
    a.update(bad)
    assert lib.erc_score_rows_backward(*a.values()) == INVALID


@pytest.mark.parametrize("bad", [dict(slots=-1), dict(slots=2**31), dict(experts=0), dict(experts=1025), dict(width=0),
                                 dict(width=65537), dict(inner=0), dict(inner=65537), dict(act=3), dict(act=-1),
                                 dict(type=3)], ids=str)
def test_block_refusals(lib, bad):
    from paper_2609_27209_gb300 import erc

    a = dict(slots=4, experts=2, width=8, inner=8, act=0, type=1)
    a.update(bad)
    shape = ctypes.byref(erc.ErcFfnShapeC(**a))
    big = 1 << 40
    assert lib.erc_expert_ffn(shape, P, P, P, P, P, P, P, big, None) == INVALID
    assert lib.erc_expert_ffn_backward(shape, P, P, P, P, P, P, P, P, P, P, big, None) == INVALID
    if "act" not in bad:
        assert lib.erc_expert_ffn_workspace_size(shape) == lib.erc_expert_ffn_backward_workspace_size(shape) == 0


def test_block_refuses_missing_and_misaligned_arrays_and_small_workspaces(lib):
    from paper_2609_27209_gb300 import erc

    shape = ctypes.byref(erc.ErcFfnShapeC(4, 2, 8, 8, 0, 1))
    odd = ctypes.c_void_p(4097)
    for missing in range(5):
        for v in (None, odd):
            a = [P] * 5
            a[missing] = v
            assert lib.erc_expert_ffn(shape, *a, P, P, 1 << 30, None) == INVALID
    assert lib.erc_expert_ffn(None, P, P, P, P, P, P, P, 1 << 30, None) == INVALID
    need = lib.erc_expert_ffn_workspace_size(shape)
    assert lib.erc_expert_ffn(shape, P, P, P, P, P, None, P, need - 1, None) == CAPACITY
    assert lib.erc_expert_ffn(shape, P, P, P, P, P, None, None, need, None) == CAPACITY
    for missing in range(6):
        for v in (None, odd):
            a = [P] * 6
            a[missing] = v
            assert lib.erc_expert_ffn_backward(shape, *a, P, P, P, P, 1 << 30, None) == INVALID
    need = lib.erc_expert_ffn_backward_workspace_size(shape)
    assert lib.erc_expert_ffn_backward(shape, P, P, P, P, P, P, P, P, P, P, need - 1, None) == CAPACITY


@pytest.mark.parametrize("bad", [dict(count=-1), dict(x=None), dict(kind=5), dict(p=-0.1), dict(p=1.1), dict(p=math.nan),
                                 dict(key_dev=ctypes.c_void_p(4100)), dict(first=-4), dict(first=2), dict(out=None),
                                 dict(residual=ctypes.c_void_p(4097)), dict(count=2**49)], ids=str)
def test_dropout_refusals(lib, bad):
    a = dict(count=8, x=P, kind=F32, residual=None, p=0.5, key=1, key_dev=None, first=0, out=P, s=None)
    a.update(bad)
    assert lib.erc_dropout(*a.values()) == INVALID


def test_the_binding_refuses_host_tensors_and_wrong_types():
    from paper_2609_27209_gb300 import erc

    x = torch.zeros(4, 8)
    for call in (lambda: erc.erc_score_rows(x), lambda: erc.erc_dropout(x, 0.5, 1), lambda: erc.erc_dropout(None, 0.5, 1),
                 lambda: erc.erc_score_rows_backward(x, None, torch.zeros(4, 2)),
                 lambda: erc.erc_expert_ffn(x, torch.zeros(2, dtype=torch.int64), torch.zeros(1, 16, 8), torch.zeros(1, 8, 8)),
                 lambda: erc.erc_expert_ffn_backward(x, x, x, None, x, x)):
        with pytest.raises(erc.ErcError) as e:
            call()
        assert e.value.status == INVALID


def test_shape_layout_matches_the_header(tmp_path):
    import os
    import subprocess

    from paper_2609_27209_gb300 import erc

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [f for f, _ in erc.ErcFfnShapeC._fields_]
    src = tmp_path / "shape.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "erc.h"\nint main(void) {\n  printf("%zu'
                   + " %zu" * len(names) + '\\n", sizeof(erc_ffn_shape), '
                   + ", ".join(f"offsetof(erc_ffn_shape, {f})" for f in names) + ");\n  return 0;\n}\n")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "shape")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "shape")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(erc.ErcFfnShapeC)] + [getattr(erc.ErcFfnShapeC, f).offset for f in names]
