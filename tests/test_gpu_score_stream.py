"""Rows of scores by the thousand, which a warp each takes: no row is too long for its sums, and masks, infinities, types and
alignments are those of the other forms."""
import math

import numpy as np
import pytest
import torch

from oracle import expert_oracle as X
from paper_2609_27209_gb300 import erc

from ._gpu import dev
from .test_gpu_score import TYPES, U, check, f32, ids_of, rows_of, spread

pytestmark = pytest.mark.gpu

MANY = 3000  # rows enough for a warp each on any part of up to 166 SMs
# Z of positive terms: a lane's 128 one by one (127 U), a sum that keeps its roundings (2 U), two halves, 32 lanes (6 U), the
# exponential (2^-22 = 4 U) of a term and of the scalings to a new anchor, which halve (8 U), and their products
FEW = 170 * U


def rows_of_one(row, kind):
    """MANY rows that are all the same memory."""
    return torch.from_numpy(row).to(kind).to(dev()).view(1, -1).expand(MANY, row.size)


def near_the_oracle(x, i, temperature=1.0):
    ids = torch.full((MANY,), i, dtype=torch.int32, device=dev())
    logp, entropy, norm, _, _ = erc.erc_score_rows(x, ids, temperature)
    assert all(torch.equal(v, v[:1].expand_as(v)) for v in (logp, entropy, norm))
    l = f32(x[0]).astype(np.float64)
    want = X.score_row(l, i, temperature)
    ex, lnz = spread(l, temperature), want[2][1]
    base = FEW + 4 * U * (ex + abs(lnz))
    assert norm[0, 0].item() == want[2][0]
    for got, value, bound in ((norm[0, 1], lnz, base), (logp[0], want[0], base + 4 * U * abs(want[0])),
                              (entropy[0], want[1], base + 4 * U * abs(want[1]) + 2 * FEW * ex)):
        assert abs(got.item() - value) <= bound, (got.item(), value, (got.item() - value) / U, bound / U)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n", [300000, 1048576, 4194304])
@pytest.mark.parametrize("gap", [0.5, 1.25, 7.0])
def test_long_rows_of_two_values(kind, n, gap):
    """Equal terms round the same way each time."""
    row = np.full(n, -gap, np.float32)
    row[n // 3] = 0.0
    near_the_oracle(rows_of_one(row, TYPES[kind]), n // 3)
    row[::5] = 0.0
    near_the_oracle(rows_of_one(row, TYPES[kind]), n - 2)


@pytest.mark.parametrize("n,top", [(300000, 1.0), (4194304, 30.0), (4194304, 0.001)])
def test_rows_that_rise_all_along(n, top):
    """Every round has a new largest entry."""
    row = np.linspace(0.0, top, n, dtype=np.float32)
    near_the_oracle(rows_of_one(row, torch.float32), n - 1)
    near_the_oracle(rows_of_one(row - np.float32(4.0), torch.float32), 0, 0.7)


@pytest.mark.parametrize("n", [300000])
def test_the_gradient_of_a_long_row_of_two_values_sums_to_zero(n):
    row = np.full(n, -1.25, np.float32)
    row[7] = 0.0
    x = rows_of_one(row, torch.float32)
    norm = erc.erc_score_rows(x)[2]
    ids = torch.full((MANY,), 7, dtype=torch.int32, device=dev())
    grad = erc.erc_score_rows_backward(x[:3], ids[:3], norm[:3].contiguous(), torch.ones(3, device=dev()))
    # sum_i p_i = 1 within ln Z's error and a few roundings of each p
    assert grad.double().sum(1).abs().max().item() <= FEW + 4 * U * math.log(n) + 32 * U


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n", [2050, 3001, 9999])
def test_masks_and_infinities(kind, n):
    rng = np.random.default_rng(n)
    x = rows_of(rng, 9, n)
    x[1] = -np.inf
    x[2] = np.nan
    x[3] = np.round(x[3])  # ties
    x[4, n // 2] = np.nan
    x[5, :: n // 3] = np.inf
    x[6] = np.finfo(np.float16).min if kind == "f16" else np.float32(-3.3e38)  # a type's lowest is a score
    x[6, n // 3] = -np.inf
    x[7, : n - 1] = -np.inf  # one entry is left, the last
    x[7, n - 1] = 3.0
    x[8, 1:] = -np.inf
    x[8, 0] = -0.0
    many = np.tile(x, (MANY // 9 + 1, 1))
    check(torch.from_numpy(many).to(dev()).to(TYPES[kind]), ids_of(rng, len(many), n), [0.7, 1.0, 2.5][n % 3], 0, every=101)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("pad,lead", [(0, 1), (1, 0), (3, 2), (8, 3)])
def test_rows_of_changing_alignment(kind, pad, lead):
    n = 2500
    rng = np.random.default_rng(pad)
    buffer = torch.full((MANY * (n + pad) + lead,), float("nan"), device=dev()).to(TYPES[kind])
    view = buffer[lead:].as_strided((MANY, n), (n + pad, 1))
    view.copy_(torch.from_numpy(rows_of(rng, MANY, n)))
    check(view, ids_of(rng, MANY, n), 1.0, 0, every=97)


def test_a_row_does_not_depend_on_how_many_there_are():
    """Few rows take another form: the same row within both forms' bounds."""
    x = torch.randn(MANY, 5001, generator=torch.Generator().manual_seed(1)).to(dev())
    many, few = erc.erc_score_rows(x), erc.erc_score_rows(x[:100].contiguous())
    assert (many[2][:100, 1] - few[2][:, 1]).abs().max().item() <= FEW + 640 * U
