"""The row-wise choices at the ends of their ranges: scores below 2^-126, sums that cancel or overflow,
calls from several threads, and arguments that do not fit."""
import numpy as np
import pytest
import torch

from oracle import choice_oracle as C

from ._gpu import dev
from .test_gpu_choice import TYPES, check_route

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
