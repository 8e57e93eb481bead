"""The gated feed-forward block at the ends of its ranges: an expert with as many rows as there can be."""
import numpy as np
import pytest
import torch

from oracle import expert_oracle as X
from paper_2609_27209_gb300 import erc

from ._gpu import dev
from .test_gpu_ffn import f64

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def test_an_expert_with_as_many_rows_as_there_can_be():
    slots = 2**31 - 1  # x, y and the hidden rows: 34 GB each
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB")
    g = torch.Generator().manual_seed(1)
    w_in = (torch.randn(2, 16, 8, generator=g) / 2).bfloat16().to(dev())
    w_out = (torch.randn(2, 8, 8, generator=g) / 2).bfloat16().to(dev())
    x = torch.zeros(slots, 8, dtype=torch.bfloat16, device=dev())
    at = torch.tensor([0, 300, slots - 3], device=dev())
    places = [0, 2**30, 2**31 - 2**23, slots - 403]  # the last: 400 rows and the 3 behind the experts
    for p in places:
        x[p : p + 400] = torch.randn(400, 8, generator=g).bfloat16().to(dev())
    y, _ = erc.erc_expert_ffn(x, at, w_in, w_out)
    assert not y[-3:].any()
    for p in places:
        own = np.array([0, 300 if p == 0 else 0, 400])
        want, _ = X.ffn(f64(x[p : p + 400]), own, f64(w_in), f64(w_out), 0)
        # roundings of bfloat16: of h (2^-8 of it) and of the result; sums of 8 terms, at most 8 times a result's size
        assert np.abs(f64(y[p : p + 400]) - want).max() <= 8 * 2.0**-8 * np.abs(want).max()
    assert not y[1000:10000].any()
