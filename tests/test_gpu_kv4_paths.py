"""The 4-bit paged cache where its kernels take other ways than small calls do: stages used again, many tokens, many layers, plans of many
units.  Tables, bytes and copies exactly; attention with the tolerance of test_gpu_kv4.py."""
import numpy as np
import pytest
import torch

from oracle import ref
from paper_2608_04962_b200 import binding as S
from tests.test_gpu_kv4 import _bits, _case, _check, _f64, _run
from tests.util import dev, dev_bf16, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,Hq,D", [(1, 4, 64), (1, 16, 128), (8, 4, 128)])
@pytest.mark.parametrize("missing", [2, 3, 7])
def test_pages_that_are_missing_in_turn_with_pages_that_are_there(N, Hq, D, missing):
    """Few rows: a stage is filled by plain stores for a page that does not exist and by copies for the next one, many times over, and a
    cut plan's search has used the first stage before either."""
    x = _case(4, N, Hq, 2, D, [9000, 700, 0, 5000], seed=30 + missing)
    for b in range(4):
        for i in range(x["indptr"][b], x["indptr"][b + 1]):
            if (i - x["indptr"][b]) % missing == b % missing:
                x["table"][i] = -1 if i % 2 else x["pool"].shape[0] + i
                at = (i - x["indptr"][b]) * 128
                for w in (x["K"], x["V"]):
                    w[b][at:at + 128] = 0
    O = _check(x)
    assert all(torch.equal(O, _run(x)) for _ in range(10))
