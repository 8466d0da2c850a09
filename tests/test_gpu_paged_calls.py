"""Calls of the paged cache that its documentation allows, away from the ordinary ones: gates
that are not finite in an earlier call, rows whose own page is not in the cache, rows that no
sequence brings, scales that do not bound the logits, call arrays of any content."""
import math

import pytest
import torch

from paper_2504_06949_amd import acp, ops
from tests._helpers import ensure_built
from tests.test_gpu_paged import BF, E, EPS, F32, World

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---- gates ---------------------------------------------------------------------------------

@pytest.mark.parametrize("n", [1, 16, 17, 64, 65, 3000])
@pytest.mark.parametrize("gate", [-math.inf, math.nan, math.inf])
def test_a_sum_of_gates_that_is_not_finite_stays_reported(n, gate):
    """Every later sum of the head inherits it, whatever its own gates."""
    H = 5                                                # (more heads than a workgroup sums, and not a multiple)
    cache = ops.PagedCache(60, H, 64, 1)
    table = torch.arange(60, dtype=torch.int32, device="cuda")[None]
    flags = torch.full((1, H), -1, dtype=torch.int32, device="cuda")
    at = 0
    for call, rows in enumerate((n, min(n, 400), min(n, 400))):
        kv = torch.zeros((rows, 1, 64), dtype=BF, device="cuda")
        f = torch.full((rows, H), -0.25, device="cuda")
        if call == 0:
            f[n // 2, 1] = f[n - 1, 4] = gate
        cache.append(kv, kv, f, ints(0, rows), ints(at), table, flags=flags)
        assert flags.tolist() == [[0, 2, 0, 0, 2]], call
        at += rows
