"""GPU tests of the batch operators at edges of their contract: what a status says, where weights
and scores lose digits, and calls over several steps."""

import math

import pytest
import torch

import batch_ref as R
from test_gpu_batch_ops import TYPES, attend, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _built():
    from paper_2608_00814_gb300 import _build
    _build.build()


# ------------------------------------------------------------------ scores that are not finite

@pytest.mark.parametrize("dtype, kv", TYPES[1:])
@pytest.mark.parametrize("own", [1, 16, 17, 100])
def test_attention_nan_key_beside_a_long_prefix(dtype, kv, own):
    """Own keys that leave parts for a join with the prefix's: a NaN key that is seen makes its rows NaN, and only
    those, wherever among the own keys it is."""
    counts, victims = [1 + i % 2 for i in range(100)], (3, 40, 99)
    lens = [c + 4 * i % 400 for i, c in enumerate(counts)]
    for b in victims:
        lens[b] = max(own, counts[b])
    step = R.Step(counts, lens, 16)
    q, pk, pv, kp, vp = inputs(step, 20000, 8, 1, 128, dtype, kv)
    want = torch.zeros(step.n, dtype=torch.bool)
    for b, key in zip(victims, (0, lens[40] // 2, lens[99] - counts[99])):   # all rows of a sequence see its key
        p, e = step.where(b, min(key, lens[b] - counts[b]))
        kp[p, e, 0, 9] = math.nan
        want[step.q_start[b]:step.q_start[b + 1]] = True
    out, st = attend(step, q, pk, pv, 20000, kp, vp)
    assert int(st) == 0
    nan = torch.isnan(out).cpu()
    assert torch.equal(nan.all(-1).all(-1), want) and torch.equal(nan.any(-1).any(-1), want)
