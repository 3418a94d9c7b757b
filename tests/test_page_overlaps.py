"""oos_paged_compact refuses new lengths that lie on what its blocks still read (no GPU)."""

import ctypes

import pytest

from paper_2608_00814_gb300 import binding as B
from test_batch_refusals import L, NULL, batch, cache  # noqa: F401
from test_page_refusals import cache8

SEQS, TOKENS, WIDTH = 5, 9, 4
# arrays of the call, far from each other, and their elements
SIZES = {"q_start": SEQS + 1, "seq_len": SEQS, "table": SEQS * WIDTH, "nodes": TOKENS, "length": SEQS, "status": 1}
AT = {name: 0x10000 * (i + 1) for i, name in enumerate(SIZES)}


def compact(L, kind, new):
    b = batch(n_seqs=SEQS, n_tokens=TOKENS, width=WIDTH, **{k: AT[k] for k in ("q_start", "seq_len", "table")})
    c, f = (cache8(), L.oos_paged_compact8) if kind == 8 else (cache(), L.oos_paged_compact)
    return f(ctypes.byref(c), 1, ctypes.byref(b), AT["nodes"], AT["length"], new, AT["status"], NULL)


@pytest.mark.parametrize("kind", [8, 16])
@pytest.mark.parametrize("name", list(SIZES))
def test_new_lengths_on_an_argument(L, kind, name):
    """Its first element, its last, and an array that ends on its first one."""
    for new in (AT[name], AT[name] + 4 * (SIZES[name] - 1), AT[name] - 4 * (SEQS - 1)):
        assert compact(L, kind, new) == B.OOS_EINVAL
