"""Attention over the paged cache where queries or keys are NaN or infinite, against the definition in
64 bits (GPU only): what is not a number reaches exactly the rows whose scores it is part of, however the work
is divided: one warp's keys, one stream's blocks, one CTA's part of a unit."""
import math

import pytest
import torch

from tests._gpu import flglm, need_gpu
from tests._kv import Paged, attention64, check_attention
from tests.test_gpu_kv import run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


CASES = {  # new, lens, heads, kv heads, head_dim, page
    "one key": ([1], [1], 2, 2, 64, 16),
    "a key alone in its warp": ([1], [17], 2, 2, 128, 16),
    "one token in many parts": ([1], [5000], 4, 2, 128, 32),
    "few tokens": ([3, 1, 2], [40, 300, 66], 4, 2, 64, 16),
    "one tile, two streams": ([20], [200], 4, 2, 128, 64),
    "one tile in many parts": ([40], [1500], 2, 1, 64, 64),
    "two tiles in many parts": ([150], [1100], 2, 1, 128, 128),
    "whole units": ([140] + [17] * 90, [140] + [40 + 3 * i for i in range(90)], 2, 2, 128, 16),
}


def compare(p, q, heads, o, lse):
    ro, rl, size = attention64(p, q, heads)
    # A row whose scores are all -infinity has a sum of zero: as if it saw nothing.  One with a score of +infinity is
    # infinity over infinity.
    none = (rl == -math.inf).T[..., None]
    ro, size = (torch.where(none, 0.0, x) for x in (ro, size))
    rl = torch.where(rl == math.inf, math.nan, rl)
    assert torch.equal(torch.isnan(o), torch.isnan(ro))
    check_attention(p, o, lse, (ro, rl, size))
    assert p.status.item() == 0


def key(p, s, u):
    """Where key u of sequence s lies."""
    return int(p.table[s, u // p.page]), u % p.page


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_query_that_is_not_finite(F, case, dtype, value):
    new, lens, heads, kvh, hd, page = CASES[case]
    p = Paged(F, new, lens, kvh, hd, page, dtype, seed=41)
    q = p.randn(p.T, heads, hd)
    q[0, 1, 5] = value
    q[p.T - 1, 0, hd - 1] = value
    _, o, lse = run_attention(F, p, heads, q=q)
    if math.isnan(value):
        for t, h in ((0, 1), (p.T - 1, 0)):
            assert bool(torch.isnan(o[t, h]).all()) and math.isnan(float(lse[h, t]))
    compare(p, q, heads, o, lse)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("where", ["first", "middle", "last"])
def test_a_key_that_is_not_finite(F, case, where, value):
    new, lens, heads, kvh, hd, page = CASES[case]
    p = Paged(F, new, lens, kvh, hd, page, seed=43)
    for s in {0, len(lens) - 1}:
        u = {"first": 0, "middle": lens[s] // 2, "last": lens[s] - 1}[where]
        p.k[key(p, s, u)][0, 7] = value
    q, o, lse = run_attention(F, p, heads)
    if math.isnan(value):
        assert bool(torch.isnan(o).any())
    compare(p, q, heads, o, lse)
