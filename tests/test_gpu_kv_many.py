"""Forks of so many sequences that the CTAs of the plan have some each, and hand pages out in several goes (GPU only)."""
import random

import pytest
import torch

from tests._beam import Pool
from tests._gpu import flglm, need_gpu
from tests.test_gpu_kv_pages import step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


@pytest.mark.parametrize("S,W", [(7168, 2), (7169, 2), (8192, 3), (8193, 3), (20000, 2)])
def test_many_sequences(F, S, W):
    """From sequences of their own over shared ones (parents near by and far) to chunks, tokens taken off and sequences that leave."""
    rng = random.Random(S)
    page, n_pages = 16, 4 * S
    pool = Pool(F, S, n_pages, page, W, 1, 1, 64)
    order = rng.sample(range(n_pages), S * W)
    lens = [rng.choice([0, 5, 16, 17, rng.randrange(W * page + 1)]) for _ in range(S)]
    table = [order[s * W:s * W + -(-x // page)] for s, x in enumerate(lens)]
    refs = [0] * n_pages
    for row in table:
        for q in row:
            refs[q] += 1
    for q in rng.sample([q for row in table for q in row], S // 20):  # kept by others
        refs[q] += 1
    pool.set(lens, [row + [-1] * (W - len(row)) for row in table], refs)
    side, copies = 0, 0
    for t in range(4):
        near = [s // 4 * 4 + rng.randrange(4) for s in range(S)]
        parents = [rng.choice([s, s, min(near[s], S - 1), rng.randrange(S), -1 if t else s]) for s in range(S)]
        lens = pool.get(side)[0]
        before = [lens[p] if p >= 0 else 0 for p in parents]
        new = [min(W * page - x, rng.choice([0, 1, 1, 1, 3, -7, 16])) for x in before]
        copies += len(step(pool, parents, new, side)[3])
        side = 1 - side
    assert copies > S // 10


@pytest.mark.parametrize("S", [7169, 9000])
def test_many_sequences_that_find_no_room(F, S):
    """One page short, and one sequence in the last CTA's part that outgrows its row or has no such parent: nothing changes."""
    page = 16
    pool = Pool(F, S, S + 10, page, 2, 1, 1, 64)
    state = [[16] * S, [[s, -1] for s in range(S)], [1] * S + [0] * 10]
    for parents, new, bits in ((None, [1] * 11 + [0] * (S - 11), F.FL_KV_NO_ROOM), (None, [0] * (S - 1) + [17], F.FL_KV_NO_ROOM),
                               (list(range(S - 1)) + [S], None, F.FL_KV_BAD_PARENT)):
        pool.set(*state)
        before = pool.bits()
        pool.status.zero_()
        pool.fork(parents, new)
        assert int(pool.status.item()) == bits and pool.get(1) == state
        assert all(torch.equal(a, b) for a, b in zip(before, pool.bits()))
        assert not pool.workspace[:3 * (-(-(S + 10) // 4) * 4)].any()
    pool.status.zero_()
    step(pool, None, [1] * 10 + [0] * (S - 10), 0)  # as many as there are
