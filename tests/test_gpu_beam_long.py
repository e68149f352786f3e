"""Traces of more steps than a cluster takes at a time (GPU only)."""
import numpy as np
import pytest
import torch

from tests._beam import INF, Searches, begin, device_state, trace64
from tests._gpu import flglm, need_gpu

pytestmark = pytest.mark.gpu
ROW = 8 * 2048  # steps of a cluster at a time


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


@pytest.mark.parametrize("T,B,n", [(ROW - 1, 3, 3), (ROW, 3, 3), (ROW + 1, 4, 4), (2 * ROW, 2, 1), (33000, 4, 3), (2 * ROW + 1, 16, 16)])
def test_hypotheses_that_end_around_the_border(F, T, B, n):
    """One search is over, one goes on at its last step, one in between: hypotheses of a few steps, of all, and of those next to
    where a cluster begins anew."""
    rng = np.random.default_rng(T)
    S = 3
    st = begin(S, B)
    st["scores"] = -np.cumsum(rng.uniform(0.5, 3, (S, B)).astype(np.float32), 1, dtype=np.float32).astype(np.float64)
    st["steps"], st["done"] = np.array([T, T, min(T, ROW + 1)]), np.array([1, 0, 0])
    ends = [x for x in (ROW - 1, ROW, ROW - 2, 5, T - 1, 2 * ROW, 2 * ROW - 1, 0, ROW + 1, 2047, 2048) if x < T]
    for s, some in ((0, B), (1, B // 2), (2, B // 2)):
        st["end_scores"][s, :some] = -np.sort(rng.uniform(0.01, 4, some).astype(np.float32))
        st["end_steps"][s, :some] = [min(ends[(s + i) % len(ends)], st["steps"][s] - 1) for i in range(some)]
        st["end_beams"][s, :some] = rng.integers(0, B, some)
    tokens, parents = rng.integers(0, 50, (S, T, B)), rng.integers(0, B, (S, T, B))
    run = Searches(F, S, B, 50, T, 2, 0.5)
    run.trace_tokens.copy_(torch.from_numpy(tokens))
    run.trace_parents.copy_(torch.from_numpy(parents))
    got = run.trace(device_state(st), n, pad=-3)
    out, lens, scores = trace64(st, tokens, parents, n, -3, 2, 0.5)
    assert np.array_equal(got[0].cpu().numpy(), out) and np.array_equal(got[1].cpu().numpy(), lens)
    fine = scores > -INF
    # n^0.5 within 2^-25, a division and a rounding of 2^-24 each
    assert (np.abs(got[2].double().cpu().numpy()[fine] - scores[fine]) <= 2.0 ** -22 * np.abs(scores[fine])).all()
    assert int(run.status.item()) == 0


def test_indices_out_of_range_behind_the_border(F):
    S, B, T = 1, 3, ROW + 500
    st = begin(S, B)
    st["scores"][:], st["steps"][:] = -1, T
    run = Searches(F, S, B, 50, T)
    run.trace_tokens.copy_(torch.arange(T * B).view(S, T, B))
    run.trace_parents.zero_()
    for t, x in ((ROW + 100, 3), (ROW, -1), (ROW - 1, 10 ** 9)):
        run.trace_parents[0, t, 1] = x
    out, lens, _ = run.trace(device_state(st), 3)
    assert int(run.status.item()) == F.FL_BEAM_BAD_TRACE and lens.tolist() == [[T] * 3]
    assert torch.equal(out[0, :, :T - 1].cpu(), (torch.arange(T - 1, dtype=torch.int32) * B).expand(3, T - 1))
