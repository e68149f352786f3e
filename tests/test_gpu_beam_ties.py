"""Beam search's step: what a row's sum depends on, and how exact it is (GPU only)."""
import math

import numpy as np
import pytest
import torch

from tests._beam import DTYPES, INF, Searches, begin, check_step, device_state, step64
from tests._gpu import flglm, need_gpu
from tests.test_gpu_beam import logits, row_stride, under_way, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


def stepped(F, state, x, S, B, V, dtype, **kw):
    run = Searches(F, S, B, V, 40, **kw)
    now = device_state(state)
    out = {k: torch.full_like(v, -7) for k, v in now.items()}
    run.step(now, out, x, dtype, x.shape[1])
    assert int(run.status.item()) == 0
    return out, run.tokens.cpu().numpy(), run.parents.cpu().numpy()


@pytest.mark.parametrize("S,B,V,dtype", [(64, 16, 130528, "bf16"), (61, 16, 130528, "f16"), (32, 4, 130528, "f32"), (2, 16, 130528, "f32"),
                                         (90, 7, 70001, "f32"), (5, 3, 524288, "f32"), (3, 16, 400000, "bf16")])
@pytest.mark.parametrize("resting", [0, 1, 0.4])
def test_beams_that_say_the_same_go_by_their_index(F, S, B, V, dtype, resting):
    """Beams of one search have the same logits and scores; wherever their rows are cut, the lower beam comes first."""
    gen = torch.Generator(device="cuda").manual_seed(V)
    x = torch.empty((S, B, row_stride(V, dtype)), dtype=DTYPES[dtype], device="cuda")
    x.copy_(3 * torch.randn((S, 1, x.shape[2]), generator=gen, device="cuda"))
    x[:, :, 77] = 26.0
    st = begin(S, B)
    st["scores"][:], st["steps"][:] = -1.5, 3
    rest = np.arange(S) % 5 < 2 if resting == 0.4 else np.arange(S) == S // 2 if resting else np.zeros(S, bool)
    st["done"][rest] = 1
    out, tokens, parents = stepped(F, st, x.view(S * B, -1), S, B, V, dtype)
    assert (tokens[~rest] == 77).all()
    assert np.array_equal(parents[~rest], (np.arange(S)[:, None] * B + np.arange(B))[~rest])
    scores = out["scores"].cpu().numpy()[~rest]
    assert (scores == scores[:, :1]).all()


@pytest.mark.parametrize("S,B,V,dtype", [(64, 16, 130528, "bf16"), (40, 4, 130528, "f32"), (7, 5, 1003, "f16"), (400, 2, 9000, "f32"),
                                         (3, 3, 524288, "f32")])
def test_a_search_does_not_depend_on_the_others(F, S, B, V, dtype):
    """The same bits for a search by itself, among others, and where others are over."""
    rng = np.random.default_rng(V)
    st = under_way(rng, S, B, 40)
    x = torch.randn((S * B, row_stride(V, dtype)), generator=torch.Generator(device="cuda").manual_seed(S), device="cuda").mul_(3).to(DTYPES[dtype])
    full, tokens, parents = stepped(F, st, x, S, B, V, dtype, eos=5)
    some = {k: v.copy() for k, v in st.items()}
    over = rng.random(S) < 0.5
    some["done"][over] = 1
    part, t, p = stepped(F, some, x, S, B, V, dtype, eos=5)
    assert np.array_equal(t[~over], tokens[~over]) and np.array_equal(p[~over], parents[~over])
    for k in full:
        assert torch.equal(full[k][torch.from_numpy(~over).cuda()], part[k][torch.from_numpy(~over).cuda()]), k
    for s in (0, S // 2, S - 1):
        one, t, p = stepped(F, {k: v[s:s + 1] for k, v in st.items()}, x[s * B:(s + 1) * B].clone(), 1, B, V, dtype, eos=5)
        assert np.array_equal(t[0], tokens[s]) and np.array_equal(np.where(p[0] < 0, -1, p[0] + s * B), parents[s])
        for k in full:
            assert torch.equal(one[k][0], full[k][s]), k


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_sums_of_few_logits_near_and_far_from_zero(F, dtype):
    """Eight logits within 4 of each other, at offsets on both sides of where the scaling changes.  Off from 64 bits by: the exponents'
    rounding, 6 (4 log2 e) units of 2^-24 times ln 2, 2.5e-7; their factor log2 e in 24 bits, 4 times 2^-25, 1.2e-7; three exponentials of
    2^-22 (a term, a warp's and a chunk's factor), 7.2e-7; eight additions and four products of 2^-24, 7.2e-7: 1.9e-6, under
    2^-19; and half an ulp of the score."""
    rng = np.random.default_rng(1)
    B, V = 4, 8
    at = [0.0, 1.0, -30.0, 100.0, -777.0, 4090.0, -4090.0, 4096.0, -4100.0, 20000.0, -60000.0]
    at += [] if dtype == "f16" else [1e6, -1e6]
    S = len(at)
    x = torch.from_numpy(rng.uniform(0, 4, (S, B, V)) + np.array(at)[:, None, None]).to(DTYPES[dtype])
    x = torch.minimum(x, x.amin(-1, keepdim=True) + 4)  # (offsets whose type has wide steps)
    dev = torch.full((S * B, row_stride(V, dtype)), math.nan, dtype=DTYPES[dtype], device="cuda")
    dev[:, :V] = x.view(S * B, V).cuda()
    st = begin(S, B)
    st["scores"][:], st["steps"][:] = -rng.uniform(0, 3, (S, B)).astype(np.float32), 3
    st["scores"] = -np.sort(-st["scores"])
    out, _, _ = stepped(F, st, dev, S, B, V, dtype)
    want, _, _, _, _ = step64(st, x.double().numpy(), 40, -1, 1.0, False)
    got = out["scores"].double().cpu().numpy()
    assert (np.abs(got - want["scores"]) <= 2.0 ** -24 * np.abs(want["scores"]) + 2.0 ** -19).all()


@pytest.mark.parametrize("S,dtype", [(1000, "f32"), (1000, "bf16")])
def test_whole_long_rows_in_one_part(F, S, dtype):
    """Rows of 2^19 tokens, more of them than CTAs: a CTA goes through a whole row, in stretches."""
    V = 1 << 19
    row = torch.randn(V, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").mul_(3).to(DTYPES[dtype])
    row[V - 5] = 26.0
    x = row.expand(S, V).contiguous()
    x[::3, 70000] = 27.0
    st = begin(S, 1)
    st["scores"][:, 0], st["steps"][:] = -np.arange(S) / 64, 3
    out, tokens, parents = stepped(F, st, x, S, 1, V, dtype, eos=9)
    for first in (0, 1):  # rows of each kind
        want, t, _, _, _ = step64({k: v[first:first + 1] for k, v in st.items()}, values(x[first:first + 1], 1, 1, V), 40, 9, 1.0, False)
        mine = np.arange(S)[(np.arange(S) % 3 == 0) == (first == 0)]
        assert (tokens[mine, 0] == t[0, 0]).all() and np.array_equal(parents[mine, 0], mine)
        c = want["scores"][0, 0] - st["scores"][first, 0] + st["scores"][mine, 0]
        assert (np.abs(out["scores"].double().cpu().numpy()[mine, 0] - c) <= 2.0 ** -23.9 * np.abs(c) + 2.0 ** -17).all()


@pytest.mark.parametrize("S,B,V,dtype", [(2, 3, 524288, "f32"), (300, 2, 140000, "f32"), (150, 4, 300000, "bf16")])
def test_rows_of_more_than_a_stretch(F, S, B, V, dtype):
    rng = np.random.default_rng(S)
    x = torch.randn((S * B, row_stride(V, dtype)), generator=torch.Generator(device="cuda").manual_seed(S), device="cuda").mul_(3).to(DTYPES[dtype])
    up = torch.linspace(-30, 30, V, device="cuda").to(x.dtype)
    x[0, :V], x[B, :V] = up, -2.5
    st = under_way(rng, S, B, 40)
    st["done"][S // 3::7] = 1
    out, tokens, parents = stepped(F, st, x, S, B, V, dtype, eos=V - 1)
    some = np.r_[0:2, S // 3:S // 3 + 2, S - 1] if S > 2 else np.arange(S)
    pick = torch.from_numpy(some).cuda()
    part = x.view(S, B, -1)[pick].view(len(some) * B, -1)
    want, t, p, _, _ = step64({k: v[some] for k, v in st.items()}, values(part, len(some), B, V), 40, V - 1, 1.0, False)
    rows = torch.from_numpy(parents[some] - np.where(parents[some] >= 0, (some - np.arange(len(some)))[:, None] * B, 0))
    check_step({k: v[pick] for k, v in out.items()}, torch.from_numpy(tokens[some]), rows, want, t, p)
    assert INF not in out["scores"]
