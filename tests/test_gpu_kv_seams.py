"""Every key with its own value, at every seam (GPU only).  Scores are whole numbers of log2 and values small whole
numbers, so that weights are powers of two, exact in 16 bits, and sums are exact in 32: what is left is the
rounding of the output, which no key that takes another one's value, weight or place stays below, however
long the cache."""
import math

import pytest
import torch

from tests._gpu import flglm, need_gpu
from tests._kv import UNIT, Paged, attention64
from tests.test_gpu_kv import run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


CASES = [
    # new, lens, heads, kv heads, head_dim, page, token-major, context
    ([1], [1031], 4, 4, 128, 16, False, None),
    ([1, 1, 1], [5000, 1500, 64], 4, 2, 64, 64, True, None),
    ([2, 8], [4097, 129], 2, 1, 128, 32, False, None),
    ([1], [20011], 4, 1, 128, 256, False, None),
    ([1, 3], [3000, 1031], 15, 3, 64, 128, False, None),
    ([40], [1500], 2, 2, 128, 64, False, None),
    ([300, 1, 17], [5000, 777, 1031], 4, 2, 128, 32, True, None),
    ([257], [257], 2, 2, 64, 16, False, [201]),
    ([130, 33], [2049, 4000], 8, 2, 64, 256, False, None),
    ([64] * 40, [64 + 9 * i for i in range(40)], 4, 4, 128, 16, False, [40] * 40),
    ([3, 5], [900, 1290], 48, 4, 128, 128, False, None),
]


def exact_inputs(p, heads):
    """Keys of score 0 to 3 (log2), values of -8 to 8."""
    for c in (p.k, p.v):
        finite = torch.isfinite(c[..., :1]).expand_as(c)
        c.copy_(torch.where(finite, torch.randint(-8, 9, c.shape, generator=p.gen, device="cuda").to(c.dtype), c))
    p.k[..., 0] = torch.where(torch.isfinite(p.k[..., 0]), p.k[..., 0].abs().remainder(4), p.k[..., 0])
    q = torch.zeros((p.T, heads, p.hd), dtype=p.k.dtype, device="cuda")
    q[..., 0] = 1
    return q


def bound(p, ref):
    """Half an ulp of the output; 2^-17 of it for the sum of the weights, which is taken before they are rounded
    (an exponential's 2^-22, a scale of one but for 2^-23, sums of at most 2^15 terms in 32 bits), and 2^-19 of
    sum p |v| for O where the reference of its exponents moved (a factor off by 2^-21, a few times)."""
    ro, _, size = ref
    return UNIT[p.dtype] * (1 + 2.0 ** -6) * ro.abs() + 2.0 ** -17 * ro.abs() + 2.0 ** -19 * size


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_each_key_has_its_own_value(F, case, dtype):
    new, lens, heads, kvh, hd, page, token_major, context = case
    p = Paged(F, new, lens, kvh, hd, page, dtype, token_major, seed=len(lens) + heads)
    q, o, lse = run_attention(F, p, heads, context, scale=math.log(2.0), q=exact_inputs(p, heads))
    ref = attention64(p, q, heads, context, scale=math.log(2.0))
    worst = ((o.double() - ref[0]).abs() / (bound(p, ref) + 1e-30)).amax()
    assert float(worst) <= 1, float(worst)
    assert bool(((lse.double() - ref[1]).abs() <= 2.0 ** -16 * (1 + ref[1].abs())).all()) and p.status.item() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_the_bound_sees_a_neighbours_value(F, dtype):
    """The definition with one key's value in place of its neighbour's is out of the bound at every length used."""
    for L in (1031, 5000, 20011):
        p = Paged(F, [1], [L], 1, 64, 64, dtype, seed=L)
        q = exact_inputs(p, 1)
        ref = attention64(p, q, 1, scale=math.log(2.0))
        u = L // 2 | 1
        at, of = ((int(p.table[0, x // 64]), x % 64) for x in (u, u - 1))
        p.v[at] = p.v[of]
        other = attention64(p, q, 1, scale=math.log(2.0))[0]
        assert bool(((other - ref[0]).abs() > 2 * bound(p, ref)).any())
