"""Attention over the paged cache where scores are huge, against the definition in 64 bits (GPU only)."""
import pytest
import torch

from tests._gpu import flglm, need_gpu
from tests._kv import DTYPES, Paged, check_attention
from tests.test_gpu_kv import run_attention
from tests.test_gpu_kv_nonfinite import CASES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


def softmax64(p, q, heads, scale):
    """(o, lse, sum p |v|), the maximum taken off first: a log-sum-exp of 2^80 has no bits left for the number
    of keys that share it."""
    group = heads // p.kv_heads
    o = torch.zeros((p.T, heads, p.hd), dtype=torch.float64, device="cuda")
    size, lse = torch.zeros_like(o), torch.zeros((heads, p.T), dtype=torch.float64, device="cuda")
    for s, (n, L) in enumerate(zip(p.new, p.lens)):
        k, v, t0 = p.rows(s, "k"), p.rows(s, "v"), int(p.cu_host[s])
        hidden = torch.arange(L, device="cuda")[None, :] > torch.arange(L - n, L, device="cuda")[:, None]
        for h in range(heads):
            sc = q[t0:t0 + n, h].double() @ k[:, h // group].T * scale
            sc.masked_fill_(hidden, -float("inf"))
            w = torch.softmax(sc, -1)
            o[t0:t0 + n, h], size[t0:t0 + n, h] = w @ v[:, h // group], w @ v[:, h // group].abs()
            lse[h, t0:t0 + n] = torch.logsumexp(sc, -1)
    return o, lse, size


@pytest.mark.parametrize("dtype,big", [("f16", 2.0 ** 14), ("f16", 2.0 ** 9), ("bf16", 2.0 ** 14), ("bf16", 2.0 ** 40)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("case", CASES)
def test_huge_scores(F, case, dtype, big, sign):
    """Scores of up to 2^80 in steps of 2^21 or more, exact in 32 bits until they are scaled: the keys of the
    highest level that a row sees share its weight equally, and what a scaled score is rounded by is no weight."""
    new, lens, heads, kvh, hd, page = CASES[case]
    p = Paged(F, new, lens, kvh, hd, page, dtype, seed=47)
    turn = torch.where(torch.rand(hd, generator=p.gen, device="cuda") < 0.5, -1.0, 1.0)
    for s, L in enumerate(lens):
        level = torch.randint(1, 8, (L,), generator=p.gen, device="cuda")
        level[L - 1] = 8  # the newest token's: the last row's alone
        for i in range(-(-L // page)):
            n = min(page, L - i * page)
            rows = sign * big * 2.0 ** -3 * level[i * page:i * page + n, None, None] * turn
            p.k[int(p.table[s, i]), :n] = rows.to(DTYPES[dtype]).expand(n, kvh, hd)
    q = (big * turn).to(DTYPES[dtype]).expand(p.T, heads, hd).contiguous()
    _, o, lse = run_attention(F, p, heads, q=q)
    check_attention(p, o, lse, softmax64(p, q, heads, hd ** -0.5))
    assert p.status.item() == 0
