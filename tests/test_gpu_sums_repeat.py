"""Sums over the tokens that are the same bits in every call (GPU only)."""
import pytest
import torch

import synthetic as syn
from tests._gpu import flglm, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


@pytest.mark.parametrize("T,H,dtype", [(1, 256, "f32"), (63, 512, "bf16"), (377, 1024, "f32"), (2000, 4096, "f32"), (304, 256, "bf16")])
def test_layernorm_gradients(F, T, H, dtype):
    """Against 64 bits, and the same in every call.  A sum of T products of size 1 to 4 is off by less than (T + 16) roundings of
    2^-24 of the sum of their sizes."""
    gen = torch.Generator(device="cuda").manual_seed(T + H)
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    dy, x = (torch.randn((T, H), generator=gen, device="cuda").to(kind) for _ in "dx")
    gamma = torch.randn(H, generator=gen, device="cuda")
    mean, rstd = x.float().mean(1), (x.float().var(1, unbiased=False) + 1e-5).rsqrt()
    ws = torch.empty(F.fl_k_layernorm_bwd_workspace(T, H) // 4, device="cuda")
    first = None
    for _ in range(30):
        dx, dg, db = torch.empty((T, H), dtype=torch.bfloat16, device="cuda"), torch.zeros(H, device="cuda"), torch.zeros(H, device="cuda")
        F.fl_k_layernorm_bwd(T, H, dy, x, mean, rstd, gamma, None, 0.0, dx, dg, db, ws, io_dtype=F.FL_DT_F32 if dtype == "f32" else F.FL_DT_BF16)
        first = first or (dx, dg, db)
        assert all(torch.equal(a, b) for a, b in zip((dx, dg, db), first))
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    for got, terms in ((first[1], dy.double() * xh), (first[2], dy.double())):
        assert ((got.double() - terms.sum(0)).abs() <= (T + 16) * 2.0 ** -24 * terms.abs().sum(0)).all()


def two_servers(F, steps):
    from tests.test_gpu_server import make_server
    cfg = syn.CONFIGS["tiny"].with_(hidden=1024, n_heads=16, ffn_hidden=4096, client_batch=1, seq_lens=(300, 77))
    gen = torch.Generator(device="cuda").manual_seed(5)
    states = [torch.randn((1, n, 1024), generator=gen, device="cuda").bfloat16() for n in cfg.seq_lens]
    grads = [(1e-3 * torch.randn((1, n, 1024), generator=gen, device="cuda")).bfloat16() for n in cfg.seq_lens]
    both = [make_server(F, cfg) for _ in "ab"]
    for srv in both:
        for _ in range(steps):
            outs, gi = [torch.empty_like(x) for x in states], [torch.empty_like(x) for x in states]
            srv.forward(states, cfg.seq_lens, outs)
            srv.backward_step(grads, gi, 1e-3)
        srv.sync()
    return both


def test_layernorms_of_two_servers(F):
    """After a step the gains and offsets of two handles that did the same are equal to the bit: a gain that is off by an ulp turns
    bf16 roundings of the next forward."""
    for _ in range(12):
        a, b = two_servers(F, 1)
        for t in (F.FL_T_LN1_G, F.FL_T_LN1_B, F.FL_T_LN2_G, F.FL_T_LN2_B, F.FL_T_BDENSE):
            assert (a.get_param(0, t) == b.get_param(0, t)).all(), t
        a.close()
        b.close()
