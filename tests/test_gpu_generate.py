"""Answering token by token against the training forward over whole sequences (GPU only): the same
blocks, the same tokens, in whatever chunks they come."""

import pytest
import torch

from tests._gpu import flglm, need_gpu, rel_inf

pytestmark = pytest.mark.gpu
TOL = 2e-2  # the server's outputs against the oracle's: bf16 activations over the blocks


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


def server(F, blocks, heads, head_dim, tokens, prefix=0):
    cfg = F.fl_server_cfg()
    F.lib().fl_server_cfg_default(cfg)
    cfg.n_blocks, cfg.hidden, cfg.n_heads, cfg.head_dim = blocks, heads * head_dim, heads, head_dim
    cfg.ffn_hidden, cfg.residual_alpha, cfg.max_tokens, cfg.prefix_len = 4 * cfg.hidden, 2.0, tokens, prefix
    cfg.rotary_dim, cfg.init_std = 0, 0.05
    return F.Server(cfg, 5)


@pytest.mark.parametrize("heads,head_dim,lens,prefix,glm", [
    (4, 64, [64, 33], 0, False),
    (4, 64, [70, 5, 129], 0, True),
    (2, 128, [200, 31], 7, True),
    (4, 64, [40], 64, False),
])
def test_chunks_equal_the_whole(F, heads, head_dim, lens, prefix, glm):
    from paper_2406_14898_gb300.generate import BlockStack
    srv = server(F, 2, heads, head_dim, sum(lens), prefix)
    gen = torch.Generator(device="cuda").manual_seed(sum(lens))
    x = [torch.randn((1, n, heads * head_dim), generator=gen, device="cuda").bfloat16() for n in lens]
    want = [torch.empty_like(v) for v in x]
    ctx = [max(1, n * 2 // 3) for n in lens] if glm else [0] * len(lens)
    mask = [c // 2 for c in ctx]
    srv.forward(x, lens, want, context_lens=ctx if glm else None, mask_pos=mask if glm else None)
    stack = BlockStack.from_server(srv, len(lens), max(lens) + prefix, page_size=16)
    for s, c in enumerate(ctx):
        stack.start(s, c, mask[s])
    got = [[] for _ in lens]
    at = [0] * len(lens)
    sizes = [3, 1, 1, 20, 1, 17, 2]
    step = 0
    while any(a < n for a, n in zip(at, lens)):
        # a context comes whole; then chunks of varying sizes, some sequences idle
        new = [min(n - a, max(c - a, sizes[(step + s) % 7] if (step + s) % 5 else 0))
               for s, (a, n, c) in enumerate(zip(at, lens, ctx))]
        step += 1
        if not any(new):
            continue
        y = stack.forward(torch.cat([v[0, a:a + n] for v, a, n in zip(x, at, new)]), new).split(new)
        for s, v in enumerate(y):
            got[s].append(v)
            at[s] += new[s]
    for s in range(len(lens)):
        assert rel_inf(torch.cat(got[s]).double().cpu().numpy(), want[s][0].double().cpu().numpy()) < TOL
    srv.close()


def test_pages_are_reused_and_run_out(F):
    from paper_2406_14898_gb300.generate import BlockStack
    srv = server(F, 1, 4, 64, 64)
    stack = BlockStack.from_server(srv, 2, 64, page_size=16, n_pages=5)
    x = torch.randn((64, 256), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    first = stack.forward(x[:40], [40, 0])          # three pages
    stack.forward(x[:20], [0, 20])                  # two
    with pytest.raises(MemoryError):
        stack.forward(x[:9], [9, 0])
    stack.pages.lens[0] = 40
    stack.start(1)
    stack.start(0)
    assert torch.equal(stack.forward(torch.cat([x[:40], x[:1]]), [40, 1])[:40], first)
    with pytest.raises(ValueError):
        stack.forward(x[:64], [0, 64])
    srv.close()


def test_clients_answer(F):
    """The command; a client's answer does not depend on the others that answer with it."""
    from paper_2406_14898_gb300 import generate
    together = generate.main(["--tokens", "6", "--prompts", "40", "9", "130"])
    assert [len(a) for a in together] == [6, 6, 6]
    assert all(0 <= t < 1000 for a in together for t in a)
