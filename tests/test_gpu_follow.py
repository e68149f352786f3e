"""What a sequence takes over from the one that it follows, in stacks that share pages (GPU only)."""
import random

import pytest
import torch

from tests._gpu import flglm, need_gpu, rel_inf
from tests.test_gpu_beam_search import TOL, server

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


def rows(gen, n, width=256):
    return torch.randn((n, width), generator=gen, device="cuda").bfloat16()


def alone(stack_of, tokens, context, mask):
    """The last output of the tokens in a sequence of its own."""
    one = stack_of()
    one.start(0, context, mask)
    return one.forward(tokens, [len(tokens)])[-1:]


@pytest.mark.parametrize("prefix", [0, 5])
def test_context_and_mask_come_from_the_parent(F, prefix):
    """Four sequences: two contexts of different lengths and masks, none, and one that is never more than started; all follow one
    another at random, whichever place they are in."""
    from paper_2406_14898_gb300.generate import BlockStack
    rng = random.Random(prefix)
    srv = server(F, 2, 4, 64, 128, prefix)
    gen = torch.Generator(device="cuda").manual_seed(8)
    stack = BlockStack.from_server(srv, 4, 100, page_size=16)
    given = [(20, 5, 20), (12, None, 17), (0, None, 9), (0, None, 0)]  # context, mask, tokens at first
    x = rows(gen, sum(n for _, _, n in given))
    for s, (c, m, _) in enumerate(given):
        stack.start(s, c, m)
    stack.forward(x, [n for _, _, n in given])
    have = [(c, m, t) for (c, m, _), t in zip(given, x.split([n for _, _, n in given]))]
    for t in range(9):
        parents = [0, 0, 1, 2] if t == 0 else [2, 2, 0, 3] if t == 1 else [rng.randrange(4) for _ in range(4)]
        x = rows(gen, 4)
        y = stack.follow(x, torch.tensor(parents, dtype=torch.int32, device="cuda"))
        have = [(have[p][0], have[p][1], torch.cat([have[p][2], x[s:s + 1]])) for s, p in enumerate(parents)]
        for s, (c, m, tokens) in enumerate(have):
            want = alone(lambda: BlockStack.from_server(srv, 1, 100, page_size=16), tokens, c, m)
            assert rel_inf(y[s:s + 1].double().cpu().numpy(), want.double().cpu().numpy()) < TOL, (t, s)
    srv.close()


@pytest.mark.parametrize("glm", [False, True])
def test_a_sequence_that_begins_anew_has_no_prefix(F, glm):
    """Parent -1 in a stack with a prefix: what it says is that of the same blocks without a prefix, from position 0 on."""
    from paper_2406_14898_gb300.generate import BlockStack
    srv, bare = server(F, 2, 4, 64, 64, 7), server(F, 2, 4, 64, 64)
    for b in range(2):
        for t in range(12):
            bare.set_param(b, t, srv.get_param(b, t))
    gen = torch.Generator(device="cuda").manual_seed(9)
    stack = BlockStack.from_server(srv, 3, 60, page_size=16)
    for s in range(2):  # the third is not even started
        stack.start(s, 11 if glm else 0)
    prompt = rows(gen, 11)
    stack.forward(prompt, [11, 0, 0])
    have = {0: (srv, 11 if glm else 0, prompt)}
    parents = [[0, -1, 2], [0, 1, 2], [1, -1, 0], [0, 1, 1]] + [[s, s, s] for s in (0, 1)] + [[0, 1, 2]] * 12
    for t, p in enumerate(parents):
        x = rows(gen, 3)
        y = stack.follow(x, torch.tensor(p, dtype=torch.int32, device="cuda"))
        have = {s: have.get(q, (bare, 0, prompt[:0])) for s, q in enumerate(p)}
        have = {s: (w, c, torch.cat([v, x[s:s + 1]])) for s, (w, c, v) in have.items()}
        for s, (w, c, tokens) in have.items():
            want = alone(lambda: BlockStack.from_server(w, 1, 60, page_size=16), tokens, c, None)
            assert rel_inf(y[s:s + 1].double().cpu().numpy(), want.double().cpu().numpy()) < TOL, (t, s)
    srv.close()
    bare.close()


def test_a_context_that_is_not_there_yet_is_not_followed(F):
    """As in a call of its own: a context's tokens come together, so none of them follows a sequence that has not got them."""
    from paper_2406_14898_gb300.generate import BlockStack
    srv = server(F, 1, 4, 64, 64)
    gen = torch.Generator(device="cuda").manual_seed(2)

    def stack():
        st = BlockStack.from_server(srv, 2, 60, page_size=16)
        for s in range(2):
            st.start(s, 9)
        st.forward(rows(gen, 9), [9, 0])
        return st

    good, bad = stack(), stack()
    good.follow(rows(gen, 2), torch.tensor([0, -1], dtype=torch.int32, device="cuda"))
    good.follow(rows(gen, 2), torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    with pytest.raises(RuntimeError):
        bad.follow(rows(gen, 2), torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    srv.close()
