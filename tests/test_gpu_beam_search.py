"""Answers kept under way side by side (GPU only): stacks whose sequences follow one another and share pages, and the whole
beam search over them, against sequences that are computed alone."""
import itertools
import math
import random

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


@pytest.mark.parametrize("prefix,glm,page", [(0, False, 16), (0, True, 16), (7, True, 16), (5, False, 64)])
def test_sequences_that_follow_one_another(F, prefix, glm, page):
    """Two prompts, four sequences each, parents at random, sequences that end and begin anew: every output as that of the same
    tokens in a sequence of its own."""
    from paper_2406_14898_gb300.generate import BlockStack
    rng = random.Random(prefix + page)
    srv = server(F, 2, 4, 64, 128, prefix)
    gen = torch.Generator(device="cuda").manual_seed(3)
    row = lambda: torch.randn((1, 256), generator=gen, device="cuda").bfloat16()  # noqa: E731
    stack = BlockStack.from_server(srv, 2, 100, page_size=page).with_sequences(8)
    prompts = {0: torch.cat([row() for _ in range(37)]), 4: torch.cat([row() for _ in range(16)])}
    for s in range(8):
        p = prompts[s // 4 * 4]
        stack.start(s, len(p) if glm else 0, len(p) // 3 if glm else None)
    stack.forward(torch.cat([prompts[0], prompts[4]]), [37, 0, 0, 0, 16, 0, 0, 0])
    tokens = [[prompts[s]] if s in prompts else [] for s in range(8)]
    for t in range(20):
        parents = [s // 4 * 4 + (rng.randrange(4) if t else 0) for s in range(8)]
        if t > 8:
            parents[5] = -1 if t % 5 == 0 else parents[5]
        x = [row() for _ in range(8)]
        y = stack.follow(torch.cat(x), torch.tensor(parents, dtype=torch.int32, device="cuda"))
        tokens = [(tokens[p] if p >= 0 else None) for p in parents]
        tokens = [None if h is None else h + [v] for h, v in zip(tokens, x)]  # (what began anew has neither prompt nor prefix)
        for s in range(8):
            if tokens[s] is None:
                continue
            if t % 6 == 5 or t == 19:
                whole = torch.cat(tokens[s])
                alone = BlockStack.from_server(srv, 1, 100, page_size=16)
                c = len(prompts[s // 4 * 4])
                alone.start(0, c if glm else 0, c // 3 if glm else None)
                want = alone.forward(whole, [len(whole)])[-1:]
                assert rel_inf(y[s:s + 1].double().cpu().numpy(), want.double().cpu().numpy()) < TOL
    refs, table = (stack.shared.sides[0][k].cpu() for k in ("refs", "table"))
    assert torch.equal(refs.long(), torch.bincount(table[table >= 0].long(), minlength=len(refs)))
    assert page > 37 + prefix or any(n > 1 for n in refs.tolist())  # a prompt's whole pages are shared, where it has one
    for call in (lambda: stack.forward(row(), [1] + [0] * 7), lambda: stack.start(0)):
        with pytest.raises(ValueError):
            call()
    srv.close()


def test_follow_refuses_what_does_not_fit(F):
    from paper_2406_14898_gb300.generate import BlockStack
    srv = server(F, 1, 4, 64, 32)
    stack = BlockStack.from_server(srv, 3, 32, page_size=16)
    x = torch.zeros((3, 256), dtype=torch.bfloat16, device="cuda")
    parents = torch.zeros(3, dtype=torch.int32, device="cuda")
    for bad_x, bad_p in ((x[:2], parents), (x.cpu(), parents), (x, parents[:2]), (x, parents.long()), (x, parents.cpu())):
        with pytest.raises(ValueError):
            stack.follow(bad_x, bad_p)
    assert stack.shared is None  # none of them has begun to share
    for _ in range(32):
        stack.follow(x, parents)
    with pytest.raises(RuntimeError):  # longer than its row
        stack.follow(x, parents)
    srv.close()


def test_stack_of_more_blocks_than_a_call_copies(F):
    """66 blocks, a prompt's last page copied in each of them, bit by bit."""
    from paper_2406_14898_gb300.generate import BlockStack
    blocks = F.FL_KV_MAX_CACHES + 2
    srv = server(F, blocks, 4, 64, 32)
    gen = torch.Generator(device="cuda").manual_seed(6)
    row = lambda n: torch.randn((n, 256), generator=gen, device="cuda").bfloat16()  # noqa: E731
    stack = BlockStack.from_server(srv, 3, 32, page_size=16)
    prompt = row(21)
    stack.forward(prompt, [21, 0, 0])
    stack.follow(row(3), torch.zeros(3, dtype=torch.int32, device="cuda"))
    for kv in (b["kv"] for b in stack.blocks):
        for a in kv:
            pages = stack.shared.sides[0]["table"][:, 1].long()
            assert len(set(pages.tolist())) == 3 and all(torch.equal(a[p, :, :5], a[pages[0], :, :5]) for p in pages)
    srv.close()


def generator(F, n, vocab, tokens, hidden=256, blocks=2):
    from paper_2406_14898_gb300.generate import Generator
    cfg, cc = F.fl_server_cfg(), F.fl_client_cfg()
    F.lib().fl_server_cfg_default(cfg)
    cfg.n_blocks, cfg.hidden, cfg.head_dim, cfg.n_heads = blocks, hidden, 64, hidden // 64
    cfg.rotary_dim, cfg.ffn_hidden, cfg.max_tokens, cfg.init_std = 0, 4 * hidden, tokens, 0.08
    cfg.residual_alpha = (2.0 * (blocks + 2)) ** 0.5
    F.lib().fl_client_cfg_default(cc)
    cc.block, cc.vocab = cfg, vocab
    cc.block.n_blocks = 1
    return Generator([F.Client(cc, 11) for _ in range(n)], F.Server(cfg, 10), tokens)


def scored(g, prompts, answers):
    """Summed log-probabilities of the answers, the clients' side by side, each with its prompt in a sequence of its own; and what they
    may be off by: the logits by TOL of the largest, so each of the tokens' log-probabilities by twice that."""
    g.start([len(p) for p in prompts])
    z = [torch.log_softmax(v.double(), -1) for v in g.logits(prompts)]
    tol = [2 * TOL * float(v.abs().max()) for v in z]
    sums, off = [0.0] * len(prompts), [0.0] * len(prompts)
    longest = max(len(a) for a in answers)
    for t in range(longest):
        step = [a[min(t, len(a) - 1)] for a in answers]
        for k, (a, w) in enumerate(zip(answers, step)):
            if t < len(a):
                sums[k] += float(z[k][w])
                off[k] += tol[k]
        if t + 1 < longest:
            z = [torch.log_softmax(v.double(), -1) for v in g.logits([torch.tensor([w], dtype=torch.int32, device="cuda") for w in step])]
    return sums, off


@pytest.mark.parametrize("beams,eos,penalty,early", [(1, -1, 1.0, False), (4, -1, 0.0, False), (5, 7, 1.0, False), (16, 3, 0.6, True)])
def test_answers_score_what_they_say(F, beams, eos, penalty, early):
    g = generator(F, 3, 50, 64)
    gen = torch.Generator().manual_seed(1)
    prompts = [torch.randint(50, (n,), generator=gen, dtype=torch.int32).cuda() for n in (20, 3, 33)]
    found = g.beam_search(prompts, 12, beams, eos, penalty, early)
    assert [len(x) for x in found] == [beams] * 3
    for best in found:
        assert [x for _, x in best] == sorted((x for _, x in best), reverse=True)
        assert len({tuple(t) for t, _ in best}) == beams
        assert all(eos < 0 or eos not in t[:-1] for t, _ in best)
    for i in {0, beams // 2, beams - 1}:
        sums, off = scored(g, prompts, [best[i][0] for best in found])
        for (tokens, x), c, d in zip((best[i] for best in found), sums, off):
            assert abs(x * len(tokens) ** penalty - c) <= d
    if beams == 1:
        g.start([len(p) for p in prompts])
        assert [best[0][0] for best in found] == g.greedy(prompts, 12)


def test_enough_beams_find_the_best_of_all(F):
    """Four tokens and sixteen beams: no answer of three tokens is missed; the same on another stream."""
    g = generator(F, 1, 4, 32)
    prompt = [torch.tensor([1, 0, 3, 2, 2], dtype=torch.int32, device="cuda")]
    found = g.beam_search(prompt, 3, 16, length_penalty=0.0)[0]
    every = {}
    for a in itertools.product(range(4), repeat=3):
        sums, off = scored(g, prompt, [list(a)])
        every[a] = sums[0], off[0]
    for tokens, x in found:
        assert abs(x - every[tuple(tokens)][0]) <= every[tuple(tokens)][1]
    worst = found[-1][1]
    for a, (c, d) in every.items():
        if a not in {tuple(t) for t, _ in found}:
            assert c <= worst + 2 * d
    assert math.isclose(sum(math.exp(c) for c, _ in every.values()), 1.0, rel_tol=0.3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = g.beam_search(prompt, 3, 16, length_penalty=0.0)[0]
    assert again == found


def test_refusals(F):
    g = generator(F, 2, 20, 32)
    good = [torch.tensor([1, 2], dtype=torch.int32, device="cuda")] * 2
    for prompts, count, beams in ((good[:1], 4, 2), (good, 0, 2), (good, 4, 0), (good, 4, 17), (good, 32, 2), ([good[0], good[0].long()], 4, 2),
                                  ([good[0], good[0][:0]], 4, 2)):
        with pytest.raises(ValueError):
            g.beam_search(prompts, count, beams)
    with pytest.raises(F.FlError):
        g.beam_search(good, 4, 2, eos=20)
    assert len(g.beam_search(good, 31, 2)[0]) == 2
    assert [len(a) for a in g.greedy(good, 3)] == [3, 3]


def test_command(F):
    from paper_2406_14898_gb300 import generate
    found = generate.main(["--tokens", "5", "--prompts", "40", "9", "--beams", "3", "--eos", "4"])
    assert [len(x) for x in found] == [3, 3] and all(1 <= len(t) <= 5 for best in found for t, _ in best)
