"""What an answering stack keeps between calls: streams, refusals, contexts, roundings (GPU only)."""
import pytest
import torch

from tests._gpu import flglm, need_gpu, rel_inf
from tests._kv import UNIT, turn64
from tests.test_gpu_generate import server

pytestmark = pytest.mark.gpu
TOL = 2e-2  # bf16 activations over the blocks, as for chunks against the whole


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


def rows(n, width, seed=1):
    return torch.randn((n, width), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


def generator(F, n, vocab=200, blocks=2, room=160, which=None):
    """A split model, the same for every n: clients 0..n-1, or those of `which`."""
    from paper_2406_14898_gb300.generate import Generator
    srv = server(F, blocks, 4, 64, room)
    cc = F.fl_client_cfg()
    F.lib().fl_client_cfg_default(cc)
    cc.block, cc.vocab = srv.cfg, vocab
    cc.block.n_blocks = 1
    clients = [F.Client(cc, 100 + k) for k in (range(n) if which is None else which)]
    return Generator(clients, srv, room)


def prompt(k, n, vocab=200):
    gen = torch.Generator().manual_seed(k)
    return torch.randint(vocab, (n,), generator=gen, dtype=torch.int32).cuda()


# ------------------------------------------------------------------------------- streams

def test_every_call_goes_to_the_current_stream(F, monkeypatch):
    """The library's kernels run where torch's own work of the same call runs."""
    gen = generator(F, 2)
    torch.cuda.synchronize()
    st, seen = torch.cuda.Stream(), []
    plain = F.stream_ptr
    monkeypatch.setattr(F, "stream_ptr", lambda s: seen.append(plain(s)) or plain(s))
    with torch.cuda.stream(st):
        gen.greedy([prompt(0, 9), prompt(1, 30)], 2)
    torch.cuda.synchronize()
    assert len(seen) > 100 and set(seen) == {st.cuda_stream}


def test_a_stream_that_is_behind_gives_the_same_bits(F):
    """A stream of its own that is held up before each call: nothing of the call runs ahead of it."""
    p, more = [prompt(0, 9), prompt(1, 30)], [prompt(2, 1), prompt(3, 1)]
    outs = []
    for st in (None, torch.cuda.Stream()):
        gen = generator(F, 2)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            gen.start([len(t) for t in p])
            for t in (p, more):
                if st:
                    torch.cuda._sleep(20_000_000)
                outs.append(torch.stack(gen.logits(t)))
        torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])


# ------------------------------------------------------------------------------- refusals


def test_a_refused_call_changes_nothing(F):
    from paper_2406_14898_gb300.generate import BlockStack
    x = rows(40, 256)
    outs = []
    for refuse in (False, True):
        srv = server(F, 1, 4, 64, 64)
        stack = BlockStack.from_server(srv, 2, 64, page_size=16, n_pages=5)
        stack.forward(x[:30], [20, 10])
        if refuse:
            with pytest.raises(ValueError):
                stack.forward(rows(60, 256), [5, 55])  # the second sequence is too long
            with pytest.raises(MemoryError):
                stack.forward(rows(60, 256), [20, 40])  # it would fit, had the first not taken the pages
        outs.append(stack.forward(x[30:], [3, 7]))
        srv.close()
    assert torch.equal(*outs)


def test_a_call_that_failed_on_the_device_changes_nothing(F):
    from paper_2406_14898_gb300.generate import BlockStack
    srv = server(F, 1, 4, 64, 64)
    x = rows(40, 256)
    outs = []
    for fail in (False, True):
        stack = BlockStack.from_server(srv, 2, 64, page_size=16)
        stack.forward(x[:30], [20, 10])
        if fail:
            stack.status.fill_(F.FL_KV_TIMEOUT)  # as if a wait had given up
            stack.workspace[:64] = 1
            with pytest.raises(RuntimeError):
                stack.forward(x[30:], [3, 7])
        outs.append(stack.forward(x[30:], [3, 7]))
    assert torch.equal(*outs)
    srv.close()


def test_clients_are_not_ahead_of_a_server_that_refused(F):
    p = [prompt(0, 9), prompt(1, 30)]
    more = [prompt(2, 1), prompt(3, 1)]
    outs = []
    for refuse in (False, True):
        gen = generator(F, 2)
        gen.start([len(t) for t in p])
        gen.logits(p)
        if refuse:
            free, gen.server.pages.free = gen.server.pages.free, []
            held = gen.server.pages.lens[0]
            with pytest.raises(MemoryError):
                gen.logits([prompt(4, 100), more[1]])
            gen.server.pages.free = free
            assert gen.server.pages.lens[0] == held
        outs.append(torch.stack(gen.logits(more)))
    assert torch.equal(*outs)


def test_every_product_has_its_status_looked_at(F, monkeypatch):
    """A wait that gave up, set by the test in each product's status in turn, is an error, and nothing is added."""
    gen = generator(F, 1, blocks=1)
    plain, calls, spoiled = F.gemm, [], 0

    def gemm(*args, status=None, **kw):
        plain(*args, status=status, **kw)
        calls.append(status)
        if len(calls) == spoiled:
            status.fill_(1)

    monkeypatch.setattr(F, "gemm", gemm)
    gen.start([5])
    gen.logits([prompt(0, 5)])
    n = len(calls)
    assert n == 3 * 4 + 1
    for spoiled in range(n + 1, 2 * n + 1):
        del calls[n:]
        with pytest.raises(RuntimeError):
            gen.logits([prompt(1, 1)])
            pytest.fail(f"product {spoiled - n} of {n}")
        assert [x.pages.lens[0] for x in (gen.server, gen.bottom[0], gen.top[0])] == [5, 5, 5]


# ------------------------------------------------------------------------------- contexts

def test_a_context_in_two_calls_is_refused(F):
    """Its tokens see each other, so they come together; the answer's may come with them or later."""
    from paper_2406_14898_gb300.generate import BlockStack
    for prefix in (0, 7):
        srv = server(F, 1, 4, 64, 64, prefix)
        stack = BlockStack.from_server(srv, 2, 64, page_size=16)
        stack.start(0, 20)
        stack.start(1)
        x = rows(40, 256)
        for n in (1, 19):
            with pytest.raises(ValueError):
                stack.forward(x[:n], [n, 0])
        with pytest.raises(ValueError):
            stack.forward(x[:29], [19, 10])
        assert stack.pages.lens == [prefix, prefix]
        stack.forward(x[:10], [0, 10])  # an idle context, and one that is plainly causal
        stack.forward(x[:23], [22, 1])
        stack.forward(x[:2], [1, 1])
        srv.close()


# ------------------------------------------------------------------------------- arguments

def test_rows_in_any_strides(F):
    from paper_2406_14898_gb300.generate import BlockStack
    srv = server(F, 1, 4, 64, 64)
    stack = BlockStack.from_server(srv, 1, 64, page_size=16)
    want = stack.forward(rows(40, 256), [40])
    for x in (rows(40, 256).T.contiguous().T, torch.cat([rows(40, 256), rows(40, 256, 2)], 1)[:, :256],
              rows(40, 256).repeat_interleave(2, 0)[::2], rows(40, 256).float()):
        stack.start(0)
        assert torch.equal(stack.forward(x, [40]), want)
    srv.close()


def test_rows_that_do_not_fit_are_refused(F):
    from paper_2406_14898_gb300.generate import BlockStack
    srv = server(F, 1, 4, 64, 64)
    stack = BlockStack.from_server(srv, 2, 64, page_size=16)
    x = rows(40, 256)
    for rows_, new in ((x, [41, 0]), (x, [20, 19]), (x, [40]), (x, [20, 10, 10]), (x, [41, -1]), (x[:, :128], [40, 0]),
                       (x.view(-1), [40, 0]), (x.cpu(), [40, 0])):
        with pytest.raises(ValueError):
            stack.forward(rows_, new)
    assert stack.pages.lens == [0, 0]
    srv.close()


def test_no_new_tokens_are_no_rows(F):
    from paper_2406_14898_gb300.generate import BlockStack
    srv = server(F, 1, 4, 64, 64)
    stack = BlockStack.from_server(srv, 2, 64, page_size=16)
    x = rows(40, 256)
    outs = []
    for idle in (False, True):
        stack.start(0)
        stack.start(1)
        if idle:
            assert stack.forward(x[:0], [0, 0]).shape == (0, 256)
        outs.append(stack.forward(x, [40, 0]))
    assert torch.equal(*outs)
    srv.close()


def test_tokens_that_do_not_fit_are_refused(F):
    gen = generator(F, 2)
    gen.start([5, 5])
    a, b = prompt(0, 5), prompt(1, 5)
    for tokens in ([a], [a, b, b], [a.long(), b], [a, b.cpu()], [a, b[:0]], [a, b.view(1, 5)]):
        with pytest.raises(ValueError):
            gen.logits(tokens)
    with pytest.raises(RuntimeError):
        gen.logits([a, b + 200])  # past the vocabulary
    want = torch.stack(gen.logits([a, b]))
    gen.start([5, 5])
    assert torch.equal(torch.stack(gen.logits([a.repeat_interleave(3)[::3], b])), want)


# ------------------------------------------------------------------------------- positions

def test_a_sequence_may_fill_its_last_page(F):
    from paper_2406_14898_gb300.generate import BlockStack
    srv = server(F, 1, 4, 64, 64)
    x = rows(48, 256)
    outs = []
    for most in (48, 40):  # three pages either way
        stack = BlockStack.from_server(srv, 1, most, page_size=16)
        outs.append(torch.cat([stack.forward(x[:39], [39]), stack.forward(x[39:], [9])]))
        with pytest.raises(ValueError):
            stack.forward(x[:1], [1])
    assert torch.equal(*outs)
    srv.close()


def test_positions_that_do_not_exist_are_refused(F):
    from paper_2406_14898_gb300.generate import BlockStack
    srv = server(F, 1, 4, 64, 64, 7)
    stack = BlockStack.from_server(srv, 2, 64, page_size=16)
    x = rows(20, 256)
    with pytest.raises(ValueError):
        stack.forward(x, [20, 0])  # its prefix is not there yet
    stack.start(0, 20, 19)
    want = stack.forward(x, [20, 0])
    for context, mask in ((-1, None), (20, 20), (20, -1), (20, 2 ** 30)):
        with pytest.raises(ValueError):
            stack.start(0, context, mask)
    assert stack.pages.lens == [27, 0] and stack.context[0] == 27 and stack.mask_pos[0] == 19
    stack.start(0, 20)
    assert torch.equal(stack.forward(x, [20, 0]), want)
    srv.close()


# ------------------------------------------------------------------------------- roundings

@pytest.mark.parametrize("head_dim,glm", [(64, False), (128, True)])
def test_cached_keys_are_rounded_once(F, head_dim, glm):
    """Keys of the first block against their definition in 64 bits from the same 16-bit operands.  Tolerance:
    half an ulp of the key, and of each pair's sums of `hidden` products in 32 bits (in any order) at most
    hidden 2^-24 sum |a w|, 4 ulps of 32 bits for the turn."""
    from paper_2406_14898_gb300.generate import BlockStack
    heads, T = 2, 90
    H = heads * head_dim
    H = 256 * -(-H // 256)
    heads = H // head_dim
    srv = server(F, 1, heads, head_dim, T)
    stack = BlockStack.from_server(srv, 1, T, page_size=16)
    c = 60 if glm else 0
    stack.start(0, c, 33 if glm else None)
    x = rows(T, H)
    stack.forward(x, [T])
    b = stack.blocks[0]
    a = torch.empty_like(x)
    stats = torch.empty((2, T), device="cuda")
    F.fl_k_layernorm_fwd(T, H, x, *b["ln"][:2], stack.cfg.ln_eps, a, stats[0], stats[1])
    w = b["w"][0][H:2 * H].double()
    k = (a.double() @ w.T + b["b"][0][H:2 * H].double()).view(T, heads, head_dim)
    size = (a.double().abs() @ w.abs().T + b["b"][0][H:2 * H].double().abs()).view(T, heads, head_dim)
    i = torch.arange(T, device="cuda")
    first = torch.where(i < c, i, torch.tensor(33, device="cuda")) if glm else i
    rd = head_dim // 2
    turn64(k, stack.rope, first, "half", 0, rd)
    if glm:
        turn64(k, stack.rope, (i - c + 1).clamp(min=0), "half", rd, rd)
    at = stack.pages.table[0].long().cuda()
    got = b["kv"][0][at].transpose(1, 2).flatten(0, 1)[:T].double()  # [token, head, dim]
    wide = size.amax(-1, keepdim=True)
    tol = 1.001 * UNIT["bf16"] * k.abs() + 2 * (H + 4) * 2.0 ** -24 * wide
    worst = ((got - k).abs() / tol).amax()
    assert float(worst) <= 1, float(worst)
    srv.close()


# ------------------------------------------------------------------------------- replicas

def test_a_handle_of_replicas_is_asked_for_one(F):
    """Two replicas that trained on different groups of clients differ; each answers as its own forward does."""
    from paper_2406_14898_gb300.generate import BlockStack
    cfg = F.fl_server_cfg()
    F.lib().fl_server_cfg_default(cfg)
    cfg.n_blocks, cfg.hidden, cfg.n_heads, cfg.head_dim, cfg.rotary_dim = 1, 256, 4, 64, 0
    cfg.ffn_hidden, cfg.residual_alpha, cfg.max_tokens, cfg.n_replicas, cfg.init_std = 1024, 2.0, 64, 2, 0.05
    srv = F.Server(cfg, 5)
    x = [rows(32, 256, s).view(1, 32, 256) for s in (1, 2)]
    y, g = ([torch.empty_like(v) for v in x] for _ in "yg")
    torch.cuda.synchronize()
    srv.forward(x, [32, 32], y)
    srv.backward(y, g)
    srv.step(0.05)
    srv.forward(x, [32, 32], y)
    srv.sync()
    with pytest.raises(ValueError):
        BlockStack.from_server(srv, 1, 32)
    outs = [BlockStack.from_server(srv, 1, 32, replica=r).forward(x[r][0], [32]) for r in (0, 1)]
    for r in (0, 1):
        assert rel_inf(outs[r].double().cpu().numpy(), y[r][0].double().cpu().numpy()) < TOL
    other = BlockStack.from_server(srv, 1, 32, replica=0).forward(x[1][0], [32])
    assert rel_inf(other.double().cpu().numpy(), y[1][0].double().cpu().numpy()) > 10 * TOL
    srv.close()


# ------------------------------------------------------------------------------- clients

def test_a_clients_logits_do_not_depend_on_the_others(F):
    lens = [40, 9, 130]
    prompts = [prompt(k, n) for k, n in enumerate(lens)]
    steps = [[prompt(10 * j + k, 1) for k in range(3)] for j in range(3)]
    together = generator(F, 3)
    together.start(lens)
    want = [together.logits(t) for t in [prompts] + steps]
    for k in range(3):
        alone = generator(F, 1, which=[k])
        alone.start(lens[k:k + 1])
        for t, w in zip([prompts] + steps, want):
            z = alone.logits(t[k:k + 1])[0]
            assert rel_inf(z.double().cpu().numpy(), w[k].double().cpu().numpy()) < TOL
        for other in range(3):  # and the bound tells clients apart
            if other != k:
                assert rel_inf(want[0][other].double().cpu().numpy(), want[0][k].double().cpu().numpy()) > 10 * TOL
