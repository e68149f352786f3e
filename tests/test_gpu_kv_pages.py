"""Sequences that share pages (fork) and caches that are moved together (compact), against lists (GPU only)."""
import random

import pytest
import torch

from tests._beam import Pool, Refused, compact, fork, moved_bits
from tests._gpu import flglm, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


def step(pool, parents, new, side, status=0):
    """One fork, compared with the lists' (which it returns) in everything: arrays, copies and what stays."""
    S, n_pages, page, W = pool.shape
    lens, table, refs = pool.get(side)
    before = pool.bits()
    pool.sides[1 - side]["table"].fill_(-77)
    pool.fork(parents, new, side)
    want = fork(lens, table, refs, page, range(S) if parents is None else parents, [0] * S if new is None else new)
    assert pool.get(1 - side) == list(want[:3])
    assert pool.get(side) == [lens, table, refs]
    for a, b in zip(pool.bits(), moved_bits(before, want[3])):
        assert torch.equal(a, b)
    assert int(pool.status.item()) == status
    assert not pool.workspace[:3 * (-(-n_pages // 4) * 4)].any()  # counts, for the next call
    return want


@pytest.mark.parametrize("page,heads,hd,dtype,token_major,blocks", [(16, 2, 64, "bf16", False, 2), (32, 1, 128, "f16", True, 1),
                                                                    (64, 8, 128, "bf16", False, 3), (256, 3, 64, "f16", True, 2),
                                                                    (128, 32, 128, "bf16", True, 1), (16, 5, 128, "bf16", False, 64)])
def test_beams_step_by_step(F, page, heads, hd, dtype, token_major, blocks):
    """Prompts of two searches with four beams each: spread over the beams, then a token a step with new parents."""
    rng = random.Random(page + heads)
    S, W = 8, 7 + 40 // page
    pool = Pool(F, S, 2 * W + 24, page, W, blocks, heads, hd, dtype, token_major)
    side = 0
    for parents, new in ([None, [3 * page + 5, 0, 0, 0, 2 * page, 0, 0, 0]], [[0, 0, 0, 0, 4, 4, 4, 4], None]):
        step(pool, parents, new, side)
        side = 1 - side
    copies = 0
    for t in range(40):
        parents = [4 * (s // 4) + min(rng.randrange(4), rng.randrange(4)) for s in range(S)]
        if t % 9 == 8:
            parents[rng.randrange(S)] = -1
        copies += len(step(pool, parents, [1] * S, side)[3])
        side = 1 - side
    assert copies > 20


@pytest.mark.parametrize("S,n_pages,W,page", [(1, 3, 1, 16), (3, 9, 2, 256), (37, 300, 9, 16), (150, 2500, 40, 32), (5, 20001, 1500, 16),
                                              (1100, 3000, 3, 16)])
def test_any_step_from_any_state(F, S, n_pages, W, page):
    """Chains of forks with random parents, growth, tokens taken off and holders outside of the table."""
    rng = random.Random(n_pages)
    pool = Pool(F, S, n_pages, page, W, 1, 1, 64)
    side, done, refused = 0, 0, 0
    kept = []
    for t in range(14):
        parents = [rng.choice([-1, s, s, s, rng.randrange(S)]) for s in range(S)]
        grow = rng.choice([1, page, W * page // 2])
        new = [rng.choice([1, 0, rng.randint(-grow, grow)]) for _ in range(S)]
        args = (None if t == 3 else parents), (None if t == 5 else new)
        lens, table, refs = pool.get(side)
        try:
            done += len(step(pool, *args, side)[3]) > 0
        except Refused:
            refused += 1
            assert int(pool.status.item()) == F.FL_KV_NO_ROOM
            assert pool.get(1 - side) == [lens, table, refs]  # as it was
            pool.status.zero_()
        side = 1 - side
        lens, table, refs = pool.get(side)
        for q in kept:
            refs[q] -= 1
        kept = rng.sample(sorted({q for row in table for q in row if q >= 0}), min(3, len({q for row in table for q in row if q >= 0})))
        for q in kept:  # somebody keeps these pages until the next step
            refs[q] += 1
        pool.set(lens, table, refs, side)
    assert done or S < 4


def test_a_shared_page_is_copied_before_it_is_written(F):
    """Two rows and a holder outside; writers and readers; a shortened row whose last page others have as a whole one."""
    page, W = 16, 4
    def start(lens, table, more=()):
        pool = Pool(F, 4, 20, page, W)
        refs = [0] * 20
        for x, row in zip(lens, table):
            for q in row[:-(-x // page)]:
                refs[q] += 1
        for q in more:
            refs[q] += 1
        pool.set(lens, [row + [-1] * (W - len(row)) for row in table], refs)
        return pool
    shared = ([20, 20, 20, 0], [[3, 7], [3, 7], [3, 7], []])
    assert step(start(*shared), None, [1, 1, 1, 0], 0)[3] == [(7, 0, 4), (7, 1, 4)]      # all write: the first keeps it
    assert step(start(*shared), None, [1, 0, 1, 0], 0)[3] == [(7, 0, 4), (7, 1, 4)]      # one only reads: all writers leave
    assert step(start(*shared, [7]), None, [1, 1, 1, 0], 0)[3] == [(7, 0, 4), (7, 1, 4), (7, 2, 4)]
    assert step(start(*shared), None, [0, 0, 0, 0], 0)[3] == []
    assert step(start(*shared), [0, -1, -1, -1], [1, 0, 0, 0], 0)[3] == []                # the others go in the same call
    assert step(start([20, 48, 0, 0], [[3, 7], [3, 7, 9], [], []]), None, [2, 0, 0, 0], 0)[3] == [(7, 0, 4)]
    assert step(start([48, 48, 0, 0], [[3, 7, 9], [3, 7, 9], [], []]), None, [-21, 0, 0, 0], 0)[3] == []
    assert step(start([16, 16, 16, 0], [[3], [3], [3], []]), None, [1, 1, 1, 0], 0)[3] == []  # whole pages only
    # rows at one page of which the later ends sooner
    assert step(start([20, 18, 0, 0], [[3, 7], [3, 7], [], []]), None, [1, 1, 0, 0], 0)[3] == [(7, 0, 2)]


def test_pages_that_a_call_frees_serve_it(F):
    """A pool with no page to spare: the beams that go make room for the copies of those that stay."""
    page = 16
    pool = Pool(F, 3, 4, page, 2)
    pool.set([20, 20, 20], [[0, 1], [0, 2], [0, 3]], [3, 1, 1, 1])
    want = step(pool, [2, 2, 2], [1, 1, 1], 0)
    assert want[1] == [[0, 3], [0, 1], [0, 2]] and want[3] == [(3, 1, 4), (3, 2, 4)]


@pytest.mark.parametrize("parents,new,bits", [([0, 0, 0], [1, 1, 13], 16), ([0, 0, 0], [1, 1, 1], 0), ([0, 3, 0], [1, 1, 1], 32),
                                              ([0, -2, 0], [100, 1, 1], 48), ([0, 1, 2], [60, 0, 0], 16), (None, [2 ** 31 - 1, 0, 0], 16)])
def test_calls_that_cannot_be_done_change_nothing(F, parents, new, bits):
    page = 16
    pool = Pool(F, 3, 4, page, 3)
    state = [[20, 3, 0], [[1, 2, -1], [3, -1, -1], [-1] * 3], [0, 1, 1, 1]]
    pool.set(*state)
    before = pool.bits()
    if bits == 0:  # this one can
        assert fork(*state, page, parents, new)[3] == [(2, 0, 4), (2, 3, 4)]
    pool.fork(parents, new)
    assert int(pool.status.item()) == bits
    if bits:
        assert pool.get(1) == state
        assert all(torch.equal(a, b) for a, b in zip(before, pool.bits()))
    assert not pool.workspace[:12].any()


def test_entries_and_lengths_out_of_range(F):
    """They are told, brought into range or passed on; nothing outside of the buffers is touched."""
    page = 16
    pool = Pool(F, 3, 6, page, 3)
    pool.set([20, 20, 0], [[1, 9, -1], [2, -1, -1], [-1] * 3], [0, 1, 1, 0, 0, 0])
    before = pool.bits()
    pool.fork([0, 1, 1], [1, 0, 1])
    assert int(pool.status.item()) == F.FL_KV_BAD_PAGE
    assert pool.get(1) == [[21, 20, 21], [[1, 9, -1], [2, -1, -1], [2, -1, -1]], [0, 1, 2, 0, 0, 0]]
    assert all(torch.equal(a, b) for a, b in zip(before, pool.bits()))
    pool.status.zero_()
    pool.set([49, -3, 0], [[1, 2, 3], [-1] * 3, [-1] * 3], [0, 1, 1, 1, 0, 0])
    pool.fork(None, [0, 1, 0])
    assert int(pool.status.item()) == F.FL_KV_BAD_PAGE
    assert pool.get(1) == [[48, 1, 0], [[1, 2, 3], [0, -1, -1], [-1] * 3], [1, 1, 1, 1, 0, 0]]
    pool.status.zero_()
    pool.set([20, 5, 0], [[1, 9, -1], [4, -1, -1], [-1] * 3], [0, 1, 0, 0, 0, 0])
    moved, used = pool.compact()
    assert int(pool.status.item()) == F.FL_KV_BAD_PAGE and moved.tolist() == [-1, 0, -1, -1, -1, -1] and used.tolist() == [1]
    assert pool.get(1) == [[20, 5, 0], [[0, -1, -1], [-1] * 3, [-1] * 3], [1, 0, 0, 0, 0, 0]]


@pytest.mark.parametrize("n_pages,busy,page,heads,hd,dtype,token_major", [(1, 0, 16, 1, 64, "bf16", False), (1, 1, 16, 1, 64, "bf16", False),
                                                                          (9, 4, 64, 2, 128, "f16", True), (41, 41, 16, 2, 64, "bf16", False),
                                                                          (1024, 500, 16, 1, 64, "bf16", False), (1025, 3, 16, 1, 64, "f16", True),
                                                                          (20000, 11000, 16, 1, 64, "bf16", False), (17001, 1, 16, 1, 64, "bf16", False),
                                                                          (300, 140, 256, 4, 128, "bf16", False)])
def test_compact(F, n_pages, busy, page, heads, hd, dtype, token_major):
    rng = random.Random(n_pages + busy)
    order = rng.sample(range(n_pages), busy)
    refs = [0] * n_pages
    S, W = 5, 1 + busy // 3
    lens, table, at = [], [], 0
    for s in range(S):
        n = min(W, rng.randint(0, max(0, busy - at)))
        row = order[at:at + n]
        at += n
        if s == 2 and table[0] and n:
            row[0] = table[0][0]
        lens.append(max(0, len(row) * page - rng.randrange(page)))
        table.append(row + [-1] * (W - n))
        for q in row:
            refs[q] += 1
    for q in order[at:]:
        refs[q] += 2  # kept by others
    pool = Pool(F, S, n_pages, page, W, 2, heads, hd, dtype, token_major)
    pool.set(lens, table, refs)
    before = pool.bits()
    moved, used = pool.compact()
    want = compact(lens, table, refs, page)
    assert pool.get(1) == [lens, want[0], want[1]]
    assert moved.tolist() == want[2] and used.tolist() == [want[3]]
    for a, b in zip(pool.bits(), moved_bits(before, want[4])):
        assert torch.equal(a, b)
    assert int(pool.status.item()) == 0
    again, count = pool.compact(side=1)  # nothing is left to move
    assert again.tolist() == [q if q < want[3] else -1 for q in range(n_pages)] and count.tolist() == [want[3]]
    assert pool.get(0) == pool.get(1)


@pytest.mark.parametrize("heads,hd,page,pad_heads,pad_tokens,token_major", [(3, 64, 16, 8, 0, False), (2, 128, 64, 0, 8, False),
                                                                             (4, 64, 32, 0, 16, True), (5, 128, 16, 8, 24, True)])
def test_caches_with_gaps(F, heads, hd, page, pad_heads, pad_tokens, token_major):
    """Heads and tokens that do not lie next to each other; what lies between them is left alone."""
    rng = random.Random(heads)
    S, n_pages, W = 6, 30, 4
    pool = Pool(F, S, n_pages, page, W, 1, heads, hd)
    if token_major:
        head, token = hd + pad_heads, heads * (hd + pad_heads) + pad_tokens
        each = -(-page * token // head) * head
    else:
        token = hd + pad_tokens
        head = page * token + pad_heads
        each = heads * head
    raw = [torch.randint(-30000, 30000, (n_pages * each,), device="cuda", dtype=torch.int16) for _ in "kv"]
    pool.caches = F.kv_caches([F.kv_cache(*raw, n_pages, page, heads, hd, page_stride=each, head_stride=head, token_stride=token)])
    views = [x.as_strided((n_pages, page, heads, hd), (each, token, head, 1)) for x in raw]
    pool.fork(None, [3 * page - 2, 5, 0, 0, page, 1])
    side = 1
    for t in range(6):
        parents = [rng.randrange(S) for _ in range(S)]
        lens, table, refs = pool.get(side)
        want = fork(lens, table, refs, page, parents, [1] * S)
        before = [x.clone() for x in raw]
        pool.fork(parents, [1] * S, side)
        side = 1 - side
        for x, v, b in zip(raw, views, before):
            expect = b.as_strided(v.shape, v.stride())
            for a, d, n in want[3]:
                expect[d, :n] = v[a, :n]
            assert torch.equal(x, b)
        assert pool.get(side) == list(want[:3]) and int(pool.status.item()) == 0
    lens, table, refs = pool.get(side)
    before = [x.clone() for x in raw]
    pool.compact(side=side)
    for x, v, b in zip(raw, views, before):
        expect = b.as_strided(v.shape, v.stride())
        for a, d, n in compact(lens, table, refs, page)[4]:
            expect[d] = v[a]
        assert torch.equal(x, b)


def test_no_sequences(F):
    pool = Pool(F, 0, 5, 16, 2)
    pool.sides[0]["refs"].copy_(torch.tensor([0, 1, 0, 0, 2]))
    pool.fork(None, None)
    assert pool.sides[1]["refs"].tolist() == [0, 1, 0, 0, 2]
    moved, used = pool.compact()
    assert moved.tolist() == [-1, 1, -1, -1, 0] and used.tolist() == [2] and pool.sides[1]["refs"].tolist() == [2, 1, 0, 0, 0]


def test_graph_of_two_steps_replayed(F):
    """Two forks there and back, captured once, follow the arrays' contents; on a stream of their own."""
    page, S, W = 16, 6, 5
    pool = Pool(F, S, 40, page, W)
    pool.set([20] * S, [[0, 1 + s] + [-1] * 3 for s in range(S)], [S] + [1] * S + [0] * (39 - S))
    parents = torch.tensor([0, 0, 1, 3, 3, 5], dtype=torch.int32, device="cuda")
    new = torch.ones(S, dtype=torch.int32, device="cuda")

    def both(stream):
        for side in (0, 1):
            F.fl_k_kv_fork(pool.caches, pool.pages[side], pool.pages[1 - side], parents, new, pool.workspace, pool.status,
                           stream=stream)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(torch.cuda.current_stream())
    lists = pool.get()
    rng = random.Random(3)
    for _ in range(12):
        p = [rng.randrange(S) for _ in range(S)]
        parents.copy_(torch.tensor(p))
        before = pool.bits()
        graph.replay()
        for _ in "ab":
            lists = list(fork(*lists[:3], page, p, [1] * S))
            before = moved_bits(before, lists[3])
        assert pool.get() == lists[:3]
        assert all(torch.equal(a, b) for a, b in zip(before, pool.bits()))
    assert int(pool.status.item()) == 0


def test_two_tables_at_once(F):
    """Two tables on two streams, each with its own workspace; one's counts lie in a CTA's shared memory, the other's in a cluster's."""
    rng = random.Random(8)
    calls, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for S, n_pages, W, seed in ((12, 400, 30, 1), (1200, 18000, 12, 2)):
        pool = Pool(F, S, n_pages, 16, W, blocks=1, heads=1, seed=seed)
        lens = [rng.randrange(1, 16 * W - 24) for _ in range(S)]
        table, refs, at = [], [0] * n_pages, 0
        for n in lens:
            held = -(-n // 16)
            table.append(list(range(at, at + held)) + [-1] * (W - held))
            refs[at:at + held] = [1] * held
            at += held
        pool.set(lens, table, refs)
        parents = [[rng.randrange(S) if rng.random() < 0.3 else s for s in range(S)] for _ in range(6)]
        calls.append((pool, parents, [torch.tensor(p, dtype=torch.int32, device="cuda") for p in parents],
                      torch.ones(S, dtype=torch.int32, device="cuda"), lens, table, refs, pool.bits()))
    torch.cuda.synchronize()
    for t in range(6):
        for stream, (pool, _, parents, new, *_) in zip(streams, calls):
            F.fl_k_kv_fork(pool.caches, pool.pages[t % 2], pool.pages[1 - t % 2], parents[t], new, pool.workspace, pool.status,
                           stream=stream)
    torch.cuda.synchronize()
    for pool, parents, _, _, *lists, bits in calls:
        for p in parents:
            lists = list(fork(*lists[:3], 16, p, [1] * len(p)))
            bits = moved_bits(bits, lists[3])
        assert pool.get() == lists[:3] and int(pool.status.item()) == 0
        assert all(torch.equal(a, b) for a, b in zip(bits, pool.bits()))
