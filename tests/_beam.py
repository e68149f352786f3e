"""Beam search and shared pages for the tests: the definitions, one search or one sequence after another."""
import math

import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
INF = math.inf


def dtype_id(F, dtype):
    return {"bf16": F.FL_DT_BF16, "f16": F.FL_DT_F16, "f32": F.FL_DT_F32}[dtype]


# ------------------------------------------------------------------------------- beam search

def begin(S, B):
    """The state before the first token (numpy)."""
    scores = np.full((S, B), -INF, np.float64)
    scores[:, 0] = 0
    return {"scores": scores, "steps": np.zeros(S, int), "done": np.zeros(S, int), "end_scores": np.full((S, B), -INF),
            "end_steps": np.zeros((S, B), int), "end_beams": np.zeros((S, B), int)}


def device_state(state):
    kinds = {"scores": torch.float32, "end_scores": torch.float32}
    return {k: torch.from_numpy(np.array(v)).to(kinds.get(k, torch.int32)).cuda() for k, v in state.items()}


def step64(state, x, max_steps, eos, penalty, early):
    """One step in 64 bits: (new state, tokens, parents (beams, -1: none), trace rows (None where a search rests), bad).
    x [S, B, V] holds the logits' values."""
    S, B, V = x.shape
    new = {k: np.array(v, copy=True) for k, v in state.items()}
    tokens, parents = np.full((S, B), max(eos, 0)), np.full((S, B), -1)
    rows, bad = [None] * S, False
    for s in range(S):
        t = state["steps"][s]
        if state["done"][s] or t >= max_steps:
            continue
        cands = []
        for b in range(B):
            score = float(state["scores"][s, b])
            if score == -INF:
                continue
            r = x[s, b].astype(np.float64)
            if np.isnan(r).any() or (r == INF).any() or not score < INF:
                bad = True
                continue
            top = r.max()
            if top == -INF:
                continue
            part = math.log(np.exp(r - top).sum())
            few = np.argsort(-r, kind="stable")[:B + 1]
            for v in set(few.tolist()) | ({eos} if eos >= 0 else set()):
                if r[v] > -INF:
                    cands.append((-(score + ((r[v] - top) - part)), b, -r[v], v))
        cands.sort()
        live = [c for c in cands if c[3] != eos][:B]
        length = float(t + 1) ** penalty
        pool = [(np.float32(e), int(n), int(b)) for e, n, b in
                zip(state["end_scores"][s], state["end_steps"][s], state["end_beams"][s]) if e > -INF]
        pool += [(np.float32(-c / length), t, b) for c, b, _, v in cands[:B] if v == eos]
        pool = sorted(pool, key=lambda p: -p[0])[:B]
        for name in ("end_scores", "end_steps", "end_beams"):
            new[name][s] = -INF if name == "end_scores" else 0
        for i, (e, n, b) in enumerate(pool):
            new["end_scores"][s, i], new["end_steps"][s, i], new["end_beams"][s, i] = e, n, b
        new["scores"][s] = -INF
        trace_parents = np.arange(B)
        for i, (c, b, _, v) in enumerate(live):
            new["scores"][s, i], tokens[s, i], parents[s, i], trace_parents[i] = -c, v, b, b
        new["steps"][s] = t + 1
        best = np.float32(-live[0][0] / length) if live else -INF
        new["done"][s] = not live or (len(pool) == B and (early or pool[-1][0] >= best))
        rows[s] = (tokens[s].copy(), trace_parents)
    return new, tokens, parents, rows, bad


def trace64(state, tokens, parents, n_best, pad, eos, penalty):
    """tokens, parents [S, T, B]: (out tokens, lengths, scores)."""
    S, T, B = tokens.shape
    out, lens, scores = np.full((S, n_best, T), pad), np.zeros((S, n_best), int), np.full((S, n_best), -INF)
    for s in range(S):
        hyps = [(np.float32(state["end_scores"][s, i]), state["end_steps"][s, i], state["end_beams"][s, i], True)
                for i in range(B)]
        n = int(state["steps"][s])
        if not state["done"][s] and n:
            hyps += [(np.float32(state["scores"][s, b] / float(n) ** penalty), n, b, False) for b in range(B)]
        hyps = sorted((h for h in hyps if h[0] > -INF), key=lambda h: -h[0])[:n_best]
        for i, (x, n, b, ended) in enumerate(hyps):
            scores[s, i], lens[s, i] = x, n + ended
            if ended and eos >= 0:
                out[s, i, n] = eos
            for t in range(n - 1, -1, -1):
                out[s, i, t] = tokens[s, t, b]
                b = parents[s, t, b]
    return out, lens, scores


class Searches:
    """A search's device buffers and calls."""

    def __init__(self, F, S, B, V, max_steps, eos=-1, penalty=1.0, early=False, workspace=None):
        self.F, self.shape = F, (S, B)
        self.search = F.beam_search(S, B, V, max_steps, eos=eos, length_penalty=penalty, early=early)
        self.trace_tokens, self.trace_parents = (torch.full((S, max_steps, B), -9, dtype=torch.int32, device="cuda")
                                                 for _ in "tp")
        self.tokens, self.parents = (torch.full((S, B), -9, dtype=torch.int32, device="cuda") for _ in "tp")
        self.workspace = (torch.zeros(F.fl_k_beam_workspace(self.search) // 4, dtype=torch.int32, device="cuda")
                          if workspace is None else workspace)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(self, state, out, x, dtype, ld, **kw):
        F = self.F
        F.fl_k_beam_step(self.search, F.beam_state(**state), F.beam_state(**out), x, self.trace_tokens,
                         self.trace_parents, self.tokens, self.parents, self.workspace, self.status,
                         dtype=dtype_id(F, dtype), ld=ld, **kw)

    def trace(self, state, n_best, pad=-1):
        S, T = self.shape[0], self.search.max_steps
        out = (torch.full((S, n_best, T), -9, dtype=torch.int32, device="cuda"),
               torch.full((S, n_best), -9, dtype=torch.int32, device="cuda"), torch.zeros((S, n_best), device="cuda"))
        self.F.fl_k_beam_trace(self.search, self.F.beam_state(**state), self.trace_tokens, self.trace_parents, n_best, pad,
                               *out, self.status)
        return out


def check_step(got, tokens, parents, want, want_tokens, want_parents):
    """got, tokens, parents: device; want...: step64's.  Scores: one rounding (half an ulp, 2^-24 of the score) and the
    log-sum-exp's error, at most 2^-17 (every exponential is off by 2^-22 and by 2^-23 for each unit of its logit's distance from
    the largest, which is ln(2^19) on average at most; a thread adds 64 of them and a row at most 2^13 threads' in a
    tree, 80 roundings of 2^-24)."""
    S, B = want["scores"].shape
    assert np.array_equal(tokens.cpu().numpy(), want_tokens)
    rows = np.where(want_parents >= 0, want_parents + np.arange(S)[:, None] * B, -1)
    assert np.array_equal(parents.cpu().numpy(), rows)
    for k in ("steps", "done", "end_steps", "end_beams"):
        assert np.array_equal(got[k].cpu().numpy(), want[k]), k
    for k in ("scores", "end_scores"):
        x, y = got[k].double().cpu().numpy(), np.asarray(want[k], np.float64)
        assert np.array_equal(x == -INF, y == -INF), k
        fine = y > -INF
        assert (np.abs(x[fine] - y[fine]) <= 2.0 ** -23.9 * np.abs(y[fine]) + 2.0 ** -17).all(), k


# ------------------------------------------------------------------------------- pages

class Refused(Exception):
    pass


def fork(lens, table, refs, page, parents, new):
    """(lens, table, refs, copies (page, page, tokens)) after the call, from lists; Refused where it cannot be done."""
    S, W = len(lens), len(table[0]) if len(table) else 0
    pages = lambda n: -(-n // page)  # noqa: E731
    refs = list(refs)
    before, after, rows = [], [], []
    for p, n in zip(parents, new):
        if not -1 <= p < S:
            raise Refused
        x = lens[p] if p >= 0 else 0
        y = max(0, x + n)
        if pages(y) > W:
            raise Refused
        before.append(x)
        after.append(y)
        rows.append(list(table[p][:min(pages(x), pages(y))]) if p >= 0 else [])
    for s in range(S):
        for q in table[s][:pages(lens[s])]:
            refs[q] -= 1
    for row in rows:
        for q in row:
            refs[q] += 1
    writers = {}
    for s in range(S):
        if new[s] > 0 and before[s] % page:
            writers.setdefault(rows[s][-1], []).append(s)
    leave = {s for q, w in writers.items() for s in (w[1:] if refs[q] == len(w) else w)}
    free = [q for q, n in enumerate(refs) if n == 0]
    copies = []
    for s in range(S):
        if s in leave:
            if not free:
                raise Refused
            q = rows[s][-1]
            refs[q] -= 1
            copies.append((q, free[0], before[s] % page))
            rows[s][-1] = free.pop(0)
            refs[rows[s][-1]] = 1
        while len(rows[s]) < pages(after[s]):
            if not free:
                raise Refused
            rows[s].append(free.pop(0))
            refs[rows[s][-1]] = 1
    return after, [row + [-1] * (W - len(row)) for row in rows], refs, copies


def compact(lens, table, refs, page):
    """(table, refs, moved, used, copies)."""
    used = sum(r > 0 for r in refs)
    moved = [q if r > 0 else -1 for q, r in enumerate(refs)]
    src = [q for q in range(used, len(refs)) if refs[q] > 0]
    dst = [q for q in range(used) if refs[q] == 0]
    for a, b in zip(src, dst):
        moved[a] = b
    new_refs = [0] * len(refs)
    for q, m in enumerate(moved):
        if m >= 0:
            new_refs[m] = refs[q]
    new_table = [[moved[q] if i < -(-x // page) else -1 for i, q in enumerate(row)] for x, row in zip(lens, table)]
    return new_table, new_refs, moved, used, [(a, b, page) for a, b in zip(src, dst)]


class Pool:
    """Device side of a page table that serves `blocks` caches, [block, page, slot, head, dim]; every number in
    them has its own value."""

    def __init__(self, F, n_seqs, n_pages, page, width, blocks=2, heads=2, hd=64, dtype="bf16", token_major=False, seed=0):
        self.F, self.page, self.shape = F, page, (n_seqs, n_pages, page, width)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        shape = (blocks, n_pages) + ((page, heads, hd) if token_major else (heads, page, hd))
        storage = [torch.randint(-30000, 30000, shape, generator=gen, device="cuda", dtype=torch.int16).view(DTYPES[dtype])
                   for _ in "kv"]
        self.k, self.v = storage if token_major else [x.transpose(2, 3) for x in storage]
        one = self.k[0]
        self.caches = F.kv_caches([F.kv_cache(k, v, n_pages, page, heads, hd, dtype=dtype_id(F, dtype),
                                              page_stride=one.stride(0), token_stride=one.stride(1),
                                              head_stride=one.stride(2)) for k, v in zip(self.k, self.v)])
        self.sides = [{"lens": torch.zeros(n_seqs, dtype=torch.int32, device="cuda"),
                       "table": torch.full((n_seqs, width), -1, dtype=torch.int32, device="cuda"),
                       "refs": torch.zeros(n_pages, dtype=torch.int32, device="cuda")} for _ in "ab"]
        self.pages = [F.kv_pages(*self.shape, **side) for side in self.sides]
        self.workspace = torch.zeros(F.fl_k_kv_pages_workspace(self.pages[0]) // 4, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def set(self, lens, table, refs, side=0):
        for name, v in (("lens", lens), ("table", table), ("refs", refs)):
            self.sides[side][name].copy_(torch.tensor(v, dtype=torch.int32).view(self.sides[side][name].shape))

    def get(self, side=0):
        return [self.sides[side][name].tolist() for name in ("lens", "table", "refs")]

    def bits(self):
        """The caches' numbers, as whole numbers (copies are exact, NaN included)."""
        return [x.clone(memory_format=torch.contiguous_format).view(torch.int16) for x in (self.k, self.v)]

    def fork(self, parents, new, side=0, **kw):
        p, n = (None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda") for x in (parents, new))
        self.F.fl_k_kv_fork(self.caches, self.pages[side], self.pages[1 - side], p, n, self.workspace, self.status, **kw)
        torch.cuda.synchronize()  # the arrays above live as long as this call

    def compact(self, side=0, **kw):
        moved = torch.full((self.shape[1],), -9, dtype=torch.int32, device="cuda")
        used = torch.full((1,), -9, dtype=torch.int32, device="cuda")
        self.F.fl_k_kv_compact(self.caches, self.pages[side], self.pages[1 - side], moved, used, self.workspace, self.status,
                               **kw)
        return moved, used


def moved_bits(bits, copies):
    out = [x.clone() for x in bits]
    for x, y in zip(bits, out):
        for a, b, n in copies:
            y[:, b, :n] = x[:, a, :n]
    return out
