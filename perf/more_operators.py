"""Beam search over a paged key / value cache, as cases to time and compare.

A client that answers with several beams picks, after each token, the best continuations of all its beams; the
beams' caches then follow their parents: sequences share the pages of what they have in common, and a partly
filled page that two of them are about to write is copied.

  select   the next beams, the hypotheses that end and the state of the search, from the logits of every beam
  trace    the best hypotheses' tokens, from the back-pointers of every step
  fork     every sequence continues another one (or itself, or none): page table, shares and copied pages
  compact  the pages in use moved to the front of the cache

``own`` False: plain torch; True: the framework's entry points (``paper_2406_14898_gb300.flglm``).  ``exact`` is the
definition in 64 bits, or sequence by sequence.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _nums(text):
    return [int(x) for x in text.split()]


def _join(xs):
    return " ".join(str(x) for x in xs)


# ------------------------------------------------------------------------------- the cases

def _beam_parents(rng, clients, beams):
    """What a step of a beam search picks: the better beams have more children."""
    return [c * beams + min(rng.randrange(beams), rng.randrange(beams)) for c in range(clients) for _ in range(beams)]


def listed():
    rng = random.Random(7)
    prompts = [rng.randint(64, 512) for _ in range(16)]
    serving = [rng.randint(1, 2000) for _ in range(192)]
    return [
        # the first choice of three clients with few beams in a small vocabulary, as the test models have it: latency
        {"name": "select_small_f16", "kind": "select", "clients": 3, "beams": 5, "vocab": 1003, "row": 1008, "dtype": "f16",
         "eos": 2, "penalty": 1.0, "early": False, "first": True, "done": 0, "steps": 64},
        # one client's next step with the 6B model's vocabulary: latency
        {"name": "select_one", "kind": "select", "clients": 1, "beams": 4, "vocab": 130528, "row": 130560, "dtype": "f32",
         "eos": 130005, "penalty": 1.0, "early": False, "first": False, "done": 0, "steps": 256},
        # the clients of a generation in one call, logits in 32 bits as the LM head leaves them
        {"name": "select_clients", "kind": "select", "clients": 32, "beams": 4, "vocab": 130528, "row": 130560,
         "dtype": "f32", "eos": 130005, "penalty": 0.6, "early": False, "first": False, "done": 2, "steps": 256},
        # many clients with many beams
        {"name": "select_wide_bf16", "kind": "select", "clients": 64, "beams": 16, "vocab": 130528, "row": 130528,
         "dtype": "bf16", "eos": 130005, "penalty": 2.0, "early": True, "first": False, "done": 0, "steps": 512},
        # the answers of 16 clients
        {"name": "trace_answers", "kind": "trace", "clients": 16, "beams": 4, "steps": 256, "best": 1, "penalty": 1.0},
        # every hypothesis of many long searches
        {"name": "trace_long", "kind": "trace", "clients": 64, "beams": 16, "steps": 2048, "best": 16, "penalty": 0.6},
        # one client's own block after a step of four beams: latency
        {"name": "fork_one", "kind": "fork", "blocks": 1, "heads": 32, "head_dim": 128, "dtype": "bf16", "page": 64,
         "token_major": False, "group": 4, "common": "290", "len": "301 301 301 301", "parents": "0 0 1 3",
         "new": "1 1 1 1"},
        # 16 clients' beams in all blocks of a server
        {"name": "fork_clients", "kind": "fork", "blocks": 26, "heads": 32, "head_dim": 128, "dtype": "bf16", "page": 64,
         "token_major": False, "group": 4, "common": _join(prompts), "len": _join(p + 41 for p in prompts for _ in range(4)),
         "parents": _join(_beam_parents(rng, 16, 4)), "new": _join([1] * 64)},
        # many beams behind two long documents: long page tables, shared key / value heads, small token-major pages
        {"name": "fork_long_f16", "kind": "fork", "blocks": 26, "heads": 4, "head_dim": 128, "dtype": "f16", "page": 16,
         "token_major": True, "group": 8, "common": "65501 40001", "len": _join([65535] * 8 + [40039] * 8),
         "parents": _join(_beam_parents(rng, 2, 8)), "new": _join([1] * 16)},
        # many sequences of a server between two calls: chunks and single tokens to come, tokens taken back, sequences
        # that end and others that begin as copies
        {"name": "fork_serving", "kind": "fork", "blocks": 12, "heads": 2, "head_dim": 64, "dtype": "bf16", "page": 32,
         "token_major": False, "group": 1, "common": _join([0] * 192), "len": _join(serving),
         "parents": _join(-1 if s % 11 == 5 else (s * 7) % 192 if s % 9 == 2 else s for s in range(192)),
         "new": _join([1, 1, 256, 1, 0, -5, 1, 33][s % 8] for s in range(192))},
        # one block of a small cache: latency
        {"name": "compact_small", "kind": "compact", "blocks": 1, "heads": 4, "head_dim": 64, "dtype": "bf16", "page": 16,
         "token_major": False, "pages": 41, "len": "70 1 0 129 33", "kept": 2},
        # all blocks of a server after half of its clients have left
        {"name": "compact_clients", "kind": "compact", "blocks": 26, "heads": 32, "head_dim": 128, "dtype": "bf16",
         "page": 64, "token_major": False, "pages": 300, "len": _join(prompts + [909, 472, 683, 733]), "kept": 9},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["select", "select", "trace", "fork", "fork", "compact"])
    most = max(work(c)["bytes"] for c in listed() if c["kind"] == kind)
    while True:
        case = _DRAWN[kind](rng)
        if work(case)["bytes"] <= most:
            return case


def _draw_select(rng):
    dtype = rng.choice(["f32", "f32", "bf16", "f16"])
    vocab = rng.choice([130528, _log(rng, 20, 200000)])
    unit = 4 if dtype == "f32" else 8
    clients = _log(rng, 1, 64)
    return {"kind": "select", "clients": clients, "beams": _log(rng, 1, 16), "vocab": vocab,
            "row": -(-vocab // unit) * unit + rng.choice([0, 0, unit, 256]), "dtype": dtype,
            "eos": rng.choice([-1, vocab - 1, rng.randrange(vocab)]), "penalty": rng.choice([0.0, 0.6, 1.0, 2.0]),
            "early": rng.random() < 0.5, "first": rng.random() < 0.2, "done": rng.choice([0, 0, clients // 4]),
            "steps": _log(rng, 4, 2048)}


def _draw_trace(rng):
    beams = _log(rng, 1, 16)
    return {"kind": "trace", "clients": _log(rng, 1, 64), "beams": beams, "steps": _log(rng, 1, 4096),
            "best": rng.choice([1, beams, rng.randint(1, beams)]), "penalty": rng.choice([0.0, 0.6, 1.0, 2.0])}


def _draw_cache(rng):
    heads, head_dim = rng.choice([(32, 128), (8, 128), (4, 128), (4, 64), (2, 64), (1, 128)])
    return {"blocks": rng.choice([1, 2, 12, 26]), "heads": heads, "head_dim": head_dim, "dtype": rng.choice(["bf16", "f16"]),
            "page": rng.choice([16, 32, 64, 128, 256]), "token_major": rng.random() < 0.3}


def _page_bytes(case):
    """Of a page in all blocks, keys and values."""
    return case["blocks"] * 4 * case["page"] * case["heads"] * case["head_dim"]


def _draw_fork(rng):
    case = {"kind": "fork"} | _draw_cache(rng)
    group = rng.choice([1, 4, _log(rng, 1, 16)])
    clients = _log(rng, 1, max(1, 128 // group))
    longest = _log(rng, 16, 32768)
    common = [_log(rng, max(1, longest // 8), longest) for _ in range(clients)]
    lens = [p + n for p, n in zip(common, [rng.randint(0, 100) for _ in common]) for _ in range(group)]
    rows = clients * group
    if rng.random() < 0.5:
        parents, new = _beam_parents(rng, clients, group), [1] * rows
    else:
        chunk = _log(rng, 2, 512)
        parents = [rng.choice([-1, s, s, s, s, rng.randrange(rows)]) for s in range(rows)]
        new = [rng.choice([1, 1, 0, chunk, -rng.randint(1, 40)]) for _ in range(rows)]
    case |= {"group": group, "common": _join(common), "len": _join(lens), "parents": _join(parents), "new": _join(new)}
    while _pool(case) * _page_bytes(case) > 8e9:
        case["blocks"] = max(1, case["blocks"] // 2)
        case["heads"] = max(1, case["heads"] // 2)
        if case["blocks"] == case["heads"] == 1:
            break
    return case


def _draw_compact(rng):
    case = {"kind": "compact"} | _draw_cache(rng)
    lens = [_log(rng, 1, _log(rng, 16, 16384)) for _ in range(_log(rng, 1, 128))]
    held = sum(-(-x // case["page"]) for x in lens)
    kept = rng.randint(0, 9)
    case |= {"pages": held + kept + _log(rng, 1, held + 8), "len": _join(lens), "kept": kept}
    while case["pages"] * _page_bytes(case) > 8e9:
        case["blocks"] = max(1, case["blocks"] // 2)
        case["heads"] = max(1, case["heads"] // 2)
        if case["blocks"] == case["heads"] == 1:
            break
    return case


_DRAWN = {"select": _draw_select, "trace": _draw_trace, "fork": _draw_fork, "compact": _draw_compact}


# ------------------------------------------------------------------------------- the inputs

def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _search_state(S, B, steps, gen):
    """A search under way: live beams in descending order, some hypotheses that have ended."""
    r = lambda *shape: torch.rand(shape, generator=gen, device="cuda")  # noqa: E731
    at = (r(S) * max(1, steps - 1)).int().clamp(max=steps - 1)
    scores = -(20 + 3 * r(S, B).cumsum(1))
    count = (r(S) * (B + 1)).int().clamp(max=B)
    ended = torch.arange(B, device="cuda") < torch.minimum(count, at)[:, None]
    return {"scores": scores, "steps": at.contiguous(), "done": torch.zeros(S, dtype=torch.int32, device="cuda"),
            "end_scores": torch.where(ended, -(1 + r(S, B).cumsum(1)), -math.inf),
            "end_steps": torch.where(ended, (r(S, B) * at[:, None]).int(), 0),
            "end_beams": torch.where(ended, (r(S, B) * B).int().clamp(max=B - 1), 0)}


def _prepare_select(case, gen, st):
    S, B, V = case["clients"], case["beams"], case["vocab"]
    x = torch.randn((S * B, case["row"]), generator=gen, device="cuda", dtype=DTYPES[case["dtype"]]).mul_(3)
    banned = torch.rand(V, generator=gen, device="cuda") < 0.01  # tokens that may not follow
    x[:, :V].masked_fill_(banned, -math.inf)
    x[:, :min(V, 2)] = 1.0
    if case["eos"] >= 0:  # likely for some beams
        x[:, case["eos"]] = torch.where(torch.rand(S * B, generator=gen, device="cuda") < 0.3, 12.0, 0.0).to(x.dtype)
    st["logits"] = x
    st["state"] = _search_state(S, B, case["steps"], gen)
    if case["first"]:
        s = st["state"]
        s["scores"] = torch.where(torch.arange(B, device="cuda") > 0, -math.inf, 0.0).expand(S, B).contiguous()
        s["steps"].zero_()
        s["end_scores"].fill_(-math.inf)
        s["end_steps"].zero_()
        s["end_beams"].zero_()
    st["state"]["done"][:case["done"]] = 1
    st["next"] = {k: torch.empty_like(v) for k, v in st["state"].items()}
    for name in ("trace_tokens", "trace_parents"):
        st[name] = torch.zeros((S, case["steps"], B), dtype=torch.int32, device="cuda")
    for name in ("tokens", "parents"):
        st[name] = torch.empty((S, B), dtype=torch.int32, device="cuda")


def _prepare_trace(case, gen, st):
    S, B, T = case["clients"], case["beams"], case["steps"]
    st["state"] = _search_state(S, B, T, gen)
    st["state"]["steps"] += (torch.rand(S, generator=gen, device="cuda") < 0.5).int()
    st["state"]["steps"].clamp_(min=1)
    ended = st["state"]["end_scores"][:, 0] > -math.inf
    st["state"]["done"] = (ended & (torch.rand(S, generator=gen, device="cuda") < 0.3)).int()
    st["trace_tokens"] = torch.randint(130528, (S, T, B), generator=gen, device="cuda", dtype=torch.int32)
    a, b = (torch.randint(B, (S, T, B), generator=gen, device="cuda", dtype=torch.int32) for _ in "ab")
    st["trace_parents"] = torch.minimum(a, b)
    n = case["best"]
    st["out_tokens"] = torch.empty((S, n, T), dtype=torch.int32, device="cuda")
    st["out_lens"] = torch.empty((S, n), dtype=torch.int32, device="cuda")
    st["out_scores"] = torch.empty((S, n), device="cuda")


def _grown(case):
    """Tokens of each sequence before and after a fork."""
    lens = _nums(case["len"])
    before = [lens[p] if p >= 0 else 0 for p in _nums(case["parents"])]
    return before, [max(0, x + n) for x, n in zip(before, _nums(case["new"]))]


def _rows_pages(case):
    """Page table of a fork's sequences, pages counted from 0: what the sequences of a group have in common they share
    in whole pages."""
    page, group = case["page"], case["group"]
    rows, at = [], 0
    for s, x in enumerate(_nums(case["len"])):
        held, same = -(-x // page), _nums(case["common"])[s // group] // page
        first = rows[s - s % group] if s % group else []
        same = min(same, held, len(first))
        rows.append(first[:same] + list(range(at, at + held - same)))
        at += held - same
    return rows, at


def _pool(case):
    before, after = _grown(case)
    page = case["page"]
    return _rows_pages(case)[1] + sum(max(0, -(-y // page) - -(-x // page)) + 1 for x, y in zip(before, after)) + 3


def _caches(case, st, n_pages, gen):
    """Keys and values of every block, [block, page, slot, head, dim]; pages out of use hold what others left."""
    page, heads, hd = case["page"], case["heads"], case["head_dim"]
    shape = (case["blocks"], n_pages) + ((page, heads, hd) if case["token_major"] else (heads, page, hd))
    for w in "kv":
        x = torch.randn(shape, generator=gen, device="cuda", dtype=DTYPES[case["dtype"]])
        st[w] = x if case["token_major"] else x.transpose(2, 3)


def _prepare_pages(case, st, rows, n_pages, order, width, kept):
    """Lengths, table and the number of holders of each page, now and after the call."""
    table = torch.full((len(rows), width), -1, dtype=torch.int32)
    for s, row in enumerate(rows):
        table[s, :len(row)] = torch.tensor([order[p] for p in row], dtype=torch.int32)
    refs = torch.bincount(table[table >= 0].long(), minlength=n_pages).to(torch.int32)
    for p in kept:
        refs[p] += 1
    st["pages"] = {"lens": _i32(_nums(case["len"])), "table": table.cuda(), "refs": refs.cuda()}
    st["next"] = {k: torch.empty_like(v) for k, v in st["pages"].items()}
    st["n_pages"], st["status"] = n_pages, torch.zeros(1, dtype=torch.int32, device="cuda")


def _prepare_fork(case, gen, st):
    rows, _ = _rows_pages(case)
    n_pages = _pool(case)
    order = torch.randperm(n_pages, generator=gen, device="cuda").tolist()
    width = -(-max(_nums(case["len"]) + _grown(case)[1]) // case["page"]) + 1
    _caches(case, st, n_pages, gen)
    _prepare_pages(case, st, rows, n_pages, order, width, [])
    st["parents"], st["new"] = _i32(_nums(case["parents"])), _i32(_nums(case["new"]))


def _prepare_compact(case, gen, st):
    rows, at = [], 0
    for x in _nums(case["len"]):
        held = -(-x // case["page"])
        rows.append(list(range(at, at + held)))
        at += held
    rows[-1][:1] = rows[0][:1] if rows[-1] else []  # two sequences share their first page
    n_pages = case["pages"]
    order = torch.randperm(n_pages, generator=gen, device="cuda").tolist()
    _caches(case, st, n_pages, gen)
    # pages that no sequence has, but somebody else (a prompt that is kept for later)
    _prepare_pages(case, st, rows, n_pages, order, max(map(len, rows)) + 2, order[at:at + case["kept"]])
    st["moved"] = torch.empty(n_pages, dtype=torch.int32, device="cuda")
    st["used"] = torch.empty(1, dtype=torch.int32, device="cuda")


def _handles(case, st):
    """The framework's descriptions of a search or of a cache, which a program makes once for its buffers."""
    from paper_2406_14898_gb300 import flglm as F
    if case["kind"] in ("select", "trace"):
        st["search"] = F.beam_search(case["clients"], case["beams"], case.get("vocab", 130528), case["steps"],
                                     eos=case.get("eos", 2), length_penalty=case["penalty"],
                                     early=case.get("early", False))
        st["from"] = F.beam_state(**st["state"])
        st["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        if case["kind"] == "select":
            st["to"] = F.beam_state(**st["next"])
            st["workspace"] = torch.zeros(F.fl_k_beam_workspace(st["search"]) // 4, dtype=torch.int32, device="cuda")
        return
    one = st["k"][0]
    st["caches"] = F.kv_caches([F.kv_cache(k, v, st["n_pages"], case["page"], case["heads"], case["head_dim"],
                                           dtype=F.FL_DT_F16 if case["dtype"] == "f16" else F.FL_DT_BF16,
                                           page_stride=one.stride(0), token_stride=one.stride(1),
                                           head_stride=one.stride(2)) for k, v in zip(st["k"], st["v"])])
    S, width = st["pages"]["table"].shape
    st["from"], st["to"] = (F.kv_pages(S, st["n_pages"], case["page"], width, **st[w]) for w in ("pages", "next"))
    st["workspace"] = torch.zeros(F.fl_k_kv_pages_workspace(st["from"]) // 4, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    st = {"case": case}
    {"select": _prepare_select, "trace": _prepare_trace, "fork": _prepare_fork,
     "compact": _prepare_compact}[case["kind"]](case, gen, st)
    if own:
        _handles(case, st)
    return st


# ------------------------------------------------------------------------------- the plain forms

def _in_order(x):
    """Whole numbers in the order of the floats x; no two of a row alike, the lower index first among equal values."""
    bits = (x + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
    return (bits << 32) + (2 ** 32 - 1 - torch.arange(x.shape[-1], device="cuda"))


def _plain_select(case, st):
    S, B, V, eos, old = case["clients"], case["beams"], case["vocab"], case["eos"], st["state"]
    active = (old["done"] == 0) & (old["steps"] < case["steps"])
    x = st["logits"][:, :V].float()
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    lse = (torch.exp(x - top).sum(-1, dtype=torch.float64).log() + top[:, 0].double()).view(S, B, 1)
    # of each beam's tokens the best that could come into question
    n = min(B + 1, V)
    token = 2 ** 32 - 1 - (_in_order(x).topk(n, -1).values & 0xffffffff)
    c = old["scores"].double()[..., None] + (x.gather(1, token).view(S, B, n).double() - lse)
    c = torch.where(active[:, None, None] & (old["scores"] > -math.inf)[..., None] & torch.isfinite(c), c, -math.inf)
    c, place = c.view(S, B * n).sort(dim=-1, descending=True, stable=True)
    token, beam = token.view(S, B * n).gather(1, place), place // n
    rank = torch.arange(B * n, device="cuda")
    ends = (token == eos) & (c > -math.inf)
    # the next beams: the best that go on
    pick = torch.where(ends, 2 * B * n, rank).sort(-1).indices[:, :B]
    score, live_token, live_beam = c.gather(1, pick), token.gather(1, pick), beam.gather(1, pick)
    score = torch.where(ends.gather(1, pick), -math.inf, score)
    live = score > -math.inf
    own_row = torch.arange(B, device="cuda").expand(S, B)
    fill = eos if eos >= 0 else 0
    live_token = torch.where(live, live_token, fill).int()
    live_beam = torch.where(live, live_beam, own_row).int()
    # hypotheses that end, into the pool
    length = (old["steps"] + 1).double()[:, None] ** case["penalty"]
    ends &= rank < B
    pool = torch.cat([old["end_scores"], torch.where(ends, (c / length).float(), -math.inf)], 1)
    pool, at = pool.sort(dim=-1, descending=True, stable=True)
    pool, at = pool[:, :B], at[:, :B]
    some = pool > -math.inf
    end_steps = torch.cat([old["end_steps"], old["steps"][:, None].expand(S, B * n)], 1).gather(1, at)
    end_beams = torch.cat([old["end_beams"], beam.int()], 1).gather(1, at)
    none = ~live.any(1)
    beaten = pool[:, -1] >= (score[:, :1] / length).float()[:, 0]
    done = (pool[:, -1] > -math.inf) & (beaten | case["early"]) | none
    a = active[:, None]
    t = old["steps"].clamp(max=case["steps"] - 1).long()
    rows = torch.arange(S, device="cuda")
    for name, value in (("trace_tokens", live_token), ("trace_parents", live_beam)):
        st[name][rows, t] = torch.where(a, value, st[name][rows, t])
    return {"tokens": torch.where(a, live_token, fill).int(),
            "parents": torch.where(a & live, live_beam + rows[:, None] * B, -1).int(),
            "scores": torch.where(a, score.float(), old["scores"]), "steps": old["steps"] + active.int(),
            "done": torch.where(active, done.int(), old["done"]),
            "end_scores": torch.where(a, pool, old["end_scores"]),
            "end_steps": torch.where(a, torch.where(some, end_steps, 0), old["end_steps"]),
            "end_beams": torch.where(a, torch.where(some, end_beams, 0), old["end_beams"]),
            "trace_tokens": st["trace_tokens"], "trace_parents": st["trace_parents"]}


def _plain_trace(case, st):
    S, B, T, n, old = case["clients"], case["beams"], case["steps"], case["best"], st["state"]
    steps = old["steps"][:, None].expand(S, B)
    live = torch.where((old["done"] == 0)[:, None] & (steps > 0), old["scores"].double(), -math.inf)
    live = (live / steps.clamp(min=1).double() ** case["penalty"]).float()
    score, at = torch.cat([old["end_scores"], live], 1).sort(dim=-1, descending=True, stable=True)
    score, at = score[:, :n], at[:, :n]
    some, ended = score > -math.inf, at < B
    before = torch.cat([old["end_steps"], steps], 1).gather(1, at)       # tokens of its chain
    beam = torch.cat([old["end_beams"], torch.arange(B, device="cuda").expand(S, B)], 1).gather(1, at).long()
    length = torch.where(some, before + ended.int(), 0)
    # the beam after each step: compositions of the steps' parents, of twice as many steps each time
    t = torch.arange(T, device="cuda")
    inside = t < before[..., None]                                       # [S, n, T]
    same = torch.arange(B, device="cuda")
    maps = torch.where(inside[..., None], st["trace_parents"].long()[:, None], same)
    d = 1
    while d < T:
        maps = torch.cat([maps[:, :, :-d].gather(3, maps[:, :, d:]), maps[:, :, -d:]], 2)
        d *= 2
    chain = torch.cat([maps[:, :, 1:].gather(3, beam[..., None, None].expand(S, n, T - 1, 1))[..., 0], beam[..., None]], 2)
    token = st["trace_tokens"].gather(2, chain.transpose(1, 2)).transpose(1, 2)
    token = torch.where(inside & some[..., None], token, PAD)
    token = torch.where((t == before[..., None]) & (ended & some)[..., None], 2, token)
    return {"tokens": token.contiguous(), "lens": length.int(), "scores": score}


PAD = -1


def _pages_of(lens, page):
    return (lens + page - 1) // page


def _counts(pages, n_pages):
    return torch.bincount(pages.long(), minlength=n_pages).to(torch.int32)


def _plain_fork(case, st):
    page, n_pages, old = case["page"], st["n_pages"], st["pages"]
    S, W = old["table"].shape
    parent, new = st["parents"].long(), st["new"]
    lens = torch.where(parent >= 0, old["lens"][parent.clamp(min=0)], 0)
    after = (lens + new).clamp(min=0)
    held, want = _pages_of(lens, page)[:, None], _pages_of(after, page)[:, None]
    i = torch.arange(W, device="cuda")
    row = torch.where(i < torch.minimum(held, want), old["table"][parent.clamp(min=0)], -1)
    gone = torch.where(i < _pages_of(old["lens"], page)[:, None], old["table"], -1)
    refs = old["refs"] + _counts(row[row >= 0], n_pages) - _counts(gone[gone >= 0], n_pages)
    # whoever is about to write a partly filled page that others have gets a copy of it
    last = row.gather(1, (held - 1).clamp(min=0).long())[:, 0].long()
    writes = (new > 0) & (lens % page > 0)
    writers = _counts(last[writes], n_pages)
    s = torch.arange(S, device="cuda")
    lowest = torch.full((n_pages,), S, device="cuda").scatter_reduce(0, last[writes], s[writes], "amin")
    at = last.clamp(min=0)
    copied = writes & ~((refs[at] == writers[at]) & (lowest[at] == s))
    first = held - copied.int()[:, None]
    fresh = (new > 0)[:, None] & (i >= first) & (i < want)
    count = fresh.sum(1)
    free = (refs == 0).nonzero()[:, 0]
    row = torch.where(fresh, free[((count.cumsum(0) - count)[:, None] + i - first).clamp(0, len(free) - 1)].int(), row)
    refs += _counts(row[fresh], n_pages) - _counts(last[copied], n_pages)
    to = row.gather(1, (held - 1).clamp(min=0).long())[:, 0].long()
    c, slot = (torch.arange(page, device="cuda") < (lens % page)[copied][:, None]).nonzero(as_tuple=True)
    src, dst = last[copied][c], to[copied][c]
    for x in (st["k"], st["v"]):
        x[:, dst, slot] = x[:, src, slot]
    return {"lens": after.int(), "table": row.int(), "refs": refs, "k": st["k"], "v": st["v"]}


def _plain_compact(case, st):
    old, n_pages = st["pages"], st["n_pages"]
    busy = old["refs"] > 0
    used = busy.sum()
    p = torch.arange(n_pages, device="cuda")
    src, dst = (busy & (p >= used)).nonzero()[:, 0], (~busy & (p < used)).nonzero()[:, 0]
    moved = torch.where(busy, p, -1)
    moved[src] = dst
    refs = torch.where(p < used, old["refs"], 0)
    refs[dst] = old["refs"][src]
    held = torch.arange(old["table"].shape[1], device="cuda") < _pages_of(old["lens"], case["page"])[:, None]
    table = torch.where(held, moved[old["table"].clamp(min=0).long()], -1)
    for x in (st["k"], st["v"]):
        x[:, dst] = x[:, src]
    return {"lens": old["lens"], "table": table.int(), "refs": refs.int(), "moved": moved.int(), "used": used.int().view(1),
            "k": st["k"], "v": st["v"]}


# ------------------------------------------------------------------------------- one pass

def _own(case, st):
    from paper_2406_14898_gb300 import flglm as F
    if case["kind"] == "select":
        dtype = {"bf16": F.FL_DT_BF16, "f16": F.FL_DT_F16, "f32": F.FL_DT_F32}[case["dtype"]]
        F.fl_k_beam_step(st["search"], st["from"], st["to"], st["logits"], st["trace_tokens"], st["trace_parents"],
                         st["tokens"], st["parents"], st["workspace"], st["status"], dtype=dtype, ld=case["row"])
        return {"tokens": st["tokens"], "parents": st["parents"], **st["next"], "trace_tokens": st["trace_tokens"],
                "trace_parents": st["trace_parents"]}
    if case["kind"] == "trace":
        F.fl_k_beam_trace(st["search"], st["from"], st["trace_tokens"], st["trace_parents"], case["best"], PAD,
                          st["out_tokens"], st["out_lens"], st["out_scores"], st["status"])
        return {"tokens": st["out_tokens"], "lens": st["out_lens"], "scores": st["out_scores"]}
    if case["kind"] == "fork":
        F.fl_k_kv_fork(st["caches"], st["from"], st["to"], st["parents"], st["new"], st["workspace"], st["status"])
        return {**st["next"], "k": st["k"], "v": st["v"]}
    F.fl_k_kv_compact(st["caches"], st["from"], st["to"], st["moved"], st["used"], st["workspace"], st["status"])
    return {**st["next"], "moved": st["moved"], "used": st["used"], "k": st["k"], "v": st["v"]}


PLAIN = {"select": _plain_select, "trace": _plain_trace, "fork": _plain_fork, "compact": _plain_compact}


def run(state):
    return (_own if own else PLAIN[state["case"]["kind"]])(state["case"], state)


# ------------------------------------------------------------------------------- the least work

def work(case):
    if case["kind"] == "select":
        rows = (case["clients"] - case["done"]) * (1 if case["first"] else case["beams"])
        each = case["clients"] * case["beams"]
        # the logits of the live beams; state in and out, trace, tokens and parents
        return {"bytes": rows * case["vocab"] * (4 if case["dtype"] == "f32" else 2) + each * (8 * 4 + 16) + 16 * case["clients"],
                "flops": 4 * rows * case["vocab"]}
    if case["kind"] == "trace":
        S, B, T, n = case["clients"], case["beams"], case["steps"], case["best"]
        # steps are half of the room on average: their parents, a token a step, the rows of tokens
        return {"bytes": S * (T // 2 * (min(B, n) * 4 + 4 * n) + 4 * n * T) + S * B * 16 + S * n * 8, "flops": S * n * T}
    page, wide = case["page"], 4 * case["blocks"] * case["heads"] * case["head_dim"]
    lens = _nums(case["len"])
    if case["kind"] == "compact":
        held = sum(-(-x // page) for x in lens)
        busy = held + case["kept"] - (1 if len(lens) > 1 and lens[0] and lens[-1] else 0)
        moves = busy * (case["pages"] - busy) // case["pages"]  # of pages in no order
        return {"bytes": 2 * moves * page * wide + 8 * held + 12 * case["pages"] + 8 * len(lens), "flops": held}
    before, after = _grown(case)
    rows, _ = _rows_pages(case)
    parents, new = _nums(case["parents"]), _nums(case["new"])
    have, writers = {}, {}
    for s, (p, x, y, n) in enumerate(zip(parents, before, after, new)):
        mine = rows[p][:min(-(-x // page), -(-y // page))] if p >= 0 else []
        for q in mine:
            have[q] = have.get(q, 0) + 1
        if n > 0 and x % page:
            writers.setdefault(mine[-1], []).append(x % page)
    copied = sum(sum(w) - (w[0] if have[q] == len(w) else 0) for q, w in writers.items())
    # the tokens that are copied; table entries in and out, holders, lengths, parents
    return {"bytes": 2 * copied * wide + 4 * (sum(-(-x // page) for x in before) + sum(-(-x // page) for x in after)) +
            8 * _pool(case) + 16 * len(lens), "flops": sum(-(-x // page) for x in after)}


# ------------------------------------------------------------------------------- the definitions

def exact(case, seed):
    st = prepare(case, seed)
    return {"select": _exact_select, "trace": _exact_trace, "fork": _exact_fork, "compact": _exact_compact}[case["kind"]](case, st)


def _exact_select(case, st):
    B, V, eos, old = case["beams"], case["vocab"], case["eos"], st["state"]
    x = st["logits"][:, :V]
    scores, ended = old["scores"].double(), old["end_scores"].double()
    for s in range(case["clients"]):
        t = int(old["steps"][s])
        if int(old["done"][s]) or t >= case["steps"]:
            continue
        c = old["scores"][s].double()[:, None] + torch.log_softmax(x[s * B:(s + 1) * B].double(), -1)
        c = torch.where(torch.isnan(c), -math.inf, c)
        go = c.clone()
        found = ended[s].tolist()
        if eos >= 0:
            go[:, eos] = -math.inf
            for b in range(B):
                e = c[b, eos]
                before = (c > e).sum() + (c[:b] == e).sum() + (c[b, :eos] == e).sum()
                if e > -math.inf and int(before) < B:
                    found.append(float(c[b, eos]) / (t + 1) ** case["penalty"])
        ended[s] = torch.tensor(sorted(found, reverse=True)[:B], dtype=torch.float64)
        best = go.flatten().topk(min(B, B * V)).values
        scores[s] = -math.inf
        scores[s, :len(best)] = best
    return {"scores": scores, "end_scores": ended, "tokens": None, "parents": None, "steps": None, "done": None,
            "end_steps": None, "end_beams": None, "trace_tokens": None, "trace_parents": None}


def _exact_trace(case, st):
    old = {k: v.tolist() for k, v in st["state"].items()}
    scores = []
    for s in range(case["clients"]):
        found = old["end_scores"][s]
        if not old["done"][s] and old["steps"][s]:
            found = found + [x / old["steps"][s] ** case["penalty"] for x in old["scores"][s]]
        scores.append((sorted(found, reverse=True) + [-math.inf] * case["best"])[:case["best"]])
    return {"scores": torch.tensor(scores, dtype=torch.float64), "tokens": None, "lens": None}


def _moves(st, moves):
    """The caches after (page, page, tokens) were copied one after another."""
    out = {}
    for w in "kv":
        x = st[w].clone()
        for a, b, n in moves:
            x[:, b, :n] = st[w][:, a, :n]
        out[w] = x
    return out


def _exact_fork(case, st):
    """One sequence after another, with lists."""
    page, lens = case["page"], _nums(case["len"])
    table, refs = st["pages"]["table"].tolist(), st["pages"]["refs"].tolist()
    before, after = _grown(case)
    for s, x in enumerate(lens):
        for p in table[s][:-(-x // page)]:
            refs[p] -= 1
    rows = [table[p][:min(-(-x // page), -(-y // page))] if p >= 0 else []
            for p, x, y in zip(_nums(case["parents"]), before, after)]
    for row in rows:
        for p in row:
            refs[p] += 1
    writers = {}
    for s, (row, x, n) in enumerate(zip(rows, before, _nums(case["new"]))):
        if n > 0 and x % page:
            writers.setdefault(row[-1], []).append(s)
    leave = {s for p, w in writers.items() for s in (w[1:] if refs[p] == len(w) else w)}
    free = iter([p for p, n in enumerate(refs) if n == 0])
    moves = []
    for s, (row, x, y) in enumerate(zip(rows, before, after)):
        if s in leave:
            moves.append((row.pop(), next(free), x % page))
            row.append(moves[-1][1])
        while len(row) < -(-y // page):
            row.append(next(free))
    return _moves(st, moves) | {"lens": None, "table": None, "refs": None}


def _exact_compact(case, st):
    refs = st["pages"]["refs"].tolist()
    busy = [p for p, n in enumerate(refs) if n > 0]
    holes = [p for p in range(len(busy)) if refs[p] == 0]
    moves = list(zip([p for p in busy if p >= len(busy)], holes))
    return _moves(st, [(a, b, case["page"]) for a, b in moves]) | {"lens": None, "table": None, "refs": None, "moved": None,
                                                                  "used": None}
