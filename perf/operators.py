"""The operators that answer with a trained model, as cases to time and compare.

A client that generates keeps the keys and values of the tokens before in a paged cache and gives each
block a chunk of new tokens: a whole prompt, a part of one, or the one token it has just chosen.

  rotary     rotation of a projection's rows by their positions, or of its gradient back
  append     a chunk's queries rotated, its keys rotated and written into the cache's pages with its values
  attention  a chunk's queries over the cached keys and values of their own sequences

``own`` False: plain torch in 32 bits; True: the framework's entry points
(``paper_2406_14898_gb300.flglm``).  ``exact`` is the definition in 64 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# lengths of the ragged client-batching workload: K = 16 clients in [64, 1024], 10214 tokens
RAGGED = "909 472 683 733 451 742 821 979 72 134 918 166 869 945 732 588"

# (query heads, key / value heads, head_dim): the 6B block, the same sharing each key / value head
# among 4 or 8 query heads, the one-block test workload, a wide group
HEADS = [(32, 32, 128), (32, 8, 128), (32, 4, 128), (4, 4, 64), (16, 2, 64), (16, 1, 128)]


def _nums(text):
    return [int(x) for x in text.split()]


def _join(xs):
    return " ".join(str(x) for x in xs)


# ------------------------------------------------------------------------------- the cases

def listed():
    clients = random.Random(32)
    decode = [clients.randint(64, 4096) for _ in range(32)]
    return [
        # a training call's queries and keys, side by side in the rows of a fused projection
        # (8192 tokens, 32 + 32 heads), half of each head rotated
        {"name": "rotary_qk", "kind": "rotary", "tokens": 8192, "heads": 64, "head_dim": 128, "rotary": 64,
         "row": 12288, "layout": "half", "dtype": "bf16", "backward": False, "max_pos": 2048, "scaling": "none"},
        # the gradient of a projection in 32 bits through an interleaved rotation of whole heads, positions
        # stretched for long contexts, an odd number of tokens
        {"name": "rotary_back_long", "kind": "rotary", "tokens": 4099, "heads": 8, "head_dim": 128, "rotary": 128,
         "row": 1024, "layout": "interleaved", "dtype": "f32", "backward": True, "max_pos": 65536,
         "scaling": "by_parts"},
        # one token of each of 8 clients: the smallest write, where latency counts
        {"name": "append_decode", "kind": "append", "heads": 32, "kv_heads": 32, "head_dim": 128, "rotary": 64,
         "layout": "half", "two_streams": False, "dtype": "bf16", "page": 64, "token_major": False,
         "new": _join([1] * 8), "len": "256 300 77 1 512 1030 255 641"},
        # the prompts of 16 ragged clients, the model's two position streams
        {"name": "append_prompt", "kind": "append", "heads": 32, "kv_heads": 32, "head_dim": 128, "rotary": 64,
         "layout": "half", "two_streams": True, "dtype": "bf16", "page": 64, "token_major": False,
         "new": RAGGED, "len": RAGGED},
        # chunks of few long sequences, shared key / value heads, small token-major pages
        {"name": "append_chunk_f16", "kind": "append", "heads": 32, "kv_heads": 8, "head_dim": 128, "rotary": 128,
         "layout": "interleaved", "two_streams": False, "dtype": "f16", "page": 16, "token_major": True,
         "new": "511 1 0 257 1023", "len": "4000 17 33 8191 1023"},
        # one client's next token after a short prompt: latency
        {"name": "attn_decode_one", "kind": "attention", "heads": 32, "kv_heads": 32, "head_dim": 128,
         "dtype": "bf16", "page": 64, "token_major": False, "glm": False, "new": "1", "len": "300"},
        # the next tokens of 32 clients, contexts from 64 to 4096 tokens
        {"name": "attn_decode_clients", "kind": "attention", "heads": 32, "kv_heads": 32, "head_dim": 128,
         "dtype": "bf16", "page": 64, "token_major": False, "glm": False, "new": _join([1] * 32),
         "len": _join(decode)},
        # the next tokens of few sequences with long contexts, shared key / value heads
        {"name": "attn_decode_long_f16", "kind": "attention", "heads": 32, "kv_heads": 4, "head_dim": 128,
         "dtype": "f16", "page": 256, "token_major": True, "glm": False, "new": "1 1 1 1",
         "len": "65536 40001 50177 65535"},
        # chunks of 8 clients' prompts (256 tokens after 1800 or so)
        {"name": "attn_chunk_clients", "kind": "attention", "heads": 32, "kv_heads": 32, "head_dim": 128,
         "dtype": "bf16", "page": 64, "token_major": False, "glm": False, "new": _join([256] * 8),
         "len": "2056 2056 1801 2300 256 1999 2047 1280"},
        # the whole prompts of 16 ragged clients, context tokens seeing each other
        {"name": "attn_prompt_glm", "kind": "attention", "heads": 32, "kv_heads": 32, "head_dim": 128,
         "dtype": "bf16", "page": 64, "token_major": False, "glm": True, "new": RAGGED, "len": RAGGED},
        # one chunk of a long document, shared key / value heads
        {"name": "attn_chunk_long", "kind": "attention", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "dtype": "bf16", "page": 128, "token_major": False, "glm": False, "new": "2048", "len": "30001"},
        # prompts, answers and idle sequences of odd sizes in one call, narrow heads, the smallest
        # pages; one sequence has nothing in its cache
        {"name": "attn_mixed_64", "kind": "attention", "heads": 16, "kv_heads": 2, "head_dim": 64,
         "dtype": "bf16", "page": 16, "token_major": False, "glm": False,
         "new": "1 700 1 0 5 1 1 333 1 17 1 1", "len": "4097 700 1 50 1029 2333 0 1333 127 17 1025 3777"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "attention", "attention"])
    if kind == "rotary":
        head_dim = rng.choice([64, 128])
        heads = rng.choice([1, 4, 8, 32, 64])
        rotary = rng.choice([head_dim // 4, head_dim // 2, head_dim])
        case = {"kind": kind, "tokens": _log(rng, 1, 8192), "heads": heads, "head_dim": head_dim, "rotary": rotary,
                "row": heads * head_dim + rng.choice([0, 0, 64, 4096]), "layout": rng.choice(["half", "interleaved"]),
                "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "backward": rng.random() < 0.5,
                "max_pos": _log(rng, 16, 65536), "scaling": rng.choice(["none", "linear", "ntk", "by_parts"])}
        while work(case)["bytes"] > work(listed()[0])["bytes"]:
            case["tokens"] //= 2
        return case
    heads, kv_heads, head_dim = rng.choice(HEADS)
    case = {"kind": kind, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim}
    if kind == "append":
        case |= {"rotary": rng.choice([head_dim // 2, head_dim]), "layout": rng.choice(["half", "interleaved"]),
                 "two_streams": False}
        case["two_streams"] = case["rotary"] * 2 == head_dim and rng.random() < 0.5
    else:
        case["glm"] = rng.random() < 0.25
    case |= {"dtype": rng.choice(["bf16", "bf16", "f16"]), "page": rng.choice([16, 32, 64, 128, 256]),
             "token_major": rng.random() < 0.3}
    seqs = _log(rng, 1, 64)
    longest = _log(rng, 16, 32768)
    lens = [_log(rng, max(1, longest // 16), longest) for _ in range(seqs)]
    form = rng.choice(["token", "few", "chunk", "prompt", "mixed"])
    chunk = _log(rng, 2, 2048)
    new = {"token": [1] * seqs, "few": [rng.randint(1, 8) for _ in lens], "chunk": [chunk] * seqs, "prompt": lens,
           "mixed": [rng.choice([0, 1, 1, chunk]) for _ in lens]}[form]
    new = [min(n, x) for n, x in zip(new, lens)]
    if not any(new):
        new[0] = 1
    most = {k: max(work(c)[k] for c in listed() if c["kind"] == kind) for k in ("bytes", "flops")}
    while True:
        case |= {"new": _join(new), "len": _join(lens)}
        w = work(case)
        # no more than the largest listed case, nor than 8 GB of the plain form's padded scores and keys
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] and (
                kind == "append" or (len(lens) * max(new) * max(lens) * heads <= 2e9 and
                                     len(lens) * max(lens) * kv_heads * head_dim <= 2e9)):
            return case
        if len(lens) > 1:
            lens, new = lens[:(len(lens) + 1) // 2], new[:(len(lens) + 1) // 2]
        else:
            lens = [max(1, lens[0] * 2 // 3)]
            new = [max(1, min(lens[0], new[0] * 2 // 3))]
        if not any(new):
            new[0] = 1


# ------------------------------------------------------------------------------- the inputs

def _context(case):
    """Context lengths of the sequences (0: plainly causal): the last eighth of a prompt, at least a
    token, is the answer span."""
    return [x - max(1, x // 8) if case.get("glm") else 0 for x in _nums(case["len"])]


def rope_table(max_pos, rotary, scaling):
    """[position][pair] = (cos, sin), 64 bits: base 10000, positions stretched 4 times by one of the
    published scalings."""
    factor, original = 4.0, max(1, max_pos // 4)
    i = torch.arange(rotary // 2, dtype=torch.float64)
    base, size = 10000.0, 1.0
    if scaling == "ntk":
        base *= factor ** (rotary / (rotary - 2))
    freq = base ** (-2.0 * i / rotary)
    if scaling == "linear":
        freq = freq / factor
    if scaling == "by_parts":
        turns = original * freq / (2 * math.pi)
        keep = ((turns - 1) / 31).clamp(0, 1)
        freq = freq / factor * (1 - keep) + freq * keep
        size = 0.1 * math.log(factor) + 1
    angle = torch.arange(max_pos, dtype=torch.float64)[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], -1) * size


def _paged(case, gen):
    """Cache, page table and packing of a case's sequences; pages are handed out in no order, and what
    their rows past a sequence's end hold is left over from others (NaN here)."""
    page, dtype = case["page"], DTYPES[case["dtype"]]
    new, lens = _nums(case["new"]), _nums(case["len"])
    held = [-(-x // page) for x in lens]
    n_pages = sum(held) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").tolist()
    table = torch.full((len(lens), max(held) + 1), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(held):
        table[s, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    table = table.cuda()
    shape = ((n_pages, page, case["kv_heads"], case["head_dim"]) if case["token_major"] else
             (n_pages, case["kv_heads"], page, case["head_dim"]))
    made = []
    for _ in "kv":
        x = torch.randn(shape, generator=gen, device="cuda", dtype=dtype)
        made.append(x if case["token_major"] else x.transpose(1, 2))  # [page, slot, head, dim]
    for s, x in enumerate(lens):
        if x % page:
            for c in made:
                c[order[sum(held[:s]) + held[s] - 1], x % page:] = math.nan
    cu = torch.zeros(len(new) + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(torch.tensor(new), 0)
    return {"k": made[0], "v": made[1], "table": table, "cu": cu.cuda(), "n_pages": n_pages,
            "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"), "tokens": sum(new), "max_new": max(new),
            "status": torch.zeros(1, dtype=torch.int32, device="cuda")}


def _handles(case, st):
    """The framework's descriptions of the cache and of a batch of sequences, which a program makes once
    for its buffers."""
    from paper_2406_14898_gb300 import flglm as F
    k = st["k"]
    st["cache"] = F.kv_cache(k, st["v"], st["n_pages"], case["page"], case["kv_heads"], case["head_dim"],
                             dtype=F.FL_DT_F16 if case["dtype"] == "f16" else F.FL_DT_BF16, page_stride=k.stride(0),
                             head_stride=k.stride(2), token_stride=k.stride(1))
    st["batch"] = F.kv_batch(len(st["lens"]), st["tokens"], st["max_new"], st["cu"], st["lens"], st["table"],
                             st["table"].shape[1])
    if case["kind"] == "attention":
        size = F.fl_k_kv_attention_workspace(case["heads"], st["cache"], st["batch"])
        st["workspace"] = torch.zeros(size // 4, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]
    st = {"case": case}
    if case["kind"] == "rotary":
        T = case["tokens"]
        st["x"] = torch.randn((T, case["row"]), generator=gen, device="cuda", dtype=dtype)
        st["y"] = torch.empty((T, case["heads"], case["head_dim"]), device="cuda", dtype=dtype)
        st["positions"] = torch.randint(case["max_pos"], (T,), generator=gen, device="cuda", dtype=torch.int32)
        st["rope"] = rope_table(case["max_pos"], case["rotary"], case["scaling"]).float().cuda()
        st["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        return st
    st |= _paged(case, gen)
    T, heads, kv_heads, hd = st["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "append":
        st["qkv"] = torch.randn((T, (heads + 2 * kv_heads) * hd), generator=gen, device="cuda", dtype=dtype)
        st["q_out"] = torch.empty((T, heads, hd), device="cuda", dtype=dtype)
        st["rope"] = rope_table(max(_nums(case["len"])) + 1, case["rotary"], "none").float().cuda()
        seq = torch.repeat_interleave(torch.arange(len(st["lens"]), device="cuda"), st["cu"].diff())
        first = (st["lens"] - st["cu"].diff() - st["cu"][:-1])[seq]
        st["positions"] = (torch.arange(T, device="cuda") + first).to(torch.int32)
        st["block_positions"] = None
        if case["two_streams"]:  # a prompt whose last third is the span: (mask position, 1, 2, ...)
            start = (st["lens"] * 2 // 3)[seq]
            st["block_positions"] = (st["positions"] - start + 1).clamp(min=0).to(torch.int32)
            st["positions"] = torch.minimum(st["positions"], start).to(torch.int32)
    else:
        st["q"] = torch.randn((T, heads, hd), generator=gen, device="cuda", dtype=dtype)
        st["o"] = torch.empty((T, heads, hd), device="cuda", dtype=dtype)
        st["lse"] = torch.empty((heads, T), device="cuda")
        st["context"] = torch.tensor(_context(case), dtype=torch.int32, device="cuda") if case["glm"] else None
    if own:
        _handles(case, st)
    return st


# ------------------------------------------------------------------------------- the plain forms

def _rotated(x, cos, sin, layout):
    """x [T, heads, rotary] turned by cos, sin [T, 1, rotary / 2]."""
    half = x.shape[-1] // 2
    if layout == "half":
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)


def _rotate_head(x, rope, layout, positions, block_positions, sign=1.0):
    rotary = 2 * rope.shape[1]
    r = rope[positions.long()][:, None]
    parts = [_rotated(x[..., :rotary], r[..., 0], sign * r[..., 1], layout)]
    if block_positions is not None:
        r = rope[block_positions.long()][:, None]
        parts.append(_rotated(x[..., rotary:2 * rotary], r[..., 0], sign * r[..., 1], layout))
        rotary *= 2
    return torch.cat(parts + [x[..., rotary:]], -1)


def _plain_rotary(case, st):
    T, heads, hd = case["tokens"], case["heads"], case["head_dim"]
    x = st["x"][:, :heads * hd].reshape(T, heads, hd).float()
    y = _rotate_head(x, st["rope"], case["layout"], st["positions"], None, -1.0 if case["backward"] else 1.0)
    return {"y": y.to(st["x"].dtype)}


def _plain_append(case, st):
    heads, kv_heads, hd, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    x = st["qkv"].float().view(st["tokens"], heads + 2 * kv_heads, hd)
    turned = _rotate_head(x[:, :heads + kv_heads], st["rope"], case["layout"], st["positions"], st["block_positions"])
    count = st["cu"].diff()
    seq = torch.repeat_interleave(torch.arange(len(count), device="cuda"), count, output_size=st["tokens"])
    slot = torch.arange(st["tokens"], device="cuda") + (st["lens"] - count - st["cu"][:-1])[seq]
    where = st["table"][seq, slot // page].long(), slot % page
    dtype = st["qkv"].dtype
    st["k"][where] = turned[:, heads:].to(dtype)
    st["v"][where] = x[:, heads + kv_heads:].to(dtype)
    return {"q": turned[:, :heads].to(dtype), "k": st["k"], "v": st["v"]}


def _plain_attention(case, st):
    heads, kv_heads, hd, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    group, S, n = heads // kv_heads, len(st["lens"]), st["max_new"]
    lens, count = st["lens"], st["cu"].diff()
    longest = st["table"].shape[1] * page
    u = torch.arange(longest, device="cuda")
    held = u < lens[:, None]
    at = st["table"][:, u // page].clamp(min=0).long(), (u % page).expand(S, -1)
    k = st["k"][at].float().masked_fill(~held[..., None, None], 0).permute(0, 2, 3, 1)  # [S, head, dim, key]
    v = st["v"][at].float().masked_fill(~held[..., None, None], 0).transpose(1, 2)      # [S, head, key, dim]
    i = torch.arange(n, device="cuda")
    rows = (st["cu"][:-1, None] + i).clamp(max=st["tokens"] - 1).long()
    q = st["q"][rows].float().view(S, n, kv_heads, group, hd).permute(0, 2, 3, 1, 4).reshape(S, kv_heads, group * n, hd)
    sees = (lens - count)[:, None] + i + 1
    if st["context"] is not None:
        sees = torch.maximum(sees, st["context"][:, None])
    sees = torch.minimum(sees, lens[:, None])
    mask = (u < sees[..., None])[:, None, None]                                        # [S, 1, 1, n, key]
    s = (q @ k).view(S, kv_heads, group, n, longest) * (1 / math.sqrt(hd))
    s = s.masked_fill(~mask, -math.inf)
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    o = (e.view(S, kv_heads, group * n, longest) @ v).view(S, kv_heads, group, n, hd)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (total.log() + torch.where(top == -math.inf, 0.0, top))[..., 0]
    seq = torch.repeat_interleave(torch.arange(S, device="cuda"), count, output_size=st["tokens"])
    j = torch.arange(st["tokens"], device="cuda") - st["cu"][seq]
    return {"o": o.permute(0, 3, 1, 2, 4).reshape(S, n, heads, hd)[seq, j].to(st["q"].dtype),
            "lse": lse.permute(0, 3, 1, 2).reshape(S, n, heads)[seq, j].T.contiguous()}


# ------------------------------------------------------------------------------- one pass

def _own(case, st):
    from paper_2406_14898_gb300 import flglm as F
    layout = F.FL_ROPE_HALF if case.get("layout") == "half" else F.FL_ROPE_INTERLEAVED
    if case["kind"] == "rotary":
        dtype = {"bf16": F.FL_DT_BF16, "f16": F.FL_DT_F16, "f32": F.FL_DT_F32}[case["dtype"]]
        F.fl_k_rotary(case["tokens"], case["heads"], case["head_dim"], case["rotary"], st["x"], st["y"], st["rope"],
                      case["max_pos"], st["positions"], st["status"], dtype=dtype, layout=layout,
                      backward=case["backward"], ldx=case["row"])
        return {"y": st["y"]}
    heads, kv_heads, hd = case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "append":
        row = (heads + 2 * kv_heads) * hd
        q = st["qkv"].data_ptr()
        F.fl_k_kv_append(st["cache"], st["batch"], heads, q, q + 2 * heads * hd, q + 2 * (heads + kv_heads) * hd,
                         st["q_out"], st["rope"], st["rope"].shape[0], st["status"], rotary_dim=case["rotary"],
                         layout=layout, positions=st["positions"], block_positions=st["block_positions"], ldq=row,
                         ldk=row, ldv=row)
        return {"q": st["q_out"], "k": st["k"], "v": st["v"]}
    F.fl_k_kv_attention(st["cache"], st["batch"], heads, st["q"], st["o"], st["workspace"], st["status"],
                        lse=st["lse"], context_lens=st["context"])
    return {"o": st["o"], "lse": st["lse"]}


PLAIN = {"rotary": _plain_rotary, "append": _plain_append, "attention": _plain_attention}


def run(state):
    return (_own if own else PLAIN[state["case"]["kind"]])(state["case"], state)


# ------------------------------------------------------------------------------- the least work

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    hd = case["head_dim"]
    if case["kind"] == "rotary":
        T, n = case["tokens"], case["tokens"] * case["heads"]
        # the rows read and written, the table's rows that can occur, the positions
        return {"bytes": 2 * n * hd * size + 4 * min(T, case["max_pos"]) * case["rotary"] + 4 * T,
                "flops": 3 * n * case["rotary"]}
    new, lens = _nums(case["new"]), _nums(case["len"])
    T, heads, kv_heads = sum(new), case["heads"], case["kv_heads"]
    if case["kind"] == "append":
        streams = 2 if case["two_streams"] else 1
        return {"bytes": 2 * T * (heads + 2 * kv_heads) * hd * size + 4 * T * streams +
                4 * min(T, max(lens) + 1) * case["rotary"] * streams,
                "flops": 3 * T * (heads + kv_heads) * case["rotary"] * streams}
    seen = pairs = 0
    for n, x, c in zip(new, lens, _context(case)):
        sees = [min(x, max(0, x - n + i + 1, c)) for i in range(n)]
        pairs += sum(sees)
        seen += max(sees, default=0)
    # queries, outputs and log-sum-exps, and the keys and values that some query sees
    return {"bytes": 2 * T * heads * hd * size + 4 * T * heads + 2 * seen * kv_heads * hd * size,
            "flops": 4 * pairs * heads * hd}


# ------------------------------------------------------------------------------- the definitions in 64 bits

def _turn64(x, angle_cos, angle_sin, rotary, layout, first):
    """Pairs of dims [first, first + rotary) of x [..., T, heads, dim], as complex numbers."""
    part = x[..., first:first + rotary]
    half = rotary // 2
    even, odd = (part[..., :half], part[..., half:]) if layout == "half" else (part[..., 0::2], part[..., 1::2])
    z = torch.complex(even, odd) * torch.complex(angle_cos, angle_sin)[:, None]
    out = torch.empty_like(part)
    if layout == "half":
        out[..., :half], out[..., half:] = z.real, z.imag
    else:
        out[..., 0::2], out[..., 1::2] = z.real, z.imag
    x[..., first:first + rotary] = out


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "rotary":
        T, heads, hd = case["tokens"], case["heads"], case["head_dim"]
        y = st["x"].double()[:, :heads * hd].reshape(T, heads, hd).clone()
        rope = st["rope"].double()[st["positions"].long()]
        _turn64(y, rope[..., 0], -rope[..., 1] if case["backward"] else rope[..., 1], case["rotary"],
                case["layout"], 0)
        return {"y": y}
    heads, kv_heads, hd, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    new, lens = _nums(case["new"]), _nums(case["len"])
    table = st["table"].tolist()
    if case["kind"] == "append":
        x = st["qkv"].double().view(st["tokens"], heads + 2 * kv_heads, hd)
        turned = x[:, :heads + kv_heads].clone()
        for stream, p in enumerate((st["positions"], st["block_positions"])):
            if p is not None:
                rope = st["rope"].double()[p.long()]
                _turn64(turned, rope[..., 0], rope[..., 1], case["rotary"], case["layout"], stream * case["rotary"])
        k, v, t = st["k"].double(), st["v"].double(), 0
        for s, (n, end) in enumerate(zip(new, lens)):
            at = end - n
            while at < end:  # page by page
                stop = min(end, (at // page + 1) * page)
                p, rows = table[s][at // page], slice(t, t + stop - at)
                k[p, at % page:at % page + stop - at] = turned[rows, heads:]
                v[p, at % page:at % page + stop - at] = x[rows, heads + kv_heads:]
                t, at = t + stop - at, stop
        return {"q": turned[:, :heads], "k": k, "v": v}
    if work(case)["flops"] > 8e12:  # over about 20 seconds in 64 bits
        return None
    o = torch.zeros((st["tokens"], heads, hd), dtype=torch.float64, device="cuda")
    lse = torch.full((heads, st["tokens"]), -math.inf, dtype=torch.float64, device="cuda")
    first = 0
    for s, (n, x, c) in enumerate(zip(new, lens, _context(case))):
        if n and x:
            pages = torch.tensor(table[s][:-(-x // page)], device="cuda")
            keys, values = (st[w][pages].flatten(0, 1)[:x].double() for w in "kv")
            limit = torch.clamp(torch.arange(x - n, x, device="cuda"), min=c - 1)
            unseen = torch.arange(x, device="cuda")[None, :] > limit[:, None]
            for h in range(heads):
                kv = h * kv_heads // heads
                logits = st["q"][first:first + n, h].double() @ keys[:, kv].T / math.sqrt(hd)
                logits[unseen] = -math.inf
                total = torch.logsumexp(logits, -1)
                lse[h, first:first + n] = total
                weights = torch.exp(logits - torch.where(total == -math.inf, 0.0, total)[:, None])
                o[first:first + n, h] = weights @ values[:, kv]
        first += n
    return {"o": o, "lse": lse}
