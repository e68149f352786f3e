"""Answering token by token with a trained split model.

A client embeds its new tokens and runs block 0, the server runs blocks 1..N-2, the client runs block N-1, the
final LayerNorm and the LM head and picks the next token: the protocol of the paper's §3.1 without its
backward.  Each part keeps the keys and values of the tokens before in a paged cache, so a call carries only
new tokens: a whole prompt, a part of one, or the one token chosen last.

``BlockStack`` is one part: blocks of a ``Server`` or of a ``Client`` as ``forward`` over packed new
tokens, from the library's entry points (``fl_k_layernorm_fwd``, ``fl_k_gemm``, ``fl_k_kv_append``,
``fl_k_kv_attention``).  Its arithmetic is that of ``fl_server_forward``: queries and keys are turned in the
projection's epilogue, before their one rounding.

    python -m paper_2406_14898_gb300.generate --tokens 16

runs a small split model with randomly initialised weights: three clients with prompts of different
lengths answer together; with ``--beams 4`` each keeps its four likeliest answers under way (``Generator.beam_search``), whose
sequences share the pages of what they have in common.
"""
from __future__ import annotations

import argparse
import contextlib
import copy
from typing import List, Optional, Sequence

import torch

from . import flglm as F

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def _stream() -> dict:
    """Where torch's own work goes: the library's calls between follow it there."""
    return {"stream": torch.cuda.current_stream()}


class Pages:
    """Which pages of the caches belong to which sequence; one table for every block of a stack."""

    def __init__(self, n_pages: int, page_size: int, n_seqs: int, max_tokens: int):
        self.page_size, self.free = page_size, list(range(n_pages - 1, -1, -1))
        self.held: List[List[int]] = [[] for _ in range(n_seqs)]
        self.lens = [0] * n_seqs
        self.table = torch.full((n_seqs, max(1, -(-max_tokens // page_size))), -1, dtype=I32)

    def extend(self, new: Sequence[int]):
        """Room for new[s] more tokens of each sequence; a refusal changes nothing."""
        need = [-(-(x + n) // self.page_size) for x, n in zip(self.lens, new)]
        for s, pages in enumerate(need):
            if pages > self.table.shape[1]:
                raise ValueError(f"sequence {s} is longer than {self.table.shape[1] * self.page_size} tokens")
        if sum(max(0, pages - len(held)) for pages, held in zip(need, self.held)) > len(self.free):
            raise MemoryError("no page is free")
        for s, n in enumerate(new):
            while len(self.held[s]) < need[s]:
                self.table[s, len(self.held[s])] = self.free[-1]
                self.held[s].append(self.free.pop())
            self.lens[s] += n

    def shorten(self, new: Sequence[int]):
        """Takes back what an extend by `new`, the last one, gave."""
        for s, n in reversed(list(enumerate(new))):
            self.lens[s] -= n
            while len(self.held[s]) > -(-self.lens[s] // self.page_size):
                self.free.append(self.held[s].pop())
                self.table[s, len(self.held[s])] = -1

    def drop(self, s: int):
        """Forgets sequence s; its pages serve others, uncleared."""
        self.free += self.held[s]
        self.held[s], self.lens[s] = [], 0
        self.table[s] = -1


class SharedPages:
    """The pages of a stack whose sequences share them, from a ``Pages`` on: which, how long and how many have each stays on the
    device (``fl_k_kv_fork``), before and after the last step in turn."""

    def __init__(self, pages: Pages, caches: Sequence["F.fl_kv_cache"]):
        n, width = pages.table.shape
        self.n_pages = len(pages.free) + sum(len(h) for h in pages.held)
        refs = torch.zeros(self.n_pages, dtype=I32)
        for h in pages.held:
            refs[h] += 1
        now = {"lens": torch.tensor(pages.lens, dtype=I32).cuda(), "table": pages.table.cuda(), "refs": refs.cuda()}
        self.sides = [now, {k: torch.empty_like(v) for k, v in now.items()}]
        self.structs = [F.kv_pages(n, self.n_pages, pages.page_size, width, **side) for side in self.sides]
        # a call takes so many of them; calls from the same sides leave the same pages
        self.caches = [F.kv_caches(caches[i:i + F.FL_KV_MAX_CACHES]) for i in range(0, len(caches), F.FL_KV_MAX_CACHES)]
        self.workspace = torch.zeros(F.fl_k_kv_pages_workspace(self.structs[0]) // 4, dtype=I32, device="cuda")
        self.cu = torch.arange(n + 1, dtype=I32, device="cuda")
        self.one = torch.ones(n, dtype=I32, device="cuda")

    def step(self, parents: torch.Tensor, status: torch.Tensor) -> "F.fl_kv_batch":
        """Every sequence follows its parent (device int32, -1: none) and gets room for a token: the batch of those."""
        for caches in self.caches:
            F.fl_k_kv_fork(caches, *self.structs, parents, self.one, self.workspace, status, **_stream())
        self.sides.reverse()
        self.structs.reverse()
        now = self.sides[0]
        n, width = now["table"].shape
        return F.kv_batch(n, n, 1, self.cu, now["lens"], now["table"], width)


class BlockStack:
    """The blocks of one part of the model, with a key / value cache each, on the current CUDA device."""

    def __init__(self, cfg: "F.fl_server_cfg", blocks, n_seqs: int, max_tokens: int, page_size: int = 64,
                 n_pages: Optional[int] = None):
        """cfg: the shapes (of ``make_cfg``); blocks: for each a function tensor id -> fp32 numpy values
        (``FL_T_*``); max_tokens: most tokens of a sequence, its prefix included (in whole pages)."""
        c = self.cfg = cfg
        H, Fh, P = c.hidden, c.ffn_hidden, c.prefix_len
        self.rdim = c.rotary_dim or c.head_dim // 2

        def dev(x, *shape):
            return torch.from_numpy(x).cuda().view(*shape)

        self.blocks = []
        for get in blocks:
            b = {"w": [dev(get(t), *s).to(BF16) for t, s in ((F.FL_T_WQKV, (3 * H, H)), (F.FL_T_WDENSE, (H, H)),
                                                             (F.FL_T_WUP, (Fh, H)), (F.FL_T_WDOWN, (H, Fh)))],
                 "b": [dev(get(t), -1) for t in (F.FL_T_BQKV, F.FL_T_BDENSE, F.FL_T_BUP, F.FL_T_BDOWN)],
                 "ln": [dev(get(t), H) for t in (F.FL_T_LN1_G, F.FL_T_LN1_B, F.FL_T_LN2_G, F.FL_T_LN2_B)],
                 "prefix": [dev(get(t), P, H).to(BF16) for t in (F.FL_T_PREFIX_K, F.FL_T_PREFIX_V)] if P else None}
            self.blocks.append(b)
        self._make_room(n_seqs, max_tokens, page_size, n_pages)

    def _make_room(self, n_seqs, max_tokens, page_size, n_pages):
        c, width = self.cfg, -(-max_tokens // page_size)
        self.max_tokens, self.page_size = max_tokens, page_size
        self.n_pages = n_seqs * width if n_pages is None else n_pages
        self.pages = Pages(self.n_pages, page_size, n_seqs, max_tokens)
        self.shared = None
        for b in self.blocks:  # handed out uncleared
            b["kv"] = [torch.empty((self.n_pages, c.n_heads, page_size, c.head_dim), dtype=BF16, device="cuda") for _ in "kv"]
            b["cache"] = F.kv_cache(b["kv"][0], b["kv"][1], self.n_pages, page_size, c.n_heads, c.head_dim)
        self.max_pos = width * page_size + 1  # of any token that its table row has room for
        self.rope = torch.empty((self.max_pos, self.rdim // 2, 2), device="cuda")
        F.fl_k_rotary_table(self.max_pos, self.rdim, c.rope_base, self.rope, **_stream())
        self.status = torch.zeros(1, dtype=I32, device="cuda")
        self.workspace = None
        self.context = [0] * n_seqs   # context lengths, prefix included; 0: plainly causal
        self.mask_pos = [0] * n_seqs
        torch.cuda.current_stream().synchronize()  # whichever stream uses them

    def with_sequences(self, n_seqs: int) -> "BlockStack":
        """A stack of the same weights (not copied) with caches of its own for n_seqs sequences."""
        other = copy.copy(self)
        other.blocks = [dict(b) for b in self.blocks]
        other._make_room(n_seqs, self.max_tokens, self.page_size, None)
        return other

    @classmethod
    def from_server(cls, srv: "F.Server", n_seqs: int, max_tokens: int, replica: Optional[int] = None, **kw):
        """replica: which one of a handle that holds several (required there: they differ until they are averaged)."""
        if replica is None:
            if srv.cfg.n_replicas > 1:
                raise ValueError(f"the server holds {srv.cfg.n_replicas} replicas: which one answers?")
            replica = 0
        return cls(srv.cfg, [lambda t, b=b: srv.get_replica_param(replica, b, t) for b in range(srv.cfg.n_blocks)], n_seqs,
                   max_tokens, **kw)

    @classmethod
    def from_client(cls, client: "F.Client", part: int, n_seqs: int, max_tokens: int, **kw):
        """part: FL_CP_BOTTOM or FL_CP_TOP."""
        return cls(client.cfg.block, [lambda t: client.get_param(part, t)], n_seqs, max_tokens, **kw)

    def start(self, s: int, context_len: int = 0, mask_pos: Optional[int] = None):
        """A new sequence in place s: its first context_len tokens see each other (GLM blank infilling, §4.1.1, the
        mask token at mask_pos or last among them) and the rest follow causally."""
        P = self.cfg.prefix_len
        if context_len < 0 or (context_len and mask_pos is not None and not 0 <= mask_pos < context_len):
            raise ValueError(f"a context of {context_len} tokens with its mask at {mask_pos}")
        self._alone()
        self.pages.drop(s)
        self.context[s] = context_len + P if context_len else 0
        self.mask_pos[s] = context_len - 1 if mask_pos is None else mask_pos
        if P:  # the P-tuning prefix takes the first places of the cache; its keys are not turned
            with self._extended([P if i == s else 0 for i in range(len(self.context))]) as batch:
                for b in self.blocks:
                    F.fl_k_kv_append(b["cache"], batch, self.cfg.n_heads, None, *b["prefix"], None, None, 0, self.status,
                                     **_stream())

    def _alone(self):
        if self.shared is not None:
            raise ValueError("the sequences share their pages: `follow` goes on with them")

    @contextlib.contextmanager
    def _extended(self, new):
        """The batch of new[s] more tokens of each sequence, which are theirs unless something raises meanwhile."""
        self.pages.extend(new)
        try:
            cu = [0]
            for n in new:
                cu.append(cu[-1] + n)
            keep = [torch.tensor(cu, dtype=I32).cuda(), torch.tensor(self.pages.lens, dtype=I32).cuda(),
                    self.pages.table.cuda()]
            yield F.kv_batch(len(new), cu[-1], max(new), *keep, self.pages.table.shape[1])
        except BaseException:
            self.pages.shorten(new)
            raise

    def _positions(self, new):
        """The two position streams of the new tokens, (i, 0) in the context, (mask, 1 ..) in the span, and the sequences' contexts."""
        first, second = [], []
        for s, n in enumerate(new):
            c = self.context[s] - self.cfg.prefix_len if self.context[s] else 0
            for i in range(self.pages.lens[s] - n - self.cfg.prefix_len, self.pages.lens[s] - self.cfg.prefix_len):
                span = c > 0 and i >= c
                first.append(self.mask_pos[s] if span else i)
                second.append(i - c + 1 if span else 0)
        on = [torch.tensor(v, dtype=I32).cuda() for v in (first, second, self.context)]
        return on if any(self.context) else (on[0], None, None)

    def forward(self, x: torch.Tensor, new: Sequence[int]) -> torch.Tensor:
        """x: bf16 [sum(new), hidden], new[s] next tokens of sequence s; returns the blocks' output of them.  A context's
        tokens come in one call, as they see each other (ValueError otherwise).  Runs on torch's current stream.  A call
        that raises has added nothing: it may be repeated."""
        new = list(new)
        if len(new) != len(self.context) or any(n < 0 for n in new):
            raise ValueError(f"new tokens {new} for {len(self.context)} sequences")
        if not x.is_cuda or x.shape != (sum(new), self.cfg.hidden):
            raise ValueError(f"x {tuple(x.shape)} on {x.device} for {sum(new)} new tokens of {self.cfg.hidden}")
        for s, (n, held, c) in enumerate(zip(new, self.pages.lens, self.context)):
            if n and held < self.cfg.prefix_len:
                raise ValueError(f"sequence {s} has not been started: its prefix is not there")
            if n and held < c and held + n < c:
                raise ValueError(f"sequence {s}: {n} tokens of a context of {c - self.cfg.prefix_len}, which come in one call")
        self._alone()
        if not any(new):
            return x.to(BF16)
        with self._extended(new) as batch:
            return self._run(x, batch, *self._positions(new))

    def follow(self, x: torch.Tensor, parents: torch.Tensor) -> torch.Tensor:
        """x: bf16 [sequences, hidden], one token behind each; sequence s first becomes what sequence parents[s] was (device int32, -1:
        an empty one, without a prefix), with its context and mask, as a step of a beam search picks it.  Whole pages are shared, a
        partly filled one is copied.  A sequence whose context is not there yet is not followed (RuntimeError).  From the first such
        call on the pages are kept on the device, and ``forward`` is refused.  A call that raises has spoilt the sequences."""
        n, c = len(self.context), self.cfg
        if not x.is_cuda or x.shape != (n, c.hidden):
            raise ValueError(f"x {tuple(x.shape)} on {x.device} for a token of {c.hidden} behind each of {n} sequences")
        if parents.dtype != I32 or not parents.is_cuda or parents.shape != (n,):
            raise ValueError(f"{parents.dtype} parents {tuple(parents.shape)} on {parents.device}, not int32 [{n}] on the device")
        if self.shared is None:
            self.shared = SharedPages(self.pages, [b["cache"] for b in self.blocks])
            prefix = [c.prefix_len if held >= c.prefix_len else 0 for held in self.pages.lens]
            self.shared.kept = torch.tensor([self.context, self.mask_pos, prefix], dtype=I32).cuda()
        batch = self.shared.step(parents.contiguous(), self.status)
        # what a sequence has of its parent beside the pages (a parent out of range has been told to the status)
        self.shared.kept = torch.where(parents >= 0, self.shared.kept[:, parents.clamp(0, n - 1).long()], 0)
        context, mask, prefix = self.shared.kept
        early = (self.shared.sides[0]["lens"] <= context).any()  # a context's tokens see each other: they come before
        self.status.bitwise_or_(torch.where(early, F.FL_KV_BAD_POSITION, 0).to(I32))
        # as _positions, on the device (no tokens: what a refused step leaves of an empty sequence)
        i = (self.shared.sides[0]["lens"] - 1 - prefix).clamp(min=0)
        if not any(self.context):
            return self._run(x, batch, i.to(I32), None, None)
        own = context - torch.where(context > 0, prefix, 0)
        span = (own > 0) & (i >= own)
        return self._run(x, batch, torch.where(span, mask, i).to(I32), torch.where(span, i - own + 1, 0).to(I32), context)

    def _run(self, x, batch, pos, pos2, context):
        c, T, H, Fh = self.cfg, len(x), self.cfg.hidden, self.cfg.ffn_hidden
        if self.workspace is None:  # the same for every batch
            size = F.fl_k_kv_attention_workspace(c.n_heads, self.blocks[0]["cache"], batch)
            self.workspace = torch.zeros(size // 4, dtype=I32, device="cuda")
        x = x.float().contiguous()
        a, o, g, u = (torch.empty((T, n), dtype=BF16, device="cuda") for n in (H, H, Fh, Fh))
        qkv = torch.empty((T, 3 * H), dtype=BF16, device="cuda")
        stats = torch.empty((2, T), device="cuda")
        status = torch.zeros(1, dtype=I32, device="cuda")
        on = _stream()

        def norm(x, gamma, beta):
            F.fl_k_layernorm_fwd(T, H, x, gamma, beta, c.ln_eps, a, stats[0], stats[1], x_dtype=F.FL_DT_F32, **on)

        def residual(M, K, inp, w, bias, x, gamma, beta):
            """alpha * (LN(x) or x) + inp w^T + bias in fp32."""
            y = torch.empty((T, H), device="cuda")
            ln = dict(ln_mean=stats[0], ln_rstd=stats[1], ln_gamma=gamma, ln_beta=beta) if c.residual_from_ln else {}
            F.gemm(M, H, K, inp, K, 0, w, K, 0, y, H, status=status, epilogue=F.FL_EPI_BIAS_RESID, bias=bias, aux=x,
                   ld_aux=H, aux_dtype=F.FL_DT_F32, d_dtype=F.FL_DT_F32, alpha=c.residual_alpha, **ln, **on)
            return y

        for b in self.blocks:
            (w_qkv, w_dense, w_up, w_down), (b_qkv, b_dense, b_up, b_down) = b["w"], b["b"]
            norm(x, *b["ln"][:2])
            F.gemm(T, 3 * H, H, a, H, 0, w_qkv, H, 0, qkv, 3 * H, status=status, epilogue=F.FL_EPI_BIAS_ROPE, bias=b_qkv,
                   pos=pos, pos2=pos2, rope_tab=self.rope, n_heads=c.n_heads, head_dim=c.head_dim,
                   rotary_dim=self.rdim, **on)
            q = qkv.data_ptr()
            F.fl_k_kv_append(b["cache"], batch, c.n_heads, None, q + 2 * H, q + 4 * H, None, None, 0, self.status,
                             ldk=3 * H, ldv=3 * H, **on)
            F.fl_k_kv_attention(b["cache"], batch, c.n_heads, q, o, self.workspace, self.status, context_lens=context,
                                ldq=3 * H, **on)
            h = residual(T, H, o, w_dense, b_dense, x, *b["ln"][:2])
            norm(h, *b["ln"][2:])
            F.gemm(T, Fh, H, a, H, 0, w_up, H, 0, g, Fh, status=status, epilogue=F.FL_EPI_BIAS_GELU, bias=b_up, aux_out=u,
                   ld_aux_out=Fh, **on)
            x = residual(T, Fh, g, w_down, b_down, h, *b["ln"][2:])
        bits, cache_bits = int(status.item()), int(self.status.item())
        if bits or cache_bits:
            self.status.zero_()
            self.workspace.zero_()  # not valid after a wait that gave up
            raise RuntimeError(f"generation: device status {bits}, cache status {cache_bits}")
        return x.to(BF16)


class Generator:
    """Clients that answer together: each has its own ends of the model, the server serves all in one call.  The weights
    are those of the handles when it is made; one that trains on needs a new generator."""

    def __init__(self, clients: Sequence["F.Client"], server: "F.Server", max_tokens: int, replica: Optional[int] = None):
        """replica: as in ``BlockStack.from_server``."""
        self.clients, n = list(clients), len(clients)
        self.server = BlockStack.from_server(server, n, max_tokens, replica)
        self.bottom = [BlockStack.from_client(c, F.FL_CP_BOTTOM, 1, max_tokens) for c in clients]
        self.top = [BlockStack.from_client(c, F.FL_CP_TOP, 1, max_tokens) for c in clients]
        self.ends = []
        for c in clients:
            H, V = c.cfg.block.hidden, c.cfg.vocab
            head = torch.zeros((-(-V // 128) * 128, H), dtype=BF16, device="cuda")  # rows in whole GEMM tiles
            head[:V] = torch.from_numpy(c.get_param(F.FL_CP_HEAD, 0)).cuda().view(V, H).to(BF16)
            self.ends.append({"embed": torch.from_numpy(c.get_param(F.FL_CP_EMBED, 0)).cuda().view(V, H).to(BF16),
                              "head": head, "eps": c.cfg.block.ln_eps,
                              "ln": [torch.from_numpy(c.get_param(F.FL_CP_FINAL_LN, t)).cuda() for t in (0, 1)]})
        torch.cuda.current_stream().synchronize()  # whichever stream uses them

    def start(self, context_lens: Optional[Sequence[int]] = None):
        for k in range(len(self.clients)):
            c = 0 if context_lens is None else context_lens[k]
            self.server.start(k, c)
            self.bottom[k].start(0, c)
            self.top[k].start(0, c)

    def _head(self, e, h: torch.Tensor, z: torch.Tensor, status: torch.Tensor):
        """fp32 logits of the rows h into z [rows, vocab in whole GEMM tiles]."""
        T, H = h.shape
        y, stats = torch.empty_like(h), torch.empty((2, T), device="cuda")
        F.fl_k_layernorm_fwd(T, H, h, *e["ln"], e["eps"], y, stats[0], stats[1], **_stream())
        F.gemm(T, z.shape[1], H, y, H, 0, e["head"], H, 0, z, z.shape[1], status=status, d_dtype=F.FL_DT_F32, **_stream())

    def logits(self, tokens: Sequence[torch.Tensor]) -> List[torch.Tensor]:
        """fp32 logits after each client's new tokens (int32 on the device), [vocab] of the last one.  A call that
        raises has added nothing to any part of the model."""
        tokens = self._checked(tokens)
        done = []
        try:
            return self._logits(tokens, done)
        except BaseException:
            for stack, new in done:
                stack.pages.shorten(new)
            raise

    def _checked(self, tokens):
        if len(tokens) != len(self.clients):
            raise ValueError(f"tokens of {len(tokens)} clients for {len(self.clients)}")
        for k, t in enumerate(tokens):
            if t.dtype != I32 or not t.is_cuda or t.dim() != 1 or not len(t):
                raise ValueError(f"client {k}: {t.dtype} tokens {tuple(t.shape)} on {t.device}, not int32 [1 or more] on the device")
        return [t.contiguous() for t in tokens]

    def _logits(self, tokens, done):
        def forward(stack, x, new):
            y = stack.forward(x, new)
            done.append((stack, new))
            return y

        hs, new = [], [len(t) for t in tokens]
        for c, e, stack, t in zip(self.clients, self.ends, self.bottom, tokens):
            h = torch.empty((len(t), c.cfg.block.hidden), dtype=BF16, device="cuda")
            F.fl_k_embedding_gather(len(t), h.shape[1], t, e["embed"], c.cfg.vocab, h, stack.status, **_stream())
            hs.append(forward(stack, h, [len(t)]))
        mid = forward(self.server, torch.cat(hs), new).split(new)
        out, status = [], torch.zeros(1, dtype=I32, device="cuda")
        for c, e, stack, h in zip(self.clients, self.ends, self.top, mid):
            last = forward(stack, h, [len(h)])[-1:].contiguous()
            z = torch.empty((1, e["head"].shape[0]), device="cuda")
            self._head(e, last, z, status)
            out.append(z[0, :c.cfg.vocab])
        if bits := int(status.item()):
            raise RuntimeError(f"generation: device status {bits} of the LM heads")
        return out

    def greedy(self, prompts: Sequence[torch.Tensor], count: int) -> List[List[int]]:
        """`count` next tokens after each prompt (int32 on the device), the likeliest each time."""
        self.start([len(p) for p in prompts])
        answers: List[List[int]] = [[] for _ in prompts]
        tokens = list(prompts)
        for _ in range(count):
            tokens = [z.argmax().to(I32).view(1) for z in self.logits(tokens)]
            for a, t in zip(answers, tokens):
                a.append(int(t))
        return answers


    def beam_search(self, prompts: Sequence[torch.Tensor], count: int, beams: int, eos: int = -1, length_penalty: float = 1.0,
                    early: bool = False) -> List[List[tuple]]:
        """The `beams` best answers of up to `count` tokens after each prompt (int32 on the device), best first: (tokens, score),
        the score being the summed log-probability over the tokens' number to the power of length_penalty.  eos: a token that
        ends an answer (and is its last); early: as in ``fl_beam_search``.  The prompts' sequences of ``logits`` are left as they are."""
        n, vocab = len(self.clients), self.clients[0].cfg.vocab
        prompts = self._checked(prompts)
        if any(c.cfg.vocab != vocab for c in self.clients):
            raise ValueError("the clients' vocabularies differ")
        if count < 1 or not 1 <= beams <= F.FL_BEAM_MAX:
            raise ValueError(f"{count} tokens with {beams} beams (1 to {F.FL_BEAM_MAX})")
        room = min(x.max_tokens - x.cfg.prefix_len for x in (self.server, *self.bottom, *self.top))
        if any(len(p) + count - 1 > room for p in prompts):
            raise ValueError(f"prompts of {[len(p) for p in prompts]} tokens and {count} more in sequences of {room}")
        # the first sequence of each client's beams has the prompt; the others follow it
        wide = Generator.__new__(Generator)
        wide.clients, wide.ends = self.clients, self.ends
        wide.server = self.server.with_sequences(n * beams)
        wide.bottom, wide.top = ([x.with_sequences(beams) for x in stacks] for stacks in (self.bottom, self.top))
        for k, p in enumerate(prompts):
            for stack, s in ((wide.server, k * beams), (wide.bottom[k], 0), (wide.top[k], 0)):
                stack.start(s, len(p))
        search = F.beam_search(n, beams, vocab, count, eos=eos, length_penalty=length_penalty, early=early)
        state = {"scores": torch.full((n, beams), -float("inf"), device="cuda"),
                 "end_scores": torch.full((n, beams), -float("inf"), device="cuda")}
        state["scores"][:, 0] = 0
        for name, shape in (("steps", n), ("done", n), ("end_steps", (n, beams)), ("end_beams", (n, beams))):
            state[name] = torch.zeros(shape, dtype=I32, device="cuda")
        now = F.beam_state(**state)
        trace = [torch.empty((n, count, beams), dtype=I32, device="cuda") for _ in range(2)]
        tokens, parents = (torch.empty((n, beams), dtype=I32, device="cuda") for _ in range(2))
        workspace = torch.empty(F.fl_k_beam_workspace(search), dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=I32, device="cuda")
        z = torch.zeros((n, beams, self.ends[0]["head"].shape[0]), device="cuda")
        for k, row in enumerate(wide._prompted(prompts, beams)):
            z[k, 0, :vocab] = row
        for t in range(count):
            F.fl_k_beam_step(search, now, now, z, *trace, tokens, parents, workspace, status, ld=z.shape[2], **_stream())
            if t + 1 == count or bool(state["done"].all()):
                break
            wide._followed(tokens, parents, z)
        out = (torch.empty((n, beams, count), dtype=I32, device="cuda"), torch.empty((n, beams), dtype=I32, device="cuda"),
               torch.empty((n, beams), device="cuda"))
        F.fl_k_beam_trace(search, now, *trace, beams, 0, *out, status, **_stream())
        if bits := int(status.item()):
            raise RuntimeError(f"beam search: device status {bits}")
        words, lens, scores = (x.tolist() for x in out)
        return [[(w[:m], x) for w, m, x in zip(words[k], lens[k], scores[k]) if m] for k in range(n)]

    def _prompted(self, prompts, beams):
        """Logits after the prompts, each in the first of its client's sequences."""
        hs, out, status = [], [], torch.zeros(1, dtype=I32, device="cuda")
        for c, e, stack, t in zip(self.clients, self.ends, self.bottom, prompts):
            h = torch.empty((len(t), c.cfg.block.hidden), dtype=BF16, device="cuda")
            F.fl_k_embedding_gather(len(t), h.shape[1], t, e["embed"], c.cfg.vocab, h, stack.status, **_stream())
            hs.append(stack.forward(h, [len(t)] + [0] * (beams - 1)))
        new = [n for t in prompts for n in [len(t)] + [0] * (beams - 1)]
        mid = self.server.forward(torch.cat(hs), new).split([len(t) for t in prompts])
        for c, e, stack, h in zip(self.clients, self.ends, self.top, mid):
            last = stack.forward(h, [len(h)] + [0] * (beams - 1))[-1:].contiguous()
            z = torch.empty((1, e["head"].shape[0]), device="cuda")
            self._head(e, last, z, status)
            out.append(z[0, :c.cfg.vocab])
        if bits := int(status.item()):
            raise RuntimeError(f"generation: device status {bits} of the LM heads")
        return out

    def _followed(self, tokens, parents, z):
        """Logits z [clients, beams, row] after tokens [clients, beams] behind the sequences parents [clients, beams] (rows of the
        server's stack)."""
        beams = tokens.shape[1]
        own = torch.where(parents < 0, -1, parents % beams).to(I32)  # rows of a client's stacks
        hs = []
        for k, (c, e, stack) in enumerate(zip(self.clients, self.ends, self.bottom)):
            h = torch.empty((beams, c.cfg.block.hidden), dtype=BF16, device="cuda")
            F.fl_k_embedding_gather(beams, h.shape[1], tokens[k], e["embed"], c.cfg.vocab, h, stack.status, **_stream())
            hs.append(stack.follow(h, own[k]))
        mid = self.server.follow(torch.cat(hs), parents.view(-1)).split(beams)
        gemm_status = torch.zeros(1, dtype=I32, device="cuda")
        for k, (e, stack, h) in enumerate(zip(self.ends, self.top, mid)):
            self._head(e, stack.follow(h, own[k]), z[k], gemm_status)
        if bits := int(gemm_status.item()):
            raise RuntimeError(f"generation: device status {bits} of the LM heads")


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--tokens", type=int, default=16, help="tokens to answer with")
    ap.add_argument("--prompts", type=int, nargs="+", default=[40, 9, 130], help="prompt lengths, one a client")
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--head-dim", type=int, default=64)
    ap.add_argument("--blocks", type=int, default=2, help="server blocks")
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--beams", type=int, default=0, help="answers under way of a client (0: the likeliest token each time)")
    ap.add_argument("--eos", type=int, default=-1, help="with beams: the token that ends an answer")
    a = ap.parse_args(argv)
    room = max(a.prompts) + a.tokens
    cfg, cc = F.fl_server_cfg(), F.fl_client_cfg()
    F.lib().fl_server_cfg_default(cfg)
    cfg.n_blocks, cfg.hidden, cfg.head_dim, cfg.n_heads = a.blocks, a.hidden, a.head_dim, a.hidden // a.head_dim
    cfg.rotary_dim, cfg.ffn_hidden, cfg.max_tokens = 0, 4 * a.hidden, room
    cfg.residual_alpha = (2.0 * (a.blocks + 2)) ** 0.5
    F.lib().fl_client_cfg_default(cc)
    cc.block, cc.vocab = cfg, a.vocab
    cc.block.n_blocks = 1
    clients = [F.Client(cc, a.seed + 1) for _ in a.prompts]  # the same model, as after averaging
    gen = torch.Generator().manual_seed(a.seed)
    prompts = [torch.randint(a.vocab, (n,), generator=gen, dtype=I32).cuda() for n in a.prompts]
    generator = Generator(clients, F.Server(cfg, a.seed), room)
    if a.beams:
        found = generator.beam_search(prompts, a.tokens, a.beams, a.eos)
        for k, best in enumerate(found):
            for tokens, score in best:
                print(f"client {k} ({a.prompts[k]} tokens), {score:.4f}: {' '.join(map(str, tokens))}")
        return found
    answers = generator.greedy(prompts, a.tokens)
    for k, x in enumerate(answers):
        print(f"client {k} ({a.prompts[k]} tokens): {' '.join(map(str, x))}")
    return answers


if __name__ == "__main__":
    main()
