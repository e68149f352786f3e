"""Paged key / value caches for the tests, and the operators' definitions over them in 64 bits."""
import math

import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}  # half an ulp, relative (8, 11, 24 bits)


def dtype_id(F, dtype):
    return {"bf16": F.FL_DT_BF16, "f16": F.FL_DT_F16, "f32": F.FL_DT_F32}[dtype]


class Paged:
    """Sequences with new[s] new tokens of lens[s] cached ones; unused slots hold `stale`."""

    def __init__(self, F, new, lens, kv_heads, head_dim, page, dtype="bf16", token_major=False, stale=math.nan, seed=0,
                 spare=2, max_new=None, scale=1.0):
        self.F, self.new, self.lens, self.page, self.dtype = F, list(new), list(lens), page, dtype
        self.kv_heads, self.hd = kv_heads, head_dim
        rng = np.random.default_rng(seed)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        held = [-(-x // page) for x in lens]
        self.n_pages = sum(held) + spare
        order = rng.permutation(self.n_pages)
        width = max(held) + 1
        table = np.full((len(lens), width), -7, np.int32)
        at = 0
        for s, n in enumerate(held):
            table[s, :n] = order[at:at + n]
            at += n
        self.table = table
        shape = (self.n_pages, page, kv_heads, head_dim) if token_major else (self.n_pages, kv_heads, page, head_dim)
        self.storage = [torch.full(shape, stale, dtype=DTYPES[dtype], device="cuda") for _ in "kv"]
        # [page, slot, head, dim]
        self.k, self.v = self.storage if token_major else [x.transpose(1, 2) for x in self.storage]
        for s, x in enumerate(lens):
            for i in range(held[s]):
                n = min(page, x - i * page)
                for c in (self.k, self.v):
                    c[int(table[s, i]), :n] = (scale * torch.randn((n, kv_heads, head_dim), generator=self.gen,
                                                                   device="cuda")).to(DTYPES[dtype])
        self.T = sum(new)
        self.cu_host = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.cu = torch.from_numpy(self.cu_host).cuda()
        self.dev_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.dev_table = torch.from_numpy(table).cuda()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.cache = F.kv_cache(self.storage[0], self.storage[1], self.n_pages, page, kv_heads, head_dim,
                                dtype=dtype_id(F, dtype), page_stride=self.k.stride(0), head_stride=self.k.stride(2),
                                token_stride=self.k.stride(1))
        self.batch = F.kv_batch(len(new), self.T, max(new) if max_new is None else max_new, self.cu, self.dev_lens,
                                self.dev_table, width)

    def randn(self, *shape, scale=1.0):
        return (scale * torch.randn(shape, generator=self.gen, device="cuda")).to(DTYPES[self.dtype])

    def rows(self, s, which):
        """Keys or values of sequence s in 64 bits, [lens[s], kv_heads, head_dim]."""
        n = -(-self.lens[s] // self.page)
        pages = torch.from_numpy(self.table[s, :n].astype(np.int64)).cuda()
        return getattr(self, which)[pages].flatten(0, 1)[:self.lens[s]].double()

    def workspace(self, heads):
        return torch.zeros(self.F.fl_k_kv_attention_workspace(heads, self.cache, self.batch) // 4, dtype=torch.int32,
                           device="cuda")


def attention64(p, q, heads, context=None, scale=None):
    """(o, lse, bound): the definition row by row, and sum_u p_u |v_u|, which the rounding of p goes by.
    Keys that a row does not see take no part in it whatever they hold."""
    hd, group = p.hd, heads // p.kv_heads
    scale = 1 / math.sqrt(hd) if scale is None else scale
    o = torch.zeros((p.T, heads, hd), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(o)
    lse = torch.full((heads, p.T), -math.inf, dtype=torch.float64, device="cuda")
    for s, (n, L) in enumerate(zip(p.new, p.lens)):
        if n == 0 or L == 0:
            continue
        k, v = p.rows(s, "k"), p.rows(s, "v")
        c = 0 if context is None else context[s]
        t0 = int(p.cu_host[s])
        sees = [max(0, min(L, max(L - n + i + 1, c))) for i in range(n)]
        qs = q[t0:t0 + n].double()
        finite = bool(torch.isfinite(v).all() and torch.isfinite(k).all())
        for h in range(heads):
            kh, vh = k[:, h // group], v[:, h // group]
            if finite:
                sc = qs[:, h] @ kh.T * scale
                mask = torch.arange(L, device="cuda")[None, :] >= torch.tensor(sees, device="cuda")[:, None]
                sc.masked_fill_(mask, -math.inf)
                z = torch.logsumexp(sc, -1)
                w = torch.exp(sc - torch.where(z == -math.inf, 0.0, z)[:, None])
                lse[h, t0:t0 + n] = z
                o[t0:t0 + n, h] = w @ vh
                size[t0:t0 + n, h] = w @ vh.abs()
            else:
                for i, m in enumerate(sees):
                    if m:
                        sc = kh[:m] @ qs[i, h] * scale
                        z = torch.logsumexp(sc, -1)
                        w = torch.exp(sc - z)
                        lse[h, t0 + i] = z
                        o[t0 + i, h] = w @ vh[:m]
                        size[t0 + i, h] = w @ vh[:m].abs()
    return o, lse, size


def check_attention(p, o, lse, ref, T=None):
    """Tolerances: the output's rounding (half an ulp of o), the weights' (half an ulp of each, so
    half an ulp of sum p |v|; fp16 weights below its normal numbers are off by 2^-25 of the largest, one for each
    key), 2^-14 of sum p |v| for the scores' and exponentials' fp32 rounding (scores of at most 30 and
    their sums' error of some ulps); the log-sum-exp carries only that."""
    ro, rl, size = ref
    u = UNIT[p.dtype]
    low = 2.0 ** -25 * max(p.lens) * float(p.v[torch.isfinite(p.v)].abs().max()) if p.dtype == "f16" else 0.0
    bad = torch.isnan(ro)
    assert torch.equal(torch.isnan(o), bad)
    err = (o.double() - ro).abs()
    tol = 1.01 * u * ro.abs() + 1.01 * u * size + 2.0 ** -14 * size + low + 1e-30
    assert bool(((err <= tol) | bad).all()), float((err / tol)[~bad].max())
    empty = rl == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    assert not o[empty.T].any()
    fine = ~empty & ~torch.isnan(rl)
    assert torch.equal(torch.isnan(lse), torch.isnan(rl))
    assert bool(((lse.double() - rl).abs()[fine] <= 2.0 ** -14 + 2.0 ** -22 * rl.abs()[fine]).all())


def turn64(x, rope, positions, layout, first, rotary, backward=False):
    """Dims [first, first + rotary) of x [T, heads, dim] (64 bits) turned in place by the table's rows."""
    r = rope.double()[positions.long()]
    c, s = r[..., 0][:, None], r[..., 1][:, None]
    s = -s if backward else s
    half = rotary // 2
    ia = torch.arange(half) + first if layout == "half" else 2 * torch.arange(half) + first
    ib = ia + half if layout == "half" else ia + 1
    a, b = x[..., ia].clone(), x[..., ib].clone()
    x[..., ia], x[..., ib] = a * c - b * s, a * s + b * c
