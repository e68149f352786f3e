"""Rotary positions, the append to a paged cache and the attention over it, against their definitions in
64 bits (GPU only).  Sizes are where these go wrong: one token, none, tiles and pages that end early, rows
that see nothing, heads shared by odd numbers, strides."""
import math

import numpy as np
import pytest
import torch

from tests._gpu import flglm, need_gpu
from tests._kv import DTYPES, UNIT, Paged, attention64, check_attention, dtype_id, turn64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    need_gpu()
    return flglm()


def layout_id(F, layout):
    return {"half": F.FL_ROPE_HALF, "interleaved": F.FL_ROPE_INTERLEAVED}[layout]


# ------------------------------------------------------------------------------- rotary table

def table64(max_pos, rd, base, scaling, factor, original):
    f = base ** (-2.0 * np.arange(rd // 2) / rd)
    size = 1.0
    if scaling == 1:
        f = f / factor
    if scaling == 2:
        f = (base * factor ** (rd / (rd - 2))) ** (-2.0 * np.arange(rd // 2) / rd)
    if scaling == 3:
        keep = np.clip((original * f / (2 * np.pi) - 1) / 31, 0, 1)
        f = f / factor * (1 - keep) + f * keep
        size = 0.1 * math.log(factor) + 1
    ang = np.arange(max_pos)[:, None] * f
    return size * np.stack([np.cos(ang), np.sin(ang)], -1)


@pytest.mark.parametrize("scaling,factor,original", [(0, 1.0, 0), (1, 4.0, 0), (2, 8.0, 0), (3, 4.0, 512), (3, 1.0, 1)])
@pytest.mark.parametrize("max_pos,rd", [(1, 2), (2049, 64), (777, 96)])
def test_rotary_table(F, max_pos, rd, scaling, factor, original):
    if scaling == 2 and rd == 2:
        pytest.skip("the enlarged base needs more than one pair")
    tab = torch.full((max_pos, rd // 2, 2), math.nan, device="cuda")
    F.fl_k_rotary_table(max_pos, rd, 10000.0, tab, scaling=scaling, factor=factor, original_max_pos=original)
    ref = table64(max_pos, rd, 10000.0, scaling, factor, original)
    # one rounding to fp32; the angle (at most 2049) in doubles of two programs may differ in its last bits
    assert np.abs(tab.double().cpu().numpy() - ref).max() <= 2.0 ** -24 * 1.2 + 2049 * 2.0 ** -50


# ------------------------------------------------------------------------------- rotary

def rope_of(F, max_pos, rd):
    tab = torch.empty((max_pos, rd // 2, 2), device="cuda")
    F.fl_k_rotary_table(max_pos, rd, 10000.0, tab, scaling=F.FL_ROPE_SCALE_BY_PARTS, factor=4.0,
                        original_max_pos=max(1, max_pos // 4))
    return tab


def turned_bound(x, dtype):
    """One rounding of the result, and three of fp32 products and sums of |a| + |b| (table entries up to 1.14)."""
    return lambda ref: 1.01 * UNIT[dtype] * ref.abs() + 4 * 2.0 ** -24 * 1.2 * 2 * x.abs().max()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,heads,hd,rd,two", [(1, 1, 16, 16, False), (3, 5, 80, 32, True), (130, 7, 64, 64, False),
                                               (257, 2, 128, 64, True), (33, 3, 256, 128, False),
                                               (65, 4, 48, 16, True)])
def test_rotary_both_directions(F, T, heads, hd, rd, two, dtype, layout):
    gen = torch.Generator(device="cuda").manual_seed(T + hd)
    max_pos = 999
    tab = rope_of(F, max_pos, rd)
    # strided input rows and heads, contiguous output
    x = torch.randn((T, heads, hd + 16), generator=gen, device="cuda").to(DTYPES[dtype])
    pos = torch.randint(max_pos, (T,), generator=gen, device="cuda", dtype=torch.int32)
    pos2 = torch.randint(max_pos, (T,), generator=gen, device="cuda", dtype=torch.int32) if two else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for backward in (False, True):
        y = torch.full((T, heads, hd), math.nan, device="cuda", dtype=DTYPES[dtype])
        F.fl_k_rotary(T, heads, hd, rd, x, y, tab, max_pos, pos, status, block_positions=pos2,
                      dtype=dtype_id(F, dtype), layout=layout_id(F, layout), backward=backward, ldx=x.stride(0),
                      x_head_stride=x.stride(1))
        ref = x[..., :hd].double()
        turn64(ref, tab, pos, layout, 0, rd, backward)
        if two:
            turn64(ref, tab, pos2, layout, rd, rd, backward)
        assert bool(((y.double() - ref).abs() <= turned_bound(x.double(), dtype)(ref)).all())
        assert torch.equal(y[..., rd * (2 if two else 1):], x[..., rd * (2 if two else 1):hd])
        z = x[..., :hd].contiguous()  # in place: the same bits
        F.fl_k_rotary(T, heads, hd, rd, z, z, tab, max_pos, pos, status, block_positions=pos2,
                      dtype=dtype_id(F, dtype), layout=layout_id(F, layout), backward=backward)
        assert torch.equal(z, y)
    assert status.item() == 0


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_gradient_by_differences(F, layout):
    """<dy, R(x + e d) - R(x - e d)> / 2e against <R^T dy, d>: R is linear, so the difference quotient
    has no error but fp32's (|x|, |d| about 1, e = 1: some 2^-24 a product of 32-bit sums taken in 64 bits)."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    T, heads, hd, rd, max_pos = 37, 3, 64, 32, 500
    tab = rope_of(F, max_pos, rd)
    pos = torch.randint(max_pos, (T,), generator=gen, device="cuda", dtype=torch.int32)
    x, d, dy = (torch.randn((T, heads, hd), generator=gen, device="cuda") for _ in range(3))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def R(v, backward=False):
        y = torch.empty_like(v)
        F.fl_k_rotary(T, heads, hd, rd, v, y, tab, max_pos, pos, status, dtype=F.FL_DT_F32,
                      layout=layout_id(F, layout), backward=backward)
        return y.double()

    quotient = (dy.double() * (R(x + d) - R(x - d))).sum() / 2
    inner = (R(dy, True) * d.double()).sum()
    n = T * heads * hd
    assert abs(float(quotient - inner)) <= 16 * 2.0 ** -24 * n ** 0.5 * 8
    assert status.item() == 0


def test_rotary_bad_positions_give_zero_rows(F):
    T, heads, hd, rd, max_pos = 6, 2, 64, 32, 10
    tab = rope_of(F, max_pos, rd)
    x = torch.ones((T, heads, hd), device="cuda", dtype=torch.bfloat16)
    y = torch.full_like(x, math.nan)
    pos = torch.tensor([0, 9, 10, -1, 2 ** 31 - 1, 3], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    F.fl_k_rotary(T, heads, hd, rd, x, y, tab, max_pos, pos, status)
    assert status.item() == F.FL_KV_BAD_POSITION
    assert not y[2:5, :, :rd].any() and bool((y[..., rd:] == 1).all())
    assert bool(torch.isfinite(y).all()) and bool(y[[0, 1, 5]].any(-1).all())
    F.fl_k_rotary(0, heads, hd, rd, x, y, tab, max_pos, pos, status)  # no rows: nothing


# ------------------------------------------------------------------------------- append

APPENDS = [
    # new, lens, heads, kv heads, head_dim, page, token-major
    ([1], [1], 4, 4, 64, 16, False),
    ([1, 1, 1], [256, 17, 1030], 32, 32, 128, 64, False),
    ([0, 7, 0, 0, 131, 1, 0], [5, 7, 0, 33, 300, 128, 9], 6, 2, 128, 32, False),
    ([40, 3], [64, 1000], 8, 1, 64, 16, True),
    ([513], [700], 3, 3, 128, 256, True),
]


@pytest.mark.parametrize("new,lens,heads,kvh,hd,page,token_major", APPENDS)
@pytest.mark.parametrize("layout,part,two,dtype", [("half", 2, True, "bf16"), ("half", 1, False, "f16"),
                                                   ("interleaved", 1, False, "bf16"), ("interleaved", 4, True, "f16")])
def test_append(F, new, lens, heads, kvh, hd, page, token_major, layout, part, two, dtype):
    p = Paged(F, new, lens, kvh, hd, page, dtype, token_major, seed=hd + page)
    rd, row = hd // part, (heads + 2 * kvh) * hd
    max_pos = max(lens) + 1
    tab = rope_of(F, max_pos, rd)
    qkv = p.randn(p.T, heads + 2 * kvh, hd)
    idx = np.concatenate([np.arange(L - n, L) for n, L in zip(new, lens)]).astype(np.int64)
    seq = np.repeat(np.arange(len(new)), new)
    pos = torch.from_numpy(idx.astype(np.int32)).cuda()
    pos2 = torch.randint(max_pos, (p.T,), generator=p.gen, device="cuda", dtype=torch.int32) if two else None
    ref = qkv.double()
    turned = ref[:, :heads + kvh].clone()
    turn64(turned, tab, pos, layout, 0, rd)
    if two:
        turn64(turned, tab, pos2, layout, rd, rd)
    k_want, v_want = p.k.clone(), p.v.clone()
    where = torch.from_numpy(p.table[seq, idx // page].astype(np.int64)).cuda(), torch.from_numpy(idx % page).cuda()
    v_want[where] = qkv[:, heads + kvh:]
    bound = turned_bound(ref, dtype)
    base = qkv.data_ptr()
    size = qkv.element_size()
    # with positions given, and (one stream) found from the sequences
    for given in (True, False):
        q_out = torch.full((p.T, heads, hd), math.nan, device="cuda", dtype=DTYPES[dtype])
        F.fl_k_kv_append(p.cache, p.batch, heads, base, base + heads * hd * size, base + (heads + kvh) * hd * size,
                         q_out, tab, max_pos, p.status, rotary_dim=rd, layout=layout_id(F, layout),
                         positions=pos if given else None, block_positions=pos2, ldq=row, ldk=row, ldv=row)
        assert p.status.item() == 0
        assert bool(((q_out.double() - turned[:, :heads]).abs() <= bound(turned[:, :heads])).all())
        got = p.k[where].double()
        assert bool(((got - turned[:, heads:]).abs() <= bound(turned[:, heads:])).all())
        k_want[where] = p.k[where]
        for a, b in ((p.k, k_want), (p.v, v_want)):  # every other slot as it was (NaN ones too)
            assert torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))
        p.k[where] = 7.0
        p.v[where] = 7.0


def test_append_in_place_and_without_queries_or_rotation(F):
    heads, kvh, hd = 4, 2, 64
    p = Paged(F, [3, 2], [20, 2], kvh, hd, 16, seed=3)
    tab = rope_of(F, 32, 32)
    q, k, v = p.randn(p.T, heads, hd), p.randn(p.T, kvh, hd), p.randn(p.T, kvh, hd)
    out = torch.empty_like(q)
    F.fl_k_kv_append(p.cache, p.batch, heads, q, k, v, out, tab, 32, p.status, rotary_dim=32)
    F.fl_k_kv_append(p.cache, p.batch, heads, q, k, v, q, tab, 32, p.status, rotary_dim=32)
    assert torch.equal(q, out)
    F.fl_k_kv_append(p.cache, p.batch, heads, None, k, v, None, None, 0, p.status)  # as it is: a prefix
    assert torch.equal(p.rows(1, "k"), k[3:].double()) and torch.equal(p.rows(1, "v"), v[3:].double())
    assert torch.equal(p.rows(0, "k")[17:], k[:3].double())
    assert p.status.item() == 0


def test_append_leaves_out_tokens_without_a_slot(F):
    heads, kvh, hd, page = 2, 2, 64, 16
    tab = torch.empty((64, 16, 2), device="cuda")
    F.fl_k_rotary_table(64, 32, 10000.0, tab)
    # sequence 0: more new tokens than cached ones; 1: its page is not in the cache; 2: past its table row
    p = Paged(F, [5, 1, 1, 1], [3, 4, 4, 18], kvh, hd, page, stale=2.0, seed=4)
    bad = p.dev_table.clone()
    bad[1, 0] = p.n_pages
    p.dev_lens[2] = page * p.table.shape[1] + 1
    batch = F.kv_batch(4, p.T, 5, p.cu, p.dev_lens, bad, p.table.shape[1])
    before = p.k.clone(), p.v.clone()
    q, k, v = p.randn(p.T, heads, hd), p.randn(p.T, kvh, hd), p.randn(p.T, kvh, hd)
    out = torch.full_like(q, math.nan)
    pos = torch.zeros(p.T, dtype=torch.int32, device="cuda")
    F.fl_k_kv_append(p.cache, batch, heads, q, k, v, out, tab, 64, p.status, rotary_dim=32, positions=pos)
    assert p.status.item() == F.FL_KV_BAD_PAGE
    before[0][int(p.table[0, 0]), :3], before[1][int(p.table[0, 0]), :3] = k[2:5], v[2:5]
    at = int(p.table[3, 1]), 1
    before[0][at], before[1][at] = k[7], v[7]
    assert torch.equal(p.k, before[0]) and torch.equal(p.v, before[1])
    assert torch.equal(out, q)  # position 0 turns nothing
    # a position out of range: zeros in the turned dims of the query and of the cached key
    p.status.zero_()
    pos[7] = 64
    F.fl_k_kv_append(p.cache, p.batch, heads, q, k, v, out, tab, 64, p.status, rotary_dim=32, positions=pos)
    assert p.status.item() & F.FL_KV_BAD_POSITION
    assert not out[7, :, :32].any() and not p.k[at][:, :32].any() and torch.equal(p.k[at][:, 32:], k[7, :, 32:])


# ------------------------------------------------------------------------------- attention

def run_attention(F, p, heads, context=None, scale=None, q=None, ws=None, lse=True, stream=None):
    q = p.randn(p.T, heads, p.hd) if q is None else q
    o = torch.full((p.T, heads, p.hd), math.nan, device="cuda", dtype=DTYPES[p.dtype])
    l = torch.full((heads, p.T), math.nan, device="cuda") if lse else None
    ctx = None if context is None else torch.tensor(context, dtype=torch.int32, device="cuda")
    ws = p.workspace(heads) if ws is None else ws
    F.fl_k_kv_attention(p.cache, p.batch, heads, q, o, ws, p.status, lse=l, context_lens=ctx,
                        scale=0.0 if scale is None else scale, stream=stream)
    return q, o, l


ATTENTIONS = [
    # new, lens, heads, kv heads, head_dim, page, token-major, context
    ([1], [1], 4, 4, 64, 16, False, None),
    ([1], [300], 32, 32, 128, 64, False, None),
    ([1], [5000], 4, 2, 128, 32, False, None),                                    # one sequence in many parts
    ([1] * 9, [1, 2, 15, 16, 17, 63, 64, 65, 1031], 8, 8, 128, 16, False, None),  # ends around steps and blocks
    ([1, 0, 1, 1], [0, 33, 200, 0], 4, 1, 64, 16, False, None),                   # empty caches, no new tokens
    ([3, 8, 2], [3, 500, 90], 3, 3, 128, 64, True, None),                         # few tokens, causal among them
    ([4, 1], [700, 70], 15, 3, 64, 256, False, None),                             # 5 heads a group
    ([1, 1], [900, 130], 48, 4, 128, 128, False, None),                           # 12 heads a group
    ([40, 1, 129], [40, 777, 300], 6, 6, 128, 32, False, None),                   # chunks
    ([130], [1500], 8, 2, 64, 16, True, None),
    ([257], [257], 2, 2, 128, 64, False, [200]),                                  # a GLM prompt
    ([20, 33, 7], [20, 64, 300], 4, 4, 128, 16, False, [15, 64, 999]),            # contexts around the lengths
    ([7, 5], [3, 0], 2, 2, 64, 16, False, None),                                  # tokens before the cache's first
    ([300, 5], [200, 2], 4, 2, 128, 32, False, None),
    ([3, 1, 90], [3, 500, 90], 120, 3, 64, 32, True, None),                       # 40 heads a group
    ([2, 1], [700, 129], 128, 1, 128, 16, False, None),                           # 128: one token a tile
    ([128, 129, 256, 255], [128, 129, 640, 1000], 2, 1, 128, 128, True, None),    # tiles that end exactly
    ([1] * 300, [(37 * i) % 400 for i in range(300)], 2, 2, 64, 16, False, None),  # more sequences than lanes
    ([1, 17] * 40, [200 + i for i in range(80)], 2, 1, 64, 16, False, [150, 0] * 40),
]


@pytest.mark.parametrize("case", ATTENTIONS, ids=[str(i) for i in range(len(ATTENTIONS))])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attention(F, case, dtype):
    new, lens, heads, kvh, hd, page, token_major, context = case
    p = Paged(F, new, lens, kvh, hd, page, dtype, token_major, seed=sum(lens) + heads)
    q, o, lse = run_attention(F, p, heads, context)
    assert p.status.item() == 0
    check_attention(p, o, lse, attention64(p, q, heads, context))


def test_attention_strides_scale_and_no_lse(F):
    heads, kvh, hd = 6, 3, 128
    p = Paged(F, [2, 70, 1], [100, 70, 900], kvh, hd, 64, seed=11)
    wide = p.randn(p.T, heads + 5, hd)
    o = torch.full((p.T, heads + 1, hd), math.nan, device="cuda", dtype=torch.bfloat16)
    F.fl_k_kv_attention(p.cache, p.batch, heads, wide, o, p.workspace(heads), p.status, scale=-0.2,
                        ldq=wide.stride(0), ldo=o.stride(0))
    ref = attention64(p, wide[:, :heads], heads, scale=-0.2)
    check_attention(p, o[:, :heads], ref[1].float(), ref)
    assert bool(torch.isnan(o[:, heads]).all())


@pytest.mark.parametrize("offset", [0, 8])
def test_attention_more_tokens_than_announced_and_unaligned_rows(F, offset):
    """max_new only chooses the kernel; outputs need 16-byte alignment, not 32."""
    heads, hd = 2, 64
    for new, told in (([70, 3], 1), ([2, 1], 500)):
        p = Paged(F, new, [120, 300], heads, hd, 16, seed=17, max_new=told)
        q = p.randn(p.T, heads, hd)
        room = torch.full((p.T * (heads * hd + 8) + offset,), math.nan, device="cuda", dtype=torch.bfloat16)
        lse = torch.empty((heads, p.T), device="cuda")
        F.fl_k_kv_attention(p.cache, p.batch, heads, q, room[offset:], p.workspace(heads), p.status, lse=lse,
                            ldo=heads * hd + 8)
        rows = room[offset:].view(p.T, heads * hd + 8)
        check_attention(p, rows[:, :heads * hd].reshape(p.T, heads, hd), lse, attention64(p, q, heads))
        assert bool(torch.isnan(rows[:, heads * hd:]).all()) and p.status.item() == 0


@pytest.mark.parametrize("new", [[1, 1], [1, 40]])
def test_attention_lengths_out_of_range(F, new):
    """Too long a length counts as the table row's room, a negative one as none."""
    p = Paged(F, new, [40, 64], 2, 64, 16, seed=23)
    width = 4  # four pages a row: all of sequence 1's, and room for 64
    p.dev_table = p.dev_table[:, :width].contiguous()
    p.batch = F.kv_batch(2, p.T, max(new), p.cu, p.dev_lens, p.dev_table, width)
    q, o, lse = run_attention(F, p, 2)
    p.dev_lens.copy_(torch.tensor([-5, 1000], dtype=torch.int32))
    _, o2, lse2 = run_attention(F, p, 2, q=q)
    assert p.status.item() == F.FL_KV_BAD_PAGE
    assert not o2[:1].any() and bool((lse2[:, :1] == -math.inf).all())
    assert torch.equal(o2[1:], o[1:]) and torch.equal(lse2[:, 1:], lse[:, 1:])


@pytest.mark.parametrize("new,lens,heads,kvh", [([1], [4000], 2, 2), ([2, 200], [1000, 3000], 4, 2)])
def test_attention_large_scores(F, new, lens, heads, kvh):
    """Scores up to hundreds: the running maximum moves, and one key takes almost all."""
    p = Paged(F, new, lens, kvh, 128, 64, seed=7, scale=6.0)
    q = p.randn(p.T, heads, 128, scale=6.0)
    _, o, lse = run_attention(F, p, heads, q=q)
    ro, rl, size = attention64(p, q, heads)
    # scores of up to 36 * 128 / 11.3 * 0.5 are sums of fp32 products: 2^-24 * 128 * 400 of error at most in each
    # exponent, so that much of p |v| too
    e = 2.0 ** -24 * 128 * 400
    assert bool(((lse.double() - rl).abs() <= e).all())
    assert bool(((o.double() - ro).abs() <= (2.02 * UNIT["bf16"] + e) * size).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new,heads,kvh", [([90, 1, 300], 4, 2), ([1, 1, 1], 8, 1), ([2, 40, 3], 12, 1)])
def test_attention_maxima_that_jump(F, new, heads, kvh, hd, dtype):
    """Scores that jump by up to 100 within a block of keys, in its first or its second half, upwards and
    downwards, so that earlier weights vanish; the jumps are exact in every type."""
    p = Paged(F, new, [700, 650, 1500], kvh, hd, 64, dtype=dtype, seed=29)
    sign = torch.where(torch.rand(hd, generator=p.gen, device="cuda") < 0.5, -1.0, 1.0)
    level = torch.zeros(1500, device="cuda")
    for start, x in [(0, -6), (130, -5), (192, 6), (256, 1), (300, 7), (301, 2), (448, 8), (512, 16), (530, 9), (576, 17),
                     (640, 3), (690, 18), (700, 4), (1024, 19), (1087, 30), (1088, 20), (1215, 31), (1344, 25)]:
        level[start:] = x
    for s, L in enumerate(p.lens):
        for i in range(-(-L // p.page)):
            n = min(p.page, L - i * p.page)
            rows = level[i * p.page:i * p.page + n, None, None] * sign
            p.k[int(p.table[s, i]), :n] = rows.to(p.k.dtype).expand(n, kvh, hd)
    q = sign.to(p.k.dtype).expand(p.T, heads, hd).contiguous()
    _, o, lse = run_attention(F, p, heads, q=q, scale=8 / hd)
    check_attention(p, o, lse, attention64(p, q, heads, scale=8 / hd))


def test_attention_repeats_bit_for_bit_and_workspace_is_left_clean(F):
    """Unequal shapes share one workspace; a repeated call gives the same bits whatever ran between."""
    shapes = [([1] * 5, [4097, 1, 999, 2500, 64], 8, 8), ([1], [6000], 8, 2), ([150, 1], [2000, 2000], 8, 4)]
    ps = [Paged(F, n, x, kvh, 128, 64, seed=i) for i, (n, x, h, kvh) in enumerate(shapes)]
    ws = max((p.workspace(8) for p in ps), key=lambda w: w.numel())
    first = [run_attention(F, p, 8, ws=ws) for p in ps]
    for _ in range(3):
        for p, (q, o, lse) in zip(reversed(ps), reversed(first)):
            _, o2, l2 = run_attention(F, p, 8, q=q, ws=ws)
            assert torch.equal(o, o2) and torch.equal(lse, l2)


def test_attention_reads_past_32_bits(F):
    """A cache of more than 2^32 elements and bytes: the last pages' keys and values."""
    kvh, hd, page = 32, 128, 256
    n_pages = 2 ** 32 // (kvh * hd * page) + 8
    k = torch.empty((n_pages, kvh, page, hd), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    gen = torch.Generator(device="cuda").manual_seed(1)
    pages = [n_pages - 1, 3, n_pages - 5]
    for x in (k, v):
        for i in pages:
            x[i] = torch.randn((kvh, page, hd), generator=gen, device="cuda").bfloat16()
    small = Paged(F, [1, 40], [600, 512], kvh, hd, page, seed=2)
    small.k, small.v = k.transpose(1, 2), v.transpose(1, 2)
    small.table = np.array([pages + [-1], [pages[2], pages[0], -1, -1]], np.int32)
    small.dev_table = torch.from_numpy(small.table).cuda()
    small.cache = F.kv_cache(k, v, n_pages, page, kvh, hd)
    small.batch = F.kv_batch(2, 41, 40, small.cu, small.dev_lens, small.dev_table, 4)
    q, o, lse = run_attention(F, small, 32)
    fine = torch.isfinite(small.v[pages]).all()
    assert bool(fine)
    ref = attention64(small, q, 32)
    small.v = small.v[pages]  # check_attention looks at the largest value
    check_attention(small, o, lse, ref)
    x = small.randn(41, kvh, hd)
    F.fl_k_kv_append(small.cache, small.batch, 32, None, x, x, None, None, 0, small.status)
    assert torch.equal(k[pages[2], :, 599 - 512], x[0]) and torch.equal(v[pages[0], :, 255], x[40])
    assert small.status.item() == 0


@pytest.mark.parametrize("token_major", [False, True])
def test_attention_bad_pages_count_as_zeros(F, token_major):
    heads = 2
    for new in ([1, 1], [1, 60]):
        p = Paged(F, new, [100, 200], heads, 64, 32, token_major=token_major, seed=9)
        bad = p.dev_table.clone()
        bad[1, 2], bad[1, 4] = p.n_pages, -3
        good = p.batch
        p.batch = F.kv_batch(2, p.T, max(new), p.cu, p.dev_lens, bad, p.table.shape[1])
        q, o, lse = run_attention(F, p, heads)
        assert p.status.item() == F.FL_KV_BAD_PAGE
        p.status.zero_()
        for i in (2, 4):
            p.k[int(p.table[1, i])] = 0
            p.v[int(p.table[1, i])] = 0
        p.batch = good
        _, o2, lse2 = run_attention(F, p, heads, q=q)
        assert torch.equal(o, o2) and torch.equal(lse, lse2) and p.status.item() == 0


@pytest.mark.parametrize("new,lens", [([1, 1], [70, 33]), ([5, 6], [70, 33]), ([90], [200])])
def test_attention_lowest_and_infinite_scores(F, new, lens):
    """Keys of the type's largest magnitude drive scores to +-huge; a value that is infinite or NaN reaches
    exactly the rows that see its key."""
    heads, hd = 2, 64
    p = Paged(F, new, lens, heads, hd, 16, seed=13)
    s = 0
    last = lens[s] - 1                                    # the newest token: only the last row sees it
    page, slot = int(p.table[s, last // 16]), last % 16
    p.v[page, slot, 0, 3] = math.inf
    p.v[page, slot, 1, 5] = math.nan
    q, o, lse = run_attention(F, p, heads)
    ref = attention64(p, q, heads)
    fine = torch.isfinite(ref[0])
    assert torch.equal(torch.isfinite(o), fine)
    assert int((~fine).sum()) == 2
    o2 = torch.where(fine, o, 0)
    check_attention(p, o2, lse, (torch.where(fine, ref[0], 0.0), ref[1], torch.where(fine, ref[2], 0.0)))


def test_attention_on_another_stream(F):
    p = Paged(F, [1, 30], [3000, 400], 4, 128, 64, seed=21)
    q, o, lse = run_attention(F, p, 8)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    ws = p.workspace(8)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        _, o2, l2 = run_attention(F, p, 8, q=q, ws=ws, stream=st)
    st.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, l2)


def test_a_captured_call_follows_the_lengths(F):
    """Lengths and pages are read when the graph runs."""
    heads, hd = 4, 64
    p = Paged(F, [1, 1], [100, 400], heads, hd, 16, seed=31)
    st = torch.cuda.Stream()
    q, k, v = p.randn(2, heads, hd), p.randn(2, heads, hd), p.randn(2, heads, hd)
    tab = rope_of(F, 512, 32)
    q_out, o = torch.empty_like(q), torch.empty_like(q)
    lse, ws = torch.empty((heads, 2), device="cuda"), p.workspace(heads)
    torch.cuda.synchronize()

    def step():
        F.fl_k_kv_append(p.cache, p.batch, heads, q, k, v, q_out, tab, 512, p.status, rotary_dim=32, stream=st)
        F.fl_k_kv_attention(p.cache, p.batch, heads, q_out, o, ws, p.status, lse=lse, stream=st)

    with torch.cuda.stream(st):
        step()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step()
    for lens in ([50, 300], [1, 16]):
        p.lens = lens
        p.dev_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check_attention(p, o, lse, attention64(p, q_out, heads))
    assert p.status.item() == 0
