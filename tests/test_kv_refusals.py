"""What the rotary and paged-cache calls refuse, before any device work (CPU only: addresses are made up)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def F():
    from paper_2406_14898_gb300 import build, flglm
    build.build()
    import torch
    if torch.cuda.is_available():
        pytest.skip("made-up device addresses: CPU-only check")
    flglm.lib()
    return flglm


A = [0x100000 * (i + 1) for i in range(16)]
CUDA, ARG, UNSUPPORTED, CAPACITY = -5, -1, -7, -2  # good arguments fail at the first CUDA call


def variants(call, good, cases):
    assert call(*good) == CUDA
    for i, value, code in cases:
        bad = list(good)
        bad[i] = value
        assert call(*bad) == code, (i, value)


def test_rotary_table_refusals(F):
    L = F.lib()
    variants(L.fl_k_rotary_table, [128, 64, 1e4, 0, 1.0, 0, A[0], None],
             [(0, 0, ARG), (1, 63, ARG), (1, 0, ARG), (2, 1.0, ARG), (2, float("inf"), ARG), (2, float("nan"), ARG),
              (3, 4, ARG), (3, -1, ARG), (6, None, ARG), (6, A[0] + 8, ARG)])
    assert L.fl_k_rotary_table(128, 64, 1e4, F.FL_ROPE_SCALE_LINEAR, 0.5, 0, A[0], None) == ARG
    assert L.fl_k_rotary_table(128, 2, 1e4, F.FL_ROPE_SCALE_NTK, 2.0, 0, A[0], None) == ARG
    assert L.fl_k_rotary_table(128, 64, 1e4, F.FL_ROPE_SCALE_BY_PARTS, 2.0, 0, A[0], None) == ARG
    assert L.fl_k_rotary_table(128, 64, 1e4, F.FL_ROPE_SCALE_BY_PARTS, float("nan"), 9, A[0], None) == ARG
    assert L.fl_k_rotary_table(2 ** 31 - 1, 2 ** 14, 1e4, 0, 1.0, 0, A[0], None) == CAPACITY


def test_rotary_refusals(F):
    L = F.lib()
    #       T  nh hd   rd  lay bwd dt  x     ldx  hs   y     ldy  hs   pos   pos2  tab   max status
    good = [4, 2, 128, 64, 0, 0, 0, A[0], 256, 128, A[1], 256, 128, A[2], A[3], A[4], 16, A[5], None]
    variants(L.fl_k_rotary, good,
             [(0, -1, ARG), (1, 0, ARG), (2, 120, UNSUPPORTED), (2, 272, UNSUPPORTED), (3, 0, UNSUPPORTED),
              (3, 24, UNSUPPORTED), (3, 128, UNSUPPORTED), (4, 2, ARG), (5, 2, ARG), (6, 3, ARG), (7, None, ARG),
              (7, A[0] + 8, ARG), (8, 260, UNSUPPORTED), (8, -256, UNSUPPORTED), (9, 4, UNSUPPORTED), (12, -128, UNSUPPORTED), (10, A[1] + 2, ARG), (10, None, ARG),
              (11, 1, UNSUPPORTED), (12, 1, UNSUPPORTED), (13, None, ARG), (13, A[2] + 2, ARG), (14, A[3] + 1, ARG),
              (15, None, ARG), (15, A[4] + 8, ARG), (16, 0, ARG), (17, None, ARG), (17, A[5] + 2, ARG)])
    good[0] = 0
    assert L.fl_k_rotary(*good) == 0
    good[0], good[14], good[3] = 4, None, 128
    assert L.fl_k_rotary(*good) == CUDA  # one stream over the whole head


def parts(F, **kw):
    c = dict(dtype=F.FL_DT_BF16, kv_heads=2, head_dim=128, page_size=64, n_pages=8, k=A[0], v=A[1],
             page_stride=2 * 64 * 128, head_stride=64 * 128, token_stride=128)
    b = dict(n_seqs=2, n_tokens=5, max_new=4, table_stride=3, cu_new=A[2], lens=A[3], page_table=A[4])
    for k, v in kw.items():
        (c if k in c else b)[k] = v
    return F.fl_kv_cache(**c), F.fl_kv_batch(**b)


SHARED = [("dtype", 1, UNSUPPORTED), ("kv_heads", 0, ARG), ("kv_heads", 3, ARG), ("head_dim", 96, UNSUPPORTED),
          ("page_size", 8, UNSUPPORTED), ("page_size", 48, UNSUPPORTED), ("page_size", 512, UNSUPPORTED),
          ("n_pages", 0, ARG), ("k", None, ARG), ("v", None, ARG), ("k", A[0] + 8, ARG), ("v", A[1] + 4, ARG),
          ("page_stride", 64 * 128 + 8, UNSUPPORTED), ("head_stride", 64, UNSUPPORTED), ("token_stride", 132, UNSUPPORTED),
          ("token_stride", 64, UNSUPPORTED), ("n_seqs", -1, ARG), ("n_seqs", 0, ARG), ("n_tokens", -1, ARG),
          ("max_new", -1, ARG), ("max_new", 0, ARG), ("table_stride", 0, ARG), ("table_stride", 2 ** 30, CAPACITY), ("cu_new", None, ARG),
          ("lens", None, ARG), ("page_table", None, ARG), ("cu_new", A[2] + 2, ARG), ("lens", A[3] + 1, ARG),
          ("page_table", A[4] + 2, ARG)]


def test_append_refusals(F):
    L = F.lib()
    c, b = parts(F)
    #       cache batch nh q  ldq  k     ldk  v     ldv  q_out ldqo rd lay pos   pos2  tab   max status
    good = [c, b, 4, A[5], 512, A[6], 256, A[7], 256, A[8], 512, 64, 0, A[9], None, A[10], 99, A[11], None]
    variants(L.fl_k_kv_append, good,
             [(0, None, ARG), (1, None, ARG), (2, 3, ARG), (2, 0, ARG), (3, A[5] + 8, ARG), (4, 4, UNSUPPORTED), (4, -512, UNSUPPORTED),
              (5, None, ARG), (5, A[6] + 2, ARG), (6, 4, UNSUPPORTED), (6, -256, UNSUPPORTED), (7, None, ARG), (7, A[7] + 2, ARG),
              (8, 4, UNSUPPORTED), (8, -256, UNSUPPORTED), (9, None, ARG), (9, A[8] + 2, ARG), (10, 4, UNSUPPORTED),
              (10, -512, UNSUPPORTED), (11, 24, UNSUPPORTED),
              (11, -16, UNSUPPORTED), (11, 144, UNSUPPORTED), (12, 2, ARG), (13, A[9] + 1, ARG), (15, None, ARG),
              (15, A[10] + 8, ARG), (16, 0, ARG), (17, None, ARG), (17, A[11] + 2, ARG)])
    for name, value, code in SHARED:
        c, b = parts(F, **{name: value})
        assert L.fl_k_kv_append(c, b, *good[2:]) == code, (name, value)
    bad = list(good)
    bad[11], bad[14] = 80, A[12]  # two streams of 80 in 128 dims
    assert L.fl_k_kv_append(*bad) == UNSUPPORTED
    bad[11] = 0                   # a second stream without a first
    assert L.fl_k_kv_append(*bad) == UNSUPPORTED
    c, b = parts(F, n_tokens=0)
    assert L.fl_k_kv_append(c, b, *good[2:]) == 0
    bare = list(good)             # neither queries nor a rotation: their arguments are not needed
    bare[3] = bare[9] = bare[15] = None
    bare[11] = bare[16] = 0
    assert L.fl_k_kv_append(*bare) == CUDA


def test_attention_refusals(F):
    L = F.lib()
    c, b = parts(F)
    #       cache batch nh q  ldq  scale ctx  o     ldo  lse   ws     status
    good = [c, b, 4, A[5], 512, 0.0, A[6], A[7], 512, A[8], A[9], A[10], None]
    variants(L.fl_k_kv_attention, good,
             [(0, None, ARG), (1, None, ARG), (2, 5, ARG), (2, 2 * 129, UNSUPPORTED), (3, None, ARG),
              (3, A[5] + 8, ARG), (4, 516, UNSUPPORTED), (4, -512, UNSUPPORTED), (5, float("nan"), ARG), (5, float("inf"), ARG),
              (6, A[6] + 2, ARG), (7, None, ARG), (7, A[7] + 4, ARG), (8, 4, UNSUPPORTED), (8, -512, UNSUPPORTED),
              (9, A[8] + 2, ARG), (10, None, ARG), (10, A[9] + 8, ARG), (11, None, ARG), (11, A[10] + 1, ARG)])
    for name, value, code in SHARED:
        c, b = parts(F, **{name: value})
        assert L.fl_k_kv_attention(c, b, *good[2:]) == code, (name, value)
        assert L.fl_k_kv_attention_workspace(4, c, b) == 0
    c, b = parts(F, n_tokens=0)
    assert L.fl_k_kv_attention(c, b, *good[2:]) == 0
    with pytest.raises(F.FlError):
        F.fl_k_kv_attention_workspace(5, *parts(F))
