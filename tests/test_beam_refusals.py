"""What the beam search's and the shared pages' calls refuse, before any device work (CPU only: addresses are made up)."""
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


A = [0x1000000 * (i + 1) for i in range(32)]
CUDA, ARG, UNSUPPORTED, CAPACITY = -5, -1, -7, -2  # good arguments fail at the first CUDA call


def search(F, **kw):
    x = dict(n_seqs=2, beams=4, vocab=100, max_steps=9, eos=3, early=0, length_penalty=1.0)
    return F.fl_beam_search(**(x | kw))


def state(F, at=0, **kw):
    names = ("scores", "steps", "done", "end_scores", "end_steps", "end_beams")
    return F.fl_beam_state(**(dict(zip(names, A[at:at + 6])) | kw))


SEARCHES = [("n_seqs", -1, ARG), ("n_seqs", 16385, CAPACITY), ("beams", 0, ARG), ("beams", 17, CAPACITY), ("vocab", 0, ARG),
            ("vocab", 2 ** 19 + 1, CAPACITY), ("max_steps", 0, ARG), ("max_steps", 2 ** 24 + 1, CAPACITY), ("eos", -2, ARG),
            ("eos", 100, ARG), ("early", 2, ARG), ("length_penalty", float("nan"), ARG), ("length_penalty", float("inf"), ARG),
            ("length_penalty", -1.1e6, ARG), ("length_penalty", 16.5, ARG)]


def test_step(F):
    L = F.lib()
    #       search     from         to           dtype logits ld  tokens parents tokens parents workspace status stream
    good = [search(F), state(F), state(F, 6), F.FL_DT_F32, A[12], 100, A[13], A[14], A[15], A[16], A[17], A[18], None]
    assert L.fl_k_beam_step(*good) == CUDA
    for i, value, code in [(0, None, ARG), (1, None, ARG), (2, None, ARG), (3, 3, ARG), (3, -1, ARG), (4, None, ARG), (4, A[12] + 8, ARG),
                           (5, 99, UNSUPPORTED), (5, 102, UNSUPPORTED), (5, -104, UNSUPPORTED), (6, None, ARG), (6, A[13] + 2, ARG), (7, None, ARG),
                           (7, A[14] + 1, ARG), (8, None, ARG), (8, A[15] + 2, ARG), (9, None, ARG), (9, A[16] + 2, ARG), (10, None, ARG),
                           (10, A[17] + 8, ARG), (11, None, ARG), (11, A[18] + 2, ARG)]:
        bad = list(good)
        bad[i] = value
        assert L.fl_k_beam_step(*bad) == code, (i, value)
    assert L.fl_k_beam_step(*good[:3], F.FL_DT_BF16, *good[4:]) == UNSUPPORTED  # rows of 100 16-bit numbers
    for name, value, code in SEARCHES:
        assert L.fl_k_beam_step(search(F, **{name: value}), *good[1:]) == code, (name, value)
        assert L.fl_k_beam_workspace(search(F, **{name: value})) == 0
    for name in ("scores", "steps", "done", "end_scores", "end_steps", "end_beams"):
        for at, i in ((0, 1), (6, 2)):
            for value in (None, A[20] + 2, A[at + (name == "scores")]):  # none, unaligned, another one's
                bad = list(good)
                bad[i] = state(F, at, **{name: value})
                assert L.fl_k_beam_step(*bad) == ARG, (name, value)
    assert L.fl_k_beam_step(good[0], state(F), state(F), *good[3:]) == CUDA       # in place
    assert L.fl_k_beam_step(good[0], state(F), state(F, 6, steps=A[1]), *good[3:]) == ARG
    assert L.fl_k_beam_step(good[0], state(F), state(F, 6, steps=A[2]), *good[3:]) == ARG
    assert L.fl_k_beam_step(search(F, max_steps=2 ** 24, length_penalty=-5.0), *good[1:]) == ARG  # 2^120
    assert L.fl_k_beam_step(search(F, max_steps=2 ** 24, length_penalty=-4.8), *good[1:]) == CUDA
    assert L.fl_k_beam_step(search(F, n_seqs=0), *good[1:]) == 0
    assert L.fl_k_beam_workspace(search(F)) > L.fl_k_beam_workspace(search(F, beams=3)) > 0
    with pytest.raises(F.FlError):
        F.fl_k_beam_workspace(search(F, beams=17))


def test_trace(F):
    L = F.lib()
    #       search     state     tokens parents n pad out   lens  scores status stream
    good = [search(F), state(F), A[6], A[7], 4, 0, A[8], A[9], A[10], A[11], None]
    assert L.fl_k_beam_trace(*good) == CUDA
    for i, value, code in [(0, None, ARG), (1, None, ARG), (2, None, ARG), (2, A[6] + 2, ARG), (3, None, ARG), (3, A[7] + 1, ARG), (4, 0, ARG),
                           (4, 5, ARG), (6, None, ARG), (6, A[8] + 2, ARG), (7, None, ARG), (7, A[9] + 2, ARG), (8, None, ARG),
                           (8, A[10] + 2, ARG), (9, None, ARG), (9, A[11] + 2, ARG)]:
        bad = list(good)
        bad[i] = value
        assert L.fl_k_beam_trace(*bad) == code, (i, value)
    for name, value, code in SEARCHES:
        assert L.fl_k_beam_trace(search(F, **{name: value}), *good[1:]) == code, (name, value)
    assert L.fl_k_beam_trace(search(F, n_seqs=0), *good[1:]) == 0


def cache(F, **kw):
    c = dict(dtype=F.FL_DT_BF16, kv_heads=2, head_dim=128, page_size=64, n_pages=8, k=A[0], v=A[1],
             page_stride=2 * 64 * 128, head_stride=64 * 128, token_stride=128)
    return F.fl_kv_cache(**(c | kw))


def pages(F, at=2, **kw):
    p = dict(n_seqs=3, n_pages=8, page_size=64, table_stride=4, lens=A[at], table=A[at + 1], refs=A[at + 2])
    return F.fl_kv_pages(**(p | kw))


PAGES = [("n_seqs", -1, ARG), ("n_seqs", 2 ** 20 + 1, CAPACITY), ("n_pages", 0, ARG), ("page_size", 8, UNSUPPORTED),
         ("page_size", 96, UNSUPPORTED), ("page_size", 512, UNSUPPORTED), ("table_stride", 0, ARG), ("table_stride", 2 ** 26, CAPACITY)]
CACHES = [("dtype", 1, UNSUPPORTED), ("kv_heads", 0, ARG), ("head_dim", 96, UNSUPPORTED), ("n_pages", 7, ARG), ("page_size", 32, ARG),
          ("k", None, ARG), ("v", A[1] + 8, ARG), ("token_stride", 132, UNSUPPORTED), ("head_stride", 64, UNSUPPORTED)]


@pytest.mark.parametrize("which", ["fl_k_kv_fork", "fl_k_kv_compact"])
def test_pages(F, which):
    L = F.lib()
    call = getattr(L, which)
    two = F.kv_caches([cache(F), cache(F, k=A[20], v=A[21])])
    #       caches n from      to           parents / moved, new / used, workspace, status, stream
    good = [two, 2, pages(F), pages(F, 5), A[8], A[9], A[10], A[11], None]
    assert call(*good) == CUDA
    for i, value, code in [(0, None, ARG), (1, 0, ARG), (1, F.FL_KV_MAX_CACHES + 1, ARG), (2, None, ARG), (3, None, ARG), (4, A[8] + 2, ARG),
                           (5, A[9] + 1, ARG), (6, None, ARG), (6, A[10] + 8, ARG), (7, None, ARG), (7, A[11] + 2, ARG)]:
        bad = list(good)
        bad[i] = value
        assert call(*bad) == code, (i, value)
    for i in (4, 5):  # a fork's parents and new tokens may be left out, a compaction's outputs may not
        bad = list(good)
        bad[i] = None
        assert call(*bad) == (CUDA if which == "fl_k_kv_fork" else ARG)
    for name, value, code in PAGES:
        bad = list(good)
        bad[2], bad[3] = pages(F, **{name: value}), pages(F, 5, **{name: value})
        assert call(*bad) == code, (name, value)
        assert L.fl_k_kv_pages_workspace(bad[2]) == 0
        bad[2] = pages(F)
        assert call(*bad) == ARG, (name, value)  # other sizes than `from`
    for name in ("lens", "table", "refs"):
        for value in (None, A[20] + 2, A[2], A[3], A[4]):
            bad = list(good)
            bad[3] = pages(F, 5, **{name: value})
            assert call(*bad) == ARG, (name, value)
        bad[3] = good[3]
        bad[2] = pages(F, **{name: None})
        assert call(*bad) == ARG, name
    for name, value, code in CACHES:
        bad = list(good)
        bad[0] = F.kv_caches([cache(F), cache(F, **{name: value})])
        assert call(*bad) == code, (name, value)
    for name, value in (("dtype", F.FL_DT_F16), ("kv_heads", 1), ("head_dim", 64), ("page_stride", 3 * 64 * 128), ("token_stride", 136)):
        bad = list(good)
        bad[0] = F.kv_caches([cache(F), cache(F, **{name: value})])
        assert call(*bad) == ARG, name
    assert L.fl_k_kv_pages_workspace(pages(F)) > 0
    bare = list(good)
    bare[2], bare[3] = (F.fl_kv_pages(0, 8, 64, 4, None, None, A[i]) for i in (4, 7))
    assert call(*bare) == CUDA  # no sequences: only the holders outside of the table
    with pytest.raises(F.FlError):
        F.fl_k_kv_pages_workspace(pages(F, page_size=5))
