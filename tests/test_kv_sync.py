"""Ordering that the paged attention's shared memory, TMEM and workspace depend on, read from its sources
(CPU only): a missing wait of this kind shows on a GPU only when the timing is unlucky."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_14898_gb300", "csrc")


def _code(name):
    with open(os.path.join(CSRC, name)) as fh:
        return "\n".join(line.split("//", 1)[0] for line in fh)


def _in_order(text, *parts):
    at = 0
    for p in parts:
        assert p in text[at:], p
        at = text.index(p, at) + len(p)


def _products():
    src = _code("kv_attention_tc.cu")
    return src[src.index("const int s = (int)uniform(warp - W_MMA)"):src.index("tmem_dealloc")]


def test_products_wait_for_their_operands():
    """P V of a block behind its values' stage, the room in O and each half of the weights; the next scores,
    which lie over the P that P V reads, behind that P V."""
    body = _products()
    _in_order(body, "wait(B_READY + st, ph)", "wait(B_FREE + s, uses - 1)", "wait(B_PH + s, done)", "umma_bf16_ts(",
              "wait(B_P + s, done)", "umma_bf16_ts(", "umma_commit(bars + B_O + s)", "umma_commit(bars + B_EMPTY + vs)",
              "!C::OWN_P && done > 0 && !wait(B_O + s, done - 1)", "umma_bf16(t_s", "umma_commit(bars + B_S + s)",
              "umma_commit(bars + B_EMPTY + ks)")
    assert body.count("umma_bf16_ts(") == 2 and body.count("umma_bf16(") == 1


def test_streams_take_turns_without_waiting_in_a_circle():
    """Stream 1's scores of block j wait for stream 0's turn j, stream 0's of block j + 1 for stream 1's turn j:
    each told once a block by the softmax, behind that block's scores and before its weights, in the blocks that both
    streams take part in."""
    src, body = _code("kv_attention_tc.cu"), _products()
    assert "if (j + 1 < turns && j + s >= 0 && !wait(B_TURN + 1 - s, turn + j + s)) break;" in body
    assert "turn += turns;" in body and "return two ? na[0] : 0;" in src
    soft = src[src.index("float m = -INFINITY, l = 0.f;"):src.index("if (warp == W_TMA)")]
    _in_order(soft, "wait(B_S + s, ss++)", "if (j < turns) arrive(B_TURN + s);", "tmem_st32(t_p", "arrive(B_PH + s)")
    assert soft.count("if (j < turns) arrive(B_TURN + s);") == 2  # warps with rows, warps without
    # stream 0 never has more blocks than stream 1, which therefore tells all the turns that stream 0 waits for
    assert "p.na[0] = p.two ? min(p.n, max(0, p.nb[0] - p.kb0))" in src and "p.na[1] = p.two ? p.n" in src


def test_both_streams_free_every_stage_and_query_tile():
    """A stage or a Q tile that a stream does not read is freed by an arrival, one that it reads by the
    product's commit: one of the two on every path, so that the barrier's count of two is met each phase."""
    src, body = _code("kv_attention_tc.cu"), _products()
    assert "both ? 2" in src and "both = (i >= B_EMPTY && i < B_QF) || (i >= B_QE && i < B_S)" in src
    assert "if (!pv && lane == 0) mbar_arrive(bars + B_EMPTY + st);" in body
    assert "if (!qk && lane == 0) mbar_arrive(bars + B_EMPTY + st);" in body
    assert "(qn != q || mine == 0) && lane == 0) mbar_arrive(bars + B_QE + (qn & 1))" in body
    assert "if (j + 2 == mine) umma_commit(bars + B_QE + (q & 1));" in body


def test_softmax_reads_behind_products_and_hands_over_behind_stores():
    src = _code("kv_attention_tc.cu")
    soft = src[src.index("float m = -INFINITY, l = 0.f;"):src.index("if (warp == W_TMA)")]
    _in_order(soft, "wait(B_S + s, ss++)", "tc_fence_after()", "tmem_ld32(t_s", "wait(B_O + s, pv + j - 1)",
              "tmem_ld32(t_o", "tmem_st32(t_p", "tmem_st_wait()", "arrive(B_PH + s)", "arrive(B_P + s)",
              "wait(B_O + s, pv - 1)", "tmem_ld32(t_o + c, o)", "arrive(B_FREE + s)")
    arrive = src[src.index("auto arrive = "):]
    _in_order(arrive, "tc_fence_before()", "__syncwarp()", "mbar_arrive(bars + i)")


def test_nothing_is_in_flight_when_a_cta_leaves():
    src = _code("kv_attention_tc.cu")
    end = src[src.rindex("umma_commit(bars + B_END"):src.index("int launch_tc(")]
    _in_order(end, "mbar_wait_warp(bars + B_END", "sh_flag[4] != 0", "mbar_wait_warp(bars + B_FULL", "mbar_wait_warp(bars + B_QF",
              "__syncthreads()", "tmem_dealloc(tmem, 512)")
    # every wait in the kernel is a bounded one
    kernel = src[src.index("kv_attn_tc_kernel"):src.index("int launch_tc(")]
    assert not re.search(r"\bmbar_wait\(|while \(true\) \{\s*\}", kernel)


def test_parts_are_visible_before_they_are_counted():
    """A part's stores, a barrier of the threads that made them, the count (which releases and acquires), a
    barrier, the loads of whoever joins.  Parts are written and read past L1."""
    shared = _code("kv_attention.cuh")
    assert "atom.acq_rel.gpu.global.inc.u32" in shared and "ld.acquire.gpu.global.u32" in shared
    for name, barrier in (("kv_attention.cu", "__syncthreads()"), ("kv_attention_tc.cu", "bar_sync(1 + s, 128)")):
        src = _code(name)
        at = src.index("kv_part_done(")
        before, after = src[:at], src[at:]
        assert before.rindex("__stcg(") < before.rindex(barrier)
        _in_order(after, barrier, "__ldcg(")
    src = _code("kv_attention_tc.cu")  # the look before: its barrier lies before the loads too
    _in_order(src, "kv_part_is_last(count, parts)", "bar_sync(1 + s, 128)", "__stcg(", "kv_part_done(")


def test_kernels_wait_for_the_one_before_them():
    """Every kernel waits for the one before it on its stream before it reads what that may have written."""
    for name in ("kv_cache.cu", "kv_attention.cu", "kv_attention_tc.cu"):
        for body in re.split(r"__global__", _code(name))[1:]:
            body = body[body.index("{"):body.index("\n}")]
            assert "pdl_wait();" in body
            first = min([body.index(x) for x in ("kv_plan(", ".load(", "tab[x]", "b.status") if x in body])
            assert body.index("pdl_wait();") < first
