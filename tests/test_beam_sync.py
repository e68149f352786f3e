"""What the beam search's and the shared pages' kernels depend on, read from their sources (CPU only)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_14898_gb300", "csrc")


def _code(name):
    with open(os.path.join(CSRC, name)) as fh:
        return "\n".join(line.split("//", 1)[0] for line in fh)


def _in_order(text, *parts):
    at = 0
    for p in parts:
        assert p in text[at:], p
        at = text.index(p, at) + len(p)


@pytest.mark.parametrize("name", ["beam.cu", "kv_pages.cu"])
def test_no_collective_behind_a_condition_of_its_own_expression(name):
    """A warp's shuffles, votes and reductions wait for all of its lanes: none may stand where a lane's &&, || or ?: skips it."""
    for statement in re.split(r"[;{}]", _code(name)):
        for part in re.split(r",(?![^()]*\))", statement):
            found = re.search(r"(&&|\|\||\?)(?P<rest>.*?)(__\w*_sync|__syncthreads\w*)\s*\(", part, re.S)
            assert not found, part.strip()


@pytest.mark.parametrize("name", ["beam.cu", "kv_pages.cu"])
def test_kernels_wait_for_the_one_before_them(name):
    for body in re.split(r"__global__", _code(name))[1:]:
        body = body[body.index("{"):body.index("\n}")]
        assert body[1:].lstrip().startswith("pdl_wait();") and "pdl_trigger();" in body


def test_a_units_places_are_not_written_before_they_were_read():
    """The hits of a unit lie behind a barrier when they are ranked, and a barrier divides that from the next unit's."""
    src = _code("beam.cu")
    kernel = src[src.index("beam_step_kernel(StepArgs a)"):src.index("int64_t part_bytes(")]
    _in_order(kernel, "if (tid == 0) sh_count = sh_few = 0;", "const auto raise =", "__syncthreads()", "equals = raise()", "atomicAdd(&sh_count, 1)",
              "sh_sum[warp] = sum", "if (early) raise();", "__syncthreads()", "int n = sh_count", "a.sums[", "__syncthreads()")


def test_a_place_is_read_before_it_is_asked_for_again():
    """A chunk's group has arrived before its places are read; the next request goes to another stage."""
    src = _code("beam.cu")
    loop = src[src.index("for (int first = begin, chunk = 0;"):src.index("float ref = z.ref;")]
    _in_order(loop, "cp_async_wait<STAGES - 1>()", "places = sh_ring + stage * CHUNK_PIECES + tid", "cur[i] = places", "__ballot_sync(0xffffffffu, look)",
              "__syncwarp()", "Io::word(", "__syncwarp()", "ask_more()")
    assert "static_assert(STAGES == 2 &&" in src
    first = src[src.index("const auto ask_first_ones"):src.index("cut(rows);")]
    assert first.count("ask_more();") == 2  # a group for each stage before the loop
    _in_order(src, "if (!guessed) {", "cp_async_wait<0>()", "ask_first_ones()")


def test_joined_rows_are_placed_behind_a_barrier():
    src = _code("beam.cu")
    join = src[src.index("beam_join_kernel(StepArgs a)"):src.index("beam_step_kernel(StepArgs a)")]
    _in_order(join, "j.next[b] = j.end_rank[b] = -1", "__syncthreads()", "if (!active)", "ahead_in(q, mine)", "j.next[place] =",
              "j.end_rank[b] = n", "__syncthreads()", "if (warp != 0) return;", "j.next[lane]")
    assert join.count("__syncthreads()") == 2 and join.count("return;") == 2


def test_plan_phases_are_divided_by_the_clusters_barrier():
    src = _code("kv_pages.cu")
    fork = src[src.index("fork_plan_kernel("):src.index("compact_plan_kernel(")]
    _in_order(fork, "atomicMax(of.lowest", "cluster_sync()", "of.first_writer(r.last)", "sh_totals = make_int4", "cluster_sync()",
              "ld_cluster_int4(&sh_totals", "cluster_sync()", "of.clear(q)")
    compact = src[src.index("compact_plan_kernel("):src.index("struct Caches")]
    _in_order(compact, "sh_all = make_int4", "cluster_sync()", "ld_cluster_int4(&sh_all", "sh_stay = make_int4", "cluster_sync()",
              "ld_cluster_int4(&sh_stay", "__stcg(w.list", "cluster_sync()", "__ldcg(w.list + i)")
