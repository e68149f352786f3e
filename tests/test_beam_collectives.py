"""Under which conditions the beam search's and the shared pages' kernels vote, shuffle and meet, from their sources (CPU only).

A collective waits for all lanes (a barrier for all threads) that its mask or block names, so every condition around one, and every
early return before one, has to have the same answer in a whole warp (block).  What has been found to be so by reading is listed
here; a condition that is not listed fails."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2406_14898_gb300", "csrc")
WARP = r"__(?:shfl|reduce|ballot|any|all)\w*_sync\s*\(|__syncwarp\s*\(|\bshfl64\s*\(|\bshfl_int4\s*\(|\bof_warp\s*\(|\bbusy\s*\("
BLOCK = r"__syncthreads\w*\s*\(|\bcluster_sync\s*\(|\bblock_scan\s*\(|\braise\s*\(\s*\)|\bbits\s*\(base\)|\bcount\s*\(base\)"

# The same in a whole block: of the call's sizes, the CTA's place, or of what all threads have read behind a barrier.
BLOCK_WIDE = {
    "beam.cu": {
        "int base = 0; base < rows; base += 32 * THREADS", "base", "again", "int c = c0; c < c1;",
        "int begin = part_begin; begin < part_end; begin += 32 * CHUNK_PIECES",
        "int first = begin, chunk = 0; first < end; first += CHUNK_PIECES, ++chunk", "(seen & chunk) == 0", "early", "else early",
        "end == part_end", "n > MAX_HITS", "else n > MAX_HITS", "early && n > 32", "else n <= MAX_HITS", "int r = 0; r < B; ++r",
        "c0 >= c1", "!active", "int base = (T - 1) / row * row; base >= 0; base -= row", "ctas > 1", "else ctas > 1",
    },
    "kv_pages.cu": {
        "ONE", "else ONE", "!ONE", "int tile = share ? 0 : rank; tile < tiles; tile += share ? 1 : ctas", "share", "tiles > 1",
        "int base = s0; base < s1; base += PLAN_THREADS", "s1 - s0 > PLAN_THREADS",
    },
}
# The same in a whole warp: of the warp's number, its part of the pages, or of a vote.
WARP_WIDE = {
    "beam.cu": {
        "warp < B", "warp != 0", "tid < 32", "__any_sync(0xffffffffu, end_rank >= 0)", "who & (who - 1)", "end != 0",
        "; k < B; ++k", "int d = 16; d; d >>= 1", "int d = 1; d < FL_BEAM_MAX; d <<= 1", "int o = 0; o < 32; ++o",
        "int d = 1; d < THREADS / GROUPS; d <<= 1", "unsigned who = __ballot_sync(0xffffffffu, look)", "int d = 1; d < 32; d <<= 1",
    },
    "kv_pages.cu": {
        "int d = 1; d < 32; d <<= 1", "int q = q0; q < q1; q += 32", "int q = q0; q < min(q1, all); q += 32", "int c = 0; c < ctas; ++c",
        "int64_t u0 = (int64_t)threadIdx.x / 32 * gridDim.x + blockIdx.x; u0 < all; u0 += 32ll * warps",
        "int l = 0; l < 32 && u0 + (int64_t)l * warps < all; ++l",
    },
}


def code(name):
    with open(os.path.join(CSRC, name)) as fh:
        text = "\n".join(line.split("//", 1)[0] for line in fh if not line.lstrip().startswith("#"))
    return re.sub(r'"(?:[^"\\]|\\.)*"', '""', text)


def closing(text, at):
    """The place of the bracket that closes the one at `at`."""
    depth, pair = 0, {"(": ")", "{": "}"}[text[at]]
    for i in range(at, len(text)):
        depth += (text[i] == text[at]) - (text[i] == pair)
        if depth == 0:
            return i
    raise ValueError(text[at:at + 80])


def statements(text, around=()):
    """Pieces of code without their blocks, each with the conditions around it; a lambda's body has those of its place, and its name
    as one that begins with `[`."""
    at = 0
    while at < len(text):
        m = re.compile(r"\s*(else\b\s*)?(?:(if|for|while)\b\s*(?:constexpr\s*)?\()?").match(text, at)
        before = statements.last if m[1] else None
        if m[2] or m[1]:
            if m[2]:
                end = closing(text, m.end() - 1)
                head = " ".join(text[m.end():end].split())
                yield head, around + ((f"else {before}",) if m[1] else ())
                inner, body = around + ((f"else {before}",) if m[1] else ()) + (head,), end + 1
            else:
                head, inner, body = before, around + (f"else {before}",), m.end()
            while text[body].isspace():
                body += 1
            stop = closing(text, body) + 1 if text[body] == "{" else one(text, body)
            yield from statements(text[body + 1:stop - 1] if text[body] == "{" else text[body:stop], inner)
            statements.last, at = head, stop
            continue
        at = m.end()
        if at < len(text) and text[at] == "{":
            end = closing(text, at)
            yield from statements(text[at + 1:end], around)
            at = end + 1
            continue
        stop = one(text, at)
        piece = text[at:stop]
        brace = piece.find("{")
        if brace >= 0 and re.search(r"\]\s*(\([^{]*\)\s*)?$", piece[:brace]):  # a lambda
            end = closing(piece, brace)
            yield from statements(piece[brace + 1:end], around + ("[" + piece[:brace],))
            piece = piece[:brace] + piece[end + 1:]
        yield piece, around
        at = max(stop, at + 1)


def one(text, at):
    """The end of the statement that begins at `at`."""
    m = re.compile(r"\s*(?:if|for|while)\b\s*(?:constexpr\s*)?\(").match(text, at)
    if m:
        at = closing(text, m.end() - 1) + 1
        while text[at].isspace():
            at += 1
        stop = closing(text, at) + 1 if text[at] == "{" else one(text, at)
        m = re.compile(r"\s*else\b").match(text, stop)
        if m:
            stop = m.end()
            while text[stop].isspace():
                stop += 1
            stop = closing(text, stop) + 1 if text[stop] == "{" else one(text, stop)
        return stop
    while at < len(text):
        if text[at] in "({":
            at = closing(text, at)
        elif text[at] == ";":
            return at + 1
        at += 1
    return at


def bodies(text):
    """Device functions and kernels: (name, body)."""
    for m in re.finditer(r"(?:__global__|FL_DEV)\b[^;{]*?(\w+)\s*\(", text):
        end = closing(text, m.end() - 1)
        brace = re.compile(r"\s*(?:const\s*)?(?::[^{;]*)?\{").match(text, end + 1)
        if brace and m[1] != "__launch_bounds__":
            at = brace.end() - 1
            yield m[1], text[at + 1:closing(text, at)]
        elif m[1] == "__launch_bounds__":
            m2 = re.compile(r"\s*(\w+)\s*\(").match(text, end + 1)
            at = text.index("{", closing(text, m2.end() - 1))
            yield m2[1], text[at + 1:closing(text, at)]


def faults(text, block_wide, warp_wide):
    found = []
    for name, body in bodies(text):
        statements.last = None
        pieces = list(statements(body))
        for i, (piece, around) in enumerate(pieces):
            behind = ""  # what a return here skips: the rest of its lambda, or of the function
            if re.search(r"\breturn\s*;", piece):
                place = [c for c in around if c[0] == "["]
                behind = " ".join(p for p, a in pieces[i:] if [c for c in a if c[0] == "["][:len(place)] == place)
            around = [c for c in around if c[0] != "["]
            if re.search(BLOCK, piece + behind):
                bad = [c for c in around if c not in block_wide]
            elif re.search(WARP, piece + behind):
                bad = [c for c in around if c not in block_wide and c not in warp_wide]
            else:
                continue
            found += [(name, " ".join(piece.split())[:80], c) for c in bad]
    return found


@pytest.mark.parametrize("name", ["beam.cu", "kv_pages.cu"])
def test_conditions_around_collectives_are_known(name):
    text = code(name)
    assert len(list(bodies(text))) > 10
    assert faults(text, BLOCK_WIDE[name], WARP_WIDE[name]) == []


@pytest.mark.parametrize("planted", ["if (won) head.v = __reduce_min_sync(0xffffffffu, head.v);",
                                     "if (lane < k) { at += 1; __syncwarp(); }",
                                     "for (int i = lane; i < k; i += 32) at += __shfl_sync(0xffffffffu, at, i);",
                                     "if (lane > 3) return;", "if (warp < B) __syncthreads();", "if (k > B) { } else __syncthreads();"])
def test_a_planted_one_is_found(planted):
    text = code("beam.cu")
    at = text.index("    const Cand one = lane < k ?")
    assert faults(text[:at] + planted + text[at:], BLOCK_WIDE["beam.cu"], WARP_WIDE["beam.cu"])
