"""The turns that the two streams of the chunk attention take, explored in every order in which their four roles may
run (CPU only).  A wait tells phases apart by parity alone: it is right only while its barrier is in that
phase or just past it.  The waits' conditions and phases are taken from the kernel's source; what else holds the
roles back there (the ring of stages, the two Q tiles) is left out, so that the turns are shown to be sound by
themselves."""
import itertools
import re

import pytest

from tests.test_kv_sync import _code, _products

WAIT = re.compile(r"if \(([^;{}]*?) && !wait\(B_TURN \+ ([^,]*), ([^;]*?)\)\) break;")


def rules():
    """(before the loop, inside it): compiled (condition, barrier, phase) of each wait for a turn."""
    body = _products()
    loop = body.index("for (int t = -la;")
    found = ([], [])
    for m in WAIT.finditer(body):
        cond = m[1].replace("&&", "and").replace("||", "or")
        found[m.start() > loop].append(tuple(compile(x, "kernel", "eval") for x in (cond, m[2], m[3])))
    assert sum(map(len, found)) == body.count("wait(B_TURN")
    return found


def programs(pieces, before, inside):
    """What each role does: ('S' or 'P', stream, number) is done by one and needed by another, ('turn', b) tells one, ('wait',
    b, n) waits for one."""
    mma, soft = ([], []), ([], [])
    for s in (0, 1):
        turn = at = 0
        for turns, extra in pieces:  # blocks of stream 0, how many more stream 1 has
            n = turns + (extra if s else 0)

            def waits(rules_, **env):
                for cond, which, phase in rules_:
                    if eval(cond, {}, env):
                        mma[s].append(("wait", eval(which, {}, env), eval(phase, {}, env)))

            waits(before, s=s, turn=turn, turns=turns)
            for j in range(-1, n):
                if j >= 0:
                    mma[s].append(("need", "P", s, at + j))
                if j + 1 < n:
                    waits(inside, s=s, j=j, turn=turn, turns=turns)
                    mma[s].append(("do", "S", s, at + j + 1))
            for j in range(n):
                soft[s].append(("need", "S", s, at + j))
                if j < turns:
                    soft[s].append(("turn", s))
                soft[s].append(("do", "P", s, at + j))
            turn, at = turn + turns, at + n
    return mma + soft


def explore(pieces, before, inside):
    """None, or what goes wrong in some order."""
    progs = programs(pieces, before, inside)
    done = [{x: i for i, x in enumerate(p) if x[0] == "do"} for p in progs]
    maker = {("S", 0): 0, ("S", 1): 1, ("P", 0): 2, ("P", 1): 3}
    told = [list(itertools.accumulate((x[0] == "turn" for x in p), initial=0)) for p in progs[2:]]
    seen, todo = {(0, 0, 0, 0)}, [(0, 0, 0, 0)]
    while todo:
        pcs = todo.pop()
        moved = False
        for a, p in enumerate(progs):
            if pcs[a] == len(p):
                continue
            x = p[pcs[a]]
            if x[0] == "need":
                by = maker[x[1], x[2]]
                if done[by]["do", x[1], x[2], x[3]] >= pcs[by]:
                    continue
            if x[0] == "wait":
                phases = told[x[1]][pcs[2 + x[1]]]
                if phases not in (x[2], x[2] + 1):
                    return f"wait for turn {x[2]} of stream {x[1]} with {phases} told"
                if phases == x[2]:
                    continue
            moved = True
            nxt = pcs[:a] + (pcs[a] + 1,) + pcs[a + 1:]
            if nxt not in seen:
                seen.add(nxt)
                todo.append(nxt)
        if not moved and any(pc < len(p) for pc, p in zip(pcs, progs)):
            return "all roles wait"
    return None


def test_the_kernel_tells_a_turn_for_every_block_of_both_streams():
    src = _code("kv_attention_tc.cu")
    assert src.count("arrive(B_TURN + s)") == src.count("if (j < turns) arrive(B_TURN + s);") == 2
    assert "turn += turns;" in _products()


PIECES = [[(1, 0), (1, 0)], [(1, 0), (2, 0)], [(2, 0), (1, 0), (1, 0)], [(2, 1), (2, 0)], [(3, 2), (0, 2), (3, 0)],
          [(1, 3), (0, 1), (1, 0), (2, 1)], [(4, 0), (3, 1), (2, 0)]]


@pytest.mark.parametrize("pieces", PIECES, ids=str)
def test_no_wait_takes_one_turn_for_another(pieces):
    assert explore(pieces, *rules()) is None


def test_the_exploration_sees_a_turn_that_nobody_waits_for_and_a_circle():
    """Without the wait between pieces a phase is taken for another; with stream 0 waiting as stream 1 does, both wait."""
    before, inside = rules()
    assert "told" in explore([(1, 0), (2, 0)], [], inside)
    both = [tuple(compile(x, "planted", "eval") for x in ("j + 1 < turns", "1 - s", "turn + j + 1"))]
    assert explore([(2, 0)], before, both) == "all roles wait"
