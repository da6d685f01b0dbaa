"""The hand-offs between the warps of the window backward's dK/dV kernel (csrc/window_bwd.cuh), every order in which they can
happen: the issuing thread, the tensor pipe behind it, the softmax warps, and mbarriers of which a wait tells only the parity of a phase.

No device: the roles' programs are written out here, and the places where the kernel waits for and arrives at P^T's barriers are
read from its source."""
import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_17051_b200", "csrc", "window_bwd.cuh")


def programs(tiles, bufs, slots):
    """(issuer, pipe, softmax warp): lists of steps.  bufs: S^T buffers, slots: barriers of P^T."""
    issuer, pipe, warp = [], [], []

    def issue(*ops):
        pipe.extend(ops)
        issuer.extend(("issue", len(pipe)) for _ in ops[-1:])

    ahead = 0

    def issue_s():
        nonlocal ahead
        if ahead < tiles:
            issue(("S", ahead), ("commit", "s", ahead % bufs))
            ahead += 1

    issue_s()
    issue(("dP", 0), ("commit", "dp", 0))
    if bufs > 1:
        issue_s()
    for i in range(tiles):
        issuer.append(("wait", "p", i % slots, i // slots & 1))
        issue(("dV", i))
        issue_s()
        issuer.append(("wait", "ds", 0, i & 1))
        issue(("dK", i))
        if i + 1 < tiles:
            issue(("dP", i + 1), ("commit", "dp", 0))
        warp += [("wait", "s", i % bufs, i // bufs & 1), ("P", i), ("arrive", "p", i % slots), ("wait", "dp", 0, i & 1), ("dS", i), ("arrive", "ds", 0)]
    return issuer, pipe, warp


def fault(tiles, bufs, slots, warps=2):
    """None when every order of events ends with all roles done and every product made of what it should be made of."""
    issuer, pipe, warp = programs(tiles, bufs, slots)
    # what each prefix of a program has done
    issued = [0]
    for step in issuer:
        issued.append(step[1] if step[0] == "issue" else issued[-1])

    def counts(program, match):
        out = [0]
        for step in program:
            out.append(out[-1] + (match(step)))
        return out

    arrived = {(bar, slot): counts(warp, lambda s: s == ("arrive", bar, slot)) for bar, slot in [("p", x) for x in range(slots)] + [("ds", 0)]}
    committed = {(bar, slot): counts(pipe, lambda s: s == ("commit", bar, slot)) for bar, slot in [("s", x) for x in range(bufs)] + [("dp", 0)]}
    wrote = {what: counts(warp, lambda s: s[0] == what) for what in ("P", "dS")}

    def open_(at, step):
        _, bar, slot, parity = step
        _, done, *them = at
        phases = committed[bar, slot][done] if (bar, slot) in committed else sum(arrived[bar, slot][w] for w in them) // warps
        return phases & 1 != parity

    def bad(at, op):
        them = at[2:]
        if op[0] == "S":         # over P^T of bufs tiles before, which every warp has written and dV has been made of
            return any(wrote["P"][w] < op[1] - bufs + 1 for w in them)
        if op[0] == "dV":
            return any(not op[1] < wrote["P"][w] <= op[1] + bufs for w in them)
        if op[0] == "dP":        # over dS^T of the tile before
            return any(wrote["dS"][w] < op[1] for w in them)
        if op[0] == "dK":
            return any(wrote["dS"][w] != op[1] + 1 for w in them)
        return False

    start = (0, 0) + (0,) * warps
    seen, todo = {start}, [start]
    while todo:
        at = todo.pop()
        nexts = []
        if at[0] < len(issuer) and (issuer[at[0]][0] == "issue" or open_(at, issuer[at[0]])):
            nexts.append((at[0] + 1,) + at[1:])
        if at[1] < issued[at[0]]:
            if bad(at, pipe[at[1]]):
                return "%s of tile %d from what is not there: %s" % (*pipe[at[1]], at)
            nexts.append((at[0], at[1] + 1) + at[2:])
        for w in range(2, 2 + warps):
            if at[w] < len(warp) and (warp[at[w]][0] != "wait" or open_(at, warp[at[w]])):
                nexts.append(at[:w] + (at[w] + 1,) + at[w + 1:])
        if not nexts and at != (len(issuer), len(pipe)) + (len(warp),) * warps:
            return "nobody can go on: %s" % (at,)
        for n in nexts:
            if n not in seen:
                seen.add(n)
                todo.append(n)
    return None


def test_what_the_model_says_of_one_barrier_and_two_buffers():
    """The issuer may be a tile late while the warps go on to the other buffer: one barrier does not tell the tiles apart."""
    assert fault(5, 2, 1) is not None
    assert fault(5, 1, 1) is None


@pytest.mark.parametrize("tiles", [1, 2, 3, 6])
@pytest.mark.parametrize("bufs", [1, 2])
def test_a_barrier_of_p_for_every_buffer_of_s(tiles, bufs):
    assert fault(tiles, bufs, bufs) is None


def test_three_warps():
    assert fault(4, 2, 2, warps=3) is None


def test_the_kernel_has_a_barrier_of_p_for_every_buffer_of_s():
    with open(SOURCE) as f:
        text = f.read()
    body = text[text.index("void win_bwd_dkv("):text.index("win_join_kernel")]
    waits = re.findall(r"mbar_wait\w*\(p_full([^,]*),([^,]*),", body)
    arrivals = re.findall(r"warp_arrive\(p_full([^,]*),", body)
    assert [tuple(x.strip() for x in w) for w in waits] == [("+ i % kSBufs", "(i / kSBufs) & 1")]
    assert [a.strip() for a in arrivals] == ["+ i % kSBufs"]
