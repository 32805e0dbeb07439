"""The order in which the prompt kernel of the cache's attention writes and reads its two LDS buffers, taken from its source and followed
step by step on the CPU: a buffer is written only behind a barrier that follows its last read, and read only behind one that follows the write
of what is wanted.  (On the GPU such a mistake mostly shows nothing: four wavefronts rarely drift a step apart.)"""
import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2111_09562_amd", "csrc", "k_attend_tile.hip")
EVENT = re.compile(r"\b(operands|stage)\((?:&?\w+), ([01]), ([^()]*)\)|(__syncthreads\(\))|\b(next)\(\)")


def block_end(text, at):
    """Behind the statement or the braces that begin at `at`."""
    while text[at].isspace():
        at += 1
    if text[at] != "{":
        return text.index(";", at) + 1
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return i + 1
    raise AssertionError("braces")


def for_tiles(text, rt):
    """The text with `if constexpr (RT == n) .. else ..` resolved."""
    while True:
        m = re.search(r"if constexpr \(RT == (\d)\)", text)
        if not m:
            return text
        end = block_end(text, m.end())
        yes, no, rest = text[m.end():end], "", end
        other = re.match(r"\s*else\b", text[end:])
        if other:
            rest = block_end(text, end + other.end())
            no = text[end + other.end():rest]
        text = text[:m.start()] + (yes if int(m.group(1)) == rt else no) + text[rest:]


def events(text, nested=()):
    got = []
    for m in EVENT.finditer(text):
        if m.group(4):
            got.append(("barrier",))
        elif m.group(5):
            got += nested
        else:
            got.append((m.group(1), int(m.group(2)), re.sub(r"(\d)u\b", r"\1", m.group(3))))
    return got


def schedule(rt):
    text = re.sub(r"//.*", "", open(SOURCE).read())
    text = text[text.index("while (j < end) {"):]
    text = for_tiles(text[:block_end(text, text.index("{"))], rt)
    fast_at, slow_at = text.index("if (n_fast) {"), text.index("for (; i < count; ++i)")
    fast = text[fast_at:block_end(text, text.index("{", fast_at))]
    loop_at = fast.index("for (; i < n_fast; ++i)")
    loop = fast[loop_at:]
    loop = loop[loop.index("{"):block_end(loop, loop.index("{"))]
    lam = loop[loop.index("const auto next = [&] {"):]
    lam = lam[:block_end(lam, lam.index("{"))]
    slow = text[slow_at:]
    return events(text[:fast_at]), events(fast[:loop_at]), events(loop.replace(lam, ""), events(lam)), events(slow)


@pytest.mark.parametrize("rt", [1, 2])
def test_buffers(rt):
    begin, front, step, slow = schedule(rt)
    assert len(begin) == 5 and ("operands", 0, "0") in front and sum(e[0] == "stage" for e in step) == sum(e[0] == "stage" for e in slow) == 2
    assert {e[0] for e in step} == {e[0] for e in slow} == {"operands", "stage", "barrier"}
    for n_fast in range(8):
        phase, holds, read = 0, {}, {}                # per (keys or values, buffer): (block, phase of its write); phase of the last read
        for batch in range(2):
            at = {0: 0, 1: 0}                         # block that the next write of keys, of values brings

            def run(which_events, i):
                nonlocal phase
                for e in which_events:
                    if e[0] == "barrier":
                        phase += 1
                        continue
                    where = (e[1], eval(e[2], {}, {"buf": i & 1}))
                    if e[0] == "stage":
                        assert read.get(where, -1) < phase, f"step {i}: {where} is written while others may still read it"
                        holds[where] = ((batch, at[e[1]]), phase)
                        at[e[1]] += 1
                    else:
                        assert holds[where][1] < phase, f"step {i}: {where} is read while others may still write it"
                        read[where] = phase
                        yield holds[where][0], e[1]

            assert not list(run(begin, 0))
            seen = [[], []]
            if n_fast:
                for block, kind in run(front, 0):
                    seen[kind].append(block)
            for i in range(8):
                for block, kind in run(step if i < n_fast else slow, i):
                    seen[kind].append(block)
            if n_fast in (0, 8):                      # keys and values of all blocks, each once and in their order (and keys ahead of them)
                assert seen[1] == [(batch, i) for i in range(8)]
                assert seen[0][:8] == [(batch, i) for i in range(8)]
