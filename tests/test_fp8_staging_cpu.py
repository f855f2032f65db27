"""The output staging of the e4m3 product's uncut wide tiles: a warp stores its
128 columns in four rounds through two buffers, some by a bulk store that reads
the buffer later, some directly.  A round may write its buffer only when the
bulk store of two rounds before has read it, for which it waits until at most
one bulk group is pending."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_22541_gb300", "csrc")


def _round():
    """The body of a round, without comments."""
    with open(os.path.join(CSRC, "fp8_ops.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    text = text[text.index("fp8_wide_kernel(const __grid_constant__"):]
    start = text.index("{", text.index("rd < 4; ++rd"))
    depth, end = 1, start + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
    return text[start:end]


def _commits():
    """(whether a round stored by a bulk store commits one group, whether a direct one does)."""
    body = _round()
    assert body.count("wait_group.read 1") == 1 and body.index("wait_group.read 1") < body.index("stage[lane * 4")
    # each commit's guard, the conditions it stands under and whether a round by a bulk store gets there
    by_bulk = by_hand = 0
    for m in re.finditer(r"bulk_commit_group\(\)", body):
        at, stack = m.start(), []
        for i, c in enumerate(body[:at]):
            if c == "{":
                stack.append(body[max(body.rfind(k, 0, i) for k in ";}{") + 1:i].strip())
            elif c == "}":
                stack.pop()
        assert body[body.rfind("\n", 0, at):at].strip() == "if (lane == 0)"
        conditions = [s for s in stack if s.startswith(("if", "else"))]
        left = re.findall(r"\b(?:continue|break|return)\b", body[:at])  # a bulk round leaves at its end, if at all
        assert conditions in ([], ["if (bulk)"]) and left in ([], ["continue"]), (conditions, left)
        if left:
            assert not conditions and re.search(r"if \(bulk\) \{[^{}]*continue;\s*\}|if \(bulk\) continue;", body[:at])
        by_bulk += not left
        by_hand += not conditions
    assert by_bulk <= 1 and by_hand <= 1
    return bool(by_bulk), bool(by_hand)


def _rounds(n, aligned):
    """Whether each of the four rounds of every half of 128 columns goes by a bulk store, as the kernel decides it."""
    return [[aligned and (n0 + 32 <= n or n % 8 == 0) for n0 in range(row0, row0 + 128, 32)]
            for row0 in range(0, -(-n // 128) * 128, 128)]


def test_the_model_decides_as_the_kernel_does():
    assert "const bool bulk = args.c_align == 16 && (n0 + 32 <= p.n || (p.n & 7) == 0);" in " ".join(_round().split())


@pytest.mark.parametrize("n", list(range(1, 300)) + [515, 556, 603, 4140])
@pytest.mark.parametrize("aligned", [True, False])
def test_no_buffer_is_written_while_a_bulk_store_may_read_it(n, aligned):
    by_bulk, by_hand = _commits()
    halves = _rounds(n, aligned)
    # a warp takes tiles one after another: an edge half after a full one, and after itself
    for order in ([halves[0], halves[-1], halves[-1]], [halves[-1], halves[0], halves[-1]]):
        groups = []   # committed groups, oldest first: the buffer each one reads (None: an empty group)
        for half in order:
            for rd, bulk in enumerate(half):
                # one group may stay pending, in the worst case the newest
                unread = groups[-1:]
                assert rd & 1 not in unread, (n, rd)
                if bulk and by_bulk:
                    groups.append(rd & 1)
                elif not bulk and by_hand:
                    groups.append(None)
