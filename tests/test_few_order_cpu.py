"""What one thread of the few-token layer acquires, other threads read: between
the acquire and their reads stands a barrier that orders memory (a shuffle or a
vote orders none)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_22541_gb300", "csrc")


def _text():
    with open(os.path.join(CSRC, "few.cu")) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_the_finisher_orders_the_slices_sums_before_it_adds_them():
    text = _text()
    uses = [m.start() for m in re.finditer(r"arrive_acq_rel\(a\.counters", text)]
    assert len(uses) == 1
    after = text[uses[0]:text.index("write_h<FP8>(", uses[0])]
    assert "if (lane == 0) last = arrive_acq_rel" in text
    assert "__syncwarp()" in after


def test_the_other_acquires():
    text = _text()
    # by a thread of the epilogue: a barrier of its warps follows
    assert re.search(r"if \(!epi_all\(tid != 0 \|\| bounded_wait\(\[&\]\(\) \{ return ld_acquire\(claims \+ 1\)", text)
    done = text.index("ld_acquire(done)")
    assert text.index("epi_all(ok)", done) < text.index("write_out(a, s, T", done)
    # by the thread that issues the copies of what it has acquired
    ready = text.index("ld_acquire(ready)")
    assert "fence_proxy_async_all()" in text[ready:text.index("bulk_load(", ready)]
    assert text.count("ld_acquire(") == 4  # (and the definition)
