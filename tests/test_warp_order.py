"""What the lanes of a warp may take for granted of one another, in the sources of the kernels: a place where they are not in step
breaks no result on most days, so the source is read."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_18183_b200", "csrc")


def _source(f):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(CSRC, f)).read(), flags=re.S)
    return re.sub(r"//[^\n]*", "", text)


def test_cluster_barriers_that_whole_warps_have_to_reach():
    """An aligned barrier is undefined where a warp's lanes reach it apart.  It stands in one helper, whose callers have met
    directly before; the operators on rows, which branch by lane in front of theirs, use the form without that condition."""
    for f in sorted(os.listdir(CSRC)):
        if not f.endswith((".cu", ".cuh", ".h")):
            continue
        text = _source(f)
        if not re.search(r"barrier\.cluster\.\w+[\w.]*\.aligned", text):
            continue
        helper = r"void (\w+)\(\) \{\s*asm volatile\(\"barrier\.cluster\.arrive\.release\.aligned;\" ::: \"memory\"\);\s*" \
                 r"asm volatile\(\"barrier\.cluster\.wait\.acquire\.aligned;\" ::: \"memory\"\);\s*\}"
        found = re.search(helper, text)
        assert found, f
        rest = re.sub(helper, "", text)
        assert "barrier.cluster" not in rest, f
        calls = [m.start() for m in re.finditer(r"%s\(\);" % found.group(1), rest)]
        assert calls, f
        for at in calls:
            assert re.search(r"__syncthreads\(\);\s*(if \(PAIR\) )?$", rest[:at]), (f, rest[at - 80:at])
