"""What the lanes of a warp may take for granted of one another, in the sources of the kernels: a place where they are not in step
breaks no result on most days, so the source is read."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_18183_b200", "csrc")


def _source(f):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(CSRC, f)).read(), flags=re.S)
    return re.sub(r"//[^\n]*", "", text)


def test_cluster_barriers_that_whole_warps_have_to_reach():
    """An aligned barrier is undefined where a warp's lanes reach it apart.  It stands in one helper of a file, in which the warp meets
    directly before, or whose callers have met as a block directly before."""
    for f in sorted(os.listdir(CSRC)):
        if not f.endswith((".cu", ".cuh", ".h")):
            continue
        text = _source(f)
        if not re.search(r"barrier\.cluster\.\w+[\w.]*\.aligned", text):
            continue
        helper = r"void (\w+)\(\) \{\s*(__syncwarp\(\);\s*)?asm volatile\(\"barrier\.cluster\.arrive\.release\.aligned;\" ::: \"memory\"\);\s*" \
                 r"asm volatile\(\"barrier\.cluster\.wait\.acquire\.aligned;\" ::: \"memory\"\);\s*\}"
        found = re.search(helper, text)
        assert found, f
        rest = re.sub(helper, "", text)
        assert "barrier.cluster" not in rest, f
        if found.group(2):
            continue
        calls = [m.start() for m in re.finditer(r"%s\(\);" % found.group(1), rest)]
        assert calls, f
        for at in calls:
            assert re.search(r"__syncthreads\(\);\s*(if \(PAIR\) )?$", rest[:at]), (f, rest[at - 80:at])


def test_listed_tokens_leave_the_row_before_other_lanes_sum_over_it():
    """A lane takes a listed token out of the staged row; other lanes read its place.  Votes, maxima and shuffles order no shared
    memory between them: a barrier of the warp has to stand in between."""
    text = _source("distill_kernels.cu")
    body = text[text.index(" k_distill_topk("):]
    out = [m.end() for m in re.finditer(r"ss\[e\] = from_f<TS>\(-INFINITY\);", body)]
    assert len(out) == 1
    behind = body[out[0]:]
    assert "__syncwarp();" in behind[:re.search(r"get<G>\(ss\b", behind).start()]
