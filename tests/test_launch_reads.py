"""What kernels may read before their grid wait (see common.cuh): those that read what kernels before their predecessor have written wait
first behind a kernel that triggers early, read through L2, and are named there; all others read nothing of global memory before
it.  A read moved breaks no result on most days; so the source is read."""
import re

from tests.test_launch_order import CSRC, _sources


def test_reads_before_the_wait_are_guarded_and_through_l2():
    guarded = set()
    for f, text in _sources():
        for part in text.split("__global__")[1:]:
            name = re.search(r"\b(k_[a-z0-9_]+)\s*\(", part).group(1)
            body = part[part.index("{"):]
            first = re.search(r"(if \([^;{}]*early\) )?pdl_wait\(\);", body)
            assert first, (f, name)
            assert not re.search(r"__ldg\(|__ldcg\(|__ldcs\(", body[:first.start()]), (f, name)
            if first.group(1):
                guarded.add(name)
                rest = body[first.end():]
                ahead = rest[:re.search(r"(?<!early\) )pdl_wait\(\);", rest).start()]
                assert "__ldg(" not in ahead, (f, name)
    assert guarded == {"k_gemm_skinny", "k_attention_tma", "k_accept_persistent", "k_commit", "k_pairs"}


def test_the_rule_names_them():
    text = open(CSRC + "/common.cuh").read()
    rule = text[text.index("All that precedes a late kernel"):text.index("struct Stream")]
    assert "Five kernels" in rule and "k_pairs" in rule and "k_commit" in rule
