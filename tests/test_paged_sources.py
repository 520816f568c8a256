"""What the merge kernel counts on: behind either attention kernel it may look at the step's plan before it waits."""
import os
import re

from tests.test_chained_sources import CSRC, LET_IN, WAIT

READ = lambda name: re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())                    # noqa: E731


def test_paged_attention_is_an_ordinary_launch_that_lets_the_merge_in():
    """What wrote the plan has ended when an ordinary launch starts, so the kernel may let the merge in at once; a chained one would have to wait first."""
    code = READ("attn_paged.cu")
    assert code.count(LET_IN) == 1 and WAIT not in code and "launch_chained" not in code
    assert re.findall(r"(\w+)<D, TWO><<<", code) == ["attn_paged_kernel"]
    assert code.count("return launch_paged_merge(") == 1 and code.index("<<<") < code.index("return launch_paged_merge(")


def test_the_merge_is_launched_behind_the_two_attention_kernels_only():
    code = READ("attn_tc.cu")
    assert re.findall(r"launch_chained\((hpd_merge_kernel<D, PAGED>)", code) == ["hpd_merge_kernel<D, PAGED>"]
    assert len(re.findall(r"launch_merge<", code)) == 3 and code.count("launch_merge<D, false>(p, MODE == kPrefill)") == 1
    assert code.index("launch_chained(hpd_attn_tc_kernel") < code.index("launch_merge<D, false>(p, MODE == kPrefill)")


def test_paged_appends_are_ordinary_launches():
    code = READ("append_paged.cu")
    assert LET_IN not in code and WAIT not in code and "launch_chained" not in code
    assert len(re.findall(r"append_(?:step|tokens)_kernel<(?:128|64)><<<", code)) == 4
