"""A rule that the tcgen05 form of packed attention keeps, read in its source (no GPU)."""
import pathlib
import re

import paper_2607_20507_gb300 as package

SOURCE = pathlib.Path(package.__file__).parent / "csrc" / "packed_attention_tc.cuh"


def test_warps_that_issue_products_wait_for_them_at_their_end():
    """Tensor memory is given back after every warp that commits products has waited for its own on a barrier of one
    phase; a parity of the barriers that phases share does not tell, after a wait gave up, which phase is done."""
    text = SOURCE.read_text()
    functions = dict(re.findall(r"__device__ __forceinline__ void (tc_\w+)\(([^{]*\{.*?\n\})", text, re.S))
    issuing = {name for name, body in functions.items() if "tc_commit(&" in body}
    assert issuing == {"tc_issue_scores", "tc_issue_values", "tc_softmax"}
    drains = {name: re.findall(r"tc_drain\(&bars\.drained\[(\d)\]", functions[name]) for name in issuing}
    assert sorted(sum(drains.values(), [])) == ["0", "1", "2"]
    for name in issuing:     # nothing is issued past it
        assert "tc_commit" not in functions[name].split("tc_drain")[-1]
    kernel = text[text.index("packed_attention_tc_kernel(const"):]
    assert kernel.index("tc_softmax<") < kernel.rindex("__syncthreads()") < kernel.index("tcgen05.dealloc")
    assert len(re.findall(r"mbar_init\(&bars\.drained\[i\], 1\)", kernel)) == 1


def test_the_self_test_runs_the_bounded_waits():
    """Packed attention waits on mbarriers by two functions alone, and the self-test lets both run out."""
    selftest = (SOURCE.parent / "selftest.cu").read_text()
    assert "!mbar_wait_bounded(" in selftest and re.search(r"\btc_wait\(", selftest)
    for f in (SOURCE, SOURCE.with_name("packed_attention.cu")):
        assert not re.search(r"mbarrier\.|mbar_(try|test)_wait|tc_asleep|tc_wait_long", f.read_text()), f.name
