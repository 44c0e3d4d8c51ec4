"""What the sources of the 8-bit training operators may not contain, whatever the numbers they give."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1501_06633_b200", "csrc")


def code_of(path):
    """A source file without its comments."""
    text = re.sub(r"/\*.*?\*/", " ", open(path).read(), flags=re.S)
    return re.sub(r"//[^\n]*", " ", text)


def test_kernels_that_start_early_have_no_read_only_loads():
    """A kernel that waits for the one before it (griddepcontrol.wait) is resident while its inputs are
    written: loads that assume memory which nobody writes during the kernel (ld.global.nc, as __ldg and
    const __restrict__ give) are not ordered by that wait."""
    early = [p for p in glob.glob(os.path.join(CSRC, "*.cu*")) if "wait_for_previous()" in code_of(p)]
    assert len(early) >= 5
    for path in early + [os.path.join(CSRC, "ptx_util.cuh"), os.path.join(CSRC, "umma_util.cuh")]:
        found = re.findall(r"__ldg|ld\.global\.nc|\.nc\.|__restrict__|__builtin_nontemporal_load|tex1Dfetch", code_of(path))
        assert not found, (os.path.basename(path), found)
