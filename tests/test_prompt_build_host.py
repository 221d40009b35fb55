"""The build refuses kernels of prompt attention that keep registers in scratch memory."""
import pytest

from paper_2106_10715_amd import build as B

KERNEL = """x/prompt.hip:850:1: remark: Function Name: _ZN3moe12_GLOBAL__N_1{name}ILb1EEEvNS_6prompt6PromptE [-Rpass-analysis=kernel-resource-usage]
x/prompt.hip:850:1: remark:     VGPRs: 256 [-Rpass-analysis=kernel-resource-usage]
x/prompt.hip:850:1: remark:     ScratchSize [bytes/lane]: {size} [-Rpass-analysis=kernel-resource-usage]
"""


def test_scratch_of_the_prompt_kernels():
    assert list(B.NO_SCRATCH) == ["prompt.hip"] and "prompt.hip" in B.SOURCES
    good = KERNEL.format(name="13prompt_kernel", size=0)
    assert B.check_remarks(good + "x/prompt.hip:9:1: warning: as it was\n" + good, "prompt.hip") == "x/prompt.hip:9:1: warning: as it was"
    with pytest.raises(RuntimeError, match="18prompt_join_kernel.* keeps 4 bytes"):
        B.check_remarks(good + KERNEL.format(name="18prompt_join_kernel", size=4), "prompt.hip")
    for text in ("", good.replace("ScratchSize", "Scratch"), "x/prompt.hip:9:1: warning: as it was"):
        with pytest.raises(RuntimeError, match="found to verify"):
            B.check_remarks(text, "prompt.hip")
