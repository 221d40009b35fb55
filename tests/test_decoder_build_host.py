"""The build refuses attention kernels that keep registers in scratch memory."""
import pytest

from paper_2106_10715_amd import build as B

KERNEL = """\t.amdhsa_kernel _ZN3moe12_GLOBAL__N_1{name}ILb1EEEvNS0_4AttnEd
\t\t.amdhsa_group_segment_fixed_size 100352
\t\t.amdhsa_private_segment_fixed_size {size}
\t\t.amdhsa_kernarg_size 176
\t.end_amdhsa_kernel
"""


def test_scratch_of_the_attention_kernels(monkeypatch):
    text = ""
    monkeypatch.setattr(B, "_assembly", lambda src, part: text)
    assert list(B.MOST_SCRATCH) == ["attn.hip"] and "attn.hip" in B.SOURCES
    text = KERNEL.format(name="16attn_wave_kernel", size=0) + KERNEL.format(name="11attn_kernel", size=8) + KERNEL.format(name="9kv_kernel", size=400)
    B._check_scratch("attn.hip")
    assert B.check_scratch(text, "attn_", 16) == 2
    for size in (20, 256):
        text = KERNEL.format(name="16attn_wave_kernel", size=0) + KERNEL.format(name="11attn_kernel", size=size)
        with pytest.raises(RuntimeError, match=f"11attn_kernel.* keeps {size} bytes"):
            B._check_scratch("attn.hip")
    text = KERNEL.format(name="11attn_kernel", size=0).replace("private_segment_fixed_size", "private")
    with pytest.raises(RuntimeError, match="scratch memory"):
        B._check_scratch("attn.hip")
    for text in ("", KERNEL.format(name="9kv_kernel", size=0)):
        with pytest.raises(RuntimeError, match="found to verify"):
            B._check_scratch("attn.hip")
