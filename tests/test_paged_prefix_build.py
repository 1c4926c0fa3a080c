"""What the compiler makes of the kernels of common starts."""
import os
import subprocess

from paper_2605_23081_amd import build


def test_the_walk_of_common_tokens_reloads_no_registers(tmp_path):
    """Blocks are on their way during the walk, by LDS DMA or in registers, and a reload of a spilled register waits for them.  Of the walk of own tokens,
    32 heads of 256 channels alone do it."""
    source, listing = "thrift_paged_prefix.hip", tmp_path / "prefix.s"
    subprocess.run(["hipcc", *build.flags(source), "-S", "--cuda-device-only", os.path.join(build.CSRC, source), "-o", str(listing)],
                   check=True, capture_output=True)
    text = listing.read_text()
    assert sum(f"prefix_kernelINS_{t}ELi{D}ELb{c}E" in text for t in ("3F16", "4BF16") for D in (64, 128, 256) for c in (0, 1)) == 12
    assert all("paged_decode_kernel" in k and "Li256ELi2ELb0E" in k for k in build.scratch_in_loops(text))
