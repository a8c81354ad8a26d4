"""What the compiler made of the kernels of attention over the paged key/value cache (the library's own objects; no GPU)."""
import os
import re
import subprocess

import pytest

from paper_2410_09426_amd import build

LLVM = "/opt/rocm/lib/llvm/bin"


def _private_bytes(tmp_path, source):
    """Bytes of memory of its own that a thread of each kernel has: {name: bytes}."""
    obj = os.path.join(build.CSRC, source.replace(".hip", ".o"))
    tools = [os.path.join(LLVM, t) for t in ("llvm-objcopy", "clang-offload-bundler", "llvm-readelf")]
    if not all(os.path.exists(f) for f in (*tools, obj)):
        pytest.skip("needs ROCm's llvm tools and the library's object files (python -m paper_2410_09426_amd.build)")
    fat, code = str(tmp_path / "fat"), str(tmp_path / "code")
    subprocess.run([tools[0], f"--dump-section=.hip_fatbin={fat}", obj, str(tmp_path / "rest.o")], check=True, capture_output=True)
    subprocess.run([tools[1], "--type=o", f"--input={fat}", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--output={code}", "--unbundle"], check=True,
                   capture_output=True)
    notes = subprocess.run([tools[2], "--notes", code], check=True, capture_output=True, text=True).stdout
    return {n: int(b) for n, b in re.findall(r"\.name:\s+(_Z\S+)\n\s+\.private_segment_fixed_size:\s+(\d+)", notes)}


def test_attention_keeps_no_array_in_memory(tmp_path):
    """A load from private memory in the step loop waits for the codes that are on their way to LDS, all of them.  Where 8 or 16 waves share the registers
    a few values that the loop does not touch may be spilled; nothing else lies in memory."""
    kernels = _private_bytes(tmp_path, "fq_attention.hip")
    for name in ("whole_attention_kernel", "balanced_attention_kernel", "shared_attention_kernel"):
        assert sum(name in k for k in kernels) >= 18, name
    for k, used in kernels.items():
        crowded = re.search(r"whole_attention_kernelILi(\d)ELi(\d)ELi1ELi(8|16)E", k)
        assert used == 0 or (crowded and crowded.group(1, 2) in (("3", "3"), ("3", "4"), ("4", "3")) and used <= 24), (k, used)
