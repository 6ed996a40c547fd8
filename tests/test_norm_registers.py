"""The norm's kernels hold a row in registers: none of them has scratch memory.  (Reads the library's own code objects;
no GPU needed.)"""

import os
import re
import shutil
import subprocess

import pytest

BIN = "/opt/rocm/llvm/bin"
TOOLS = [os.path.join(BIN, n) for n in ("llvm-readelf", "clang-offload-bundler")]


@pytest.mark.skipif(not all(os.path.exists(t) for t in TOOLS) or shutil.which("objcopy") is None, reason="needs the compiler's tools")
def test_no_scratch_memory(tmp_path):
    from paper_2412_15803_amd import build

    obj = os.path.join(build.BUILD_DIR, "wq_norm.o")
    if not os.path.exists(obj):
        build.build(verbose=False)
    bundle, code = tmp_path / "bundle", tmp_path / "code"
    subprocess.run(["objcopy", "--dump-section", f".hip_fatbin={bundle}", obj, str(tmp_path / "copy.o")], check=True)
    subprocess.run([TOOLS[1], "--unbundle", "--type=o", f"--input={bundle}", f"--output={code}", f"--targets=hipv4-amdgcn-amd-amdhsa--{build.ARCH}"], check=True)
    notes = subprocess.run([TOOLS[0], "--notes", str(code)], check=True, capture_output=True, text=True).stdout
    sizes = dict(re.findall(r"\.name: +(\S+)\n(?:.*\n)*? +\.private_segment_fixed_size: (\d+)", notes))
    assert len(sizes) == 27 and all("norm_kernel" in n for n in sizes)
    assert {n: s for n, s in sizes.items() if s != "0"} == {}
