"""Static check of the gradients' gfx950 code (CPU: hipcc cross-compiles): the wavefronts that a kernel's
launch bound asks for are those that its LDS lets on a SIMD, and the registers it got leave room for them.
The compiler drops a request that LDS does not allow, without a word."""

import os
import re
import subprocess

from test_wait_states import CSRC, HIPCC, ROOT, listing

LDS = 160 * 1024  # bytes of a compute unit, which has four SIMDs of 512 registers a lane


def requests():
    """Kernel name -> wavefronts on a SIMD that its launch bound asks for."""
    from paper_2606_23019_amd import build
    text = subprocess.run([HIPCC] + [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")] + [
        "-I", os.path.join(ROOT, "include"), "--cuda-device-only", "-S", "-emit-llvm", "-Xclang",
        "-disable-llvm-passes", "-o", "-", os.path.join(CSRC, "attn_bwd.hip")], check=True,
        capture_output=True, text=True).stdout
    asked = dict(re.findall(r'^attributes (#\d+) = .*"amdgpu-waves-per-eu"="(\d+)', text, re.M))
    return {name: int(asked[group]) for name, group in re.findall(
        r"^define amdgpu_kernel void @(\S+bwd_kernel\w+)\(.*\) (#\d+) ", text, re.M)}


def test_gradients_occupancy(tmp_path):
    text = listing("attn_bwd.hip", tmp_path)
    asked = requests()
    assert len(asked) == 12
    for block in text.split("  - .agpr_count")[1:]:
        field = lambda key: int(re.search(r"\.%s:\s+(\d+)" % key, block).group(1))
        name = re.search(r"\.name:\s+(\S+)", block).group(1)
        if name not in asked:
            continue
        waves = field("max_flat_workgroup_size") // 64
        by_lds = -(-(LDS // field("group_segment_fixed_size") * waves) // 4)
        assert asked[name] <= by_lds, (name, asked[name], by_lds)
        registers = -(-field("vgpr_count") // 8) * 8
        assert 512 // registers >= asked[name], (name, asked[name], registers)
