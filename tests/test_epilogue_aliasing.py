"""A residual may be the output itself (include/brq_residual.h), so no kernel that reads one may promise the compiler that its output's address is
nobody else's: on such a promise a residual's load could be moved across a store.  Looked at in the kernels' arguments as the front end hands them on
(LLVM IR before any pass), on the CPU."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_04214_amd.build import FLAGS

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_04214_amd", "csrc")
pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")


def arguments(signature):
    """The arguments of a definition, split at its own commas."""
    depth, out = 0, [""]
    for ch in signature:
        depth += (ch in "([{<") - (ch in ")]}>")
        if ch == "," and depth == 0:
            out.append("")
        else:
            out[-1] += ch
    return [a.strip() for a in out]


# kernels with an epilogue in each source, two or four to a template: the tiles' shapes are the products' own
@pytest.mark.parametrize("source,least", [("mxfp4_gemm.hip", 3), ("mxfp4_gemm_tiled.hip", 4), ("mxfp4_gemm_mid_with.hip", 14), ("mxfp4_gemm_few.hip", 10), ("mxfp4_gemm_split.hip", 4)])
def test_output_of_a_kernel_with_a_residual(source, least, tmp_path):
    ll = str(tmp_path / "k.ll")
    r = subprocess.run(["hipcc"] + FLAGS + ["--cuda-device-only", "-S", "-emit-llvm", "-Xclang", "-disable-llvm-passes", os.path.join(CSRC, source), "-o", ll],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-3000:]
    text = open(ll).read()
    # types that are an Epilogue or hold one
    holders = {m[1] for m in re.finditer(r'^(%"struct\.brq::EpilogueArg[^"]*") = type \{ %"struct\.brq::Epilogue" \}', text, re.M)} | {'%"struct.brq::Epilogue"'}
    seen = 0
    for m in re.finditer(r"^define [^\n]*amdgpu_kernel void @([^\s(]+)\((.*?)\) (?:#\d+|comdat)", text, re.M):
        args = arguments(m[2])
        last = [i for i, a in enumerate(args) if any("byref(%s)" % h in a for h in holders)]
        if not last:
            continue
        seen += 1
        outputs = [a for a in args[: last[0]] if a.startswith("ptr addrspace(1)")]
        assert outputs and "noalias" not in outputs[-1], m[1]
        assert all("noalias" in a for a in outputs[:-1]), m[1]         # (operands and slices: inputs that no output is; says that the attribute is what is looked at)
    assert seen >= least, "%d kernels with an epilogue seen" % seen
