"""Registers of the attention layer's kernels: what their figures hang on is that nothing is spilled, and how many waves a
SIMD (512 registers in eights) they leave room for."""
import re
import subprocess

import pytest

from paper_2609_33051_amd import build
from test_kernel_resources import _code_objects, _metadata


@pytest.fixture(scope="module")
def registers():
    """{"attention_kernel<unsigned short, 128, ...>": (registers, spilled registers)}"""
    out = {}
    for elf in _code_objects(open(build.LIB, "rb").read()):
        for m in _metadata(elf):
            for k in m["amdhsa.kernels"]:
                out[k[".name"]] = (k[".vgpr_count"], k[".vgpr_spill_count"])
    names = subprocess.run(["c++filt"], input="\n".join(out), capture_output=True, text=True, check=True).stdout
    return {d.replace("void skssm::(anonymous namespace)::", "").split("(")[0]: out[n] for n, d in zip(out, names.split("\n")) if "anonymous" in d}


# single tokens: three waves a SIMD (four of 64 channels), by which the workgroups that keys are shared out to are counted
@pytest.mark.parametrize("kernel,most", [
    (r"attention_kernel<unsigned short, 64, 1, true, .*", 128), (r"attention_kernel<unsigned short, (96|128), 1, true, .*", 168),
    (r"attention_kernel<unsigned short, .*", 256), (r"attention_kernel<float, .*", 512), (r"prompt_kernel<.*", 256), (r"join_kernel<.*", 128),
    (r"append_kernel<.*", 168), (r"read_kernel<.*", 64)])
def test_registers(registers, kernel, most):
    found = {n: v for n, v in registers.items() if re.fullmatch(kernel, n)}
    assert found
    for name, (regs, spilled) in found.items():
        assert regs <= most and spilled == 0, (name, regs, spilled)
