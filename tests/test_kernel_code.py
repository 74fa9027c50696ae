"""The machine code of the kernels built here, where correctness or speed hangs on it:
a scalar write of M0 and a load into LDS that takes its address from M0 need one
wait state between them, which the compiler does not add inside assembly text;
and a kernel past its line of registers loses a wave per SIMD."""
import os
import re
import subprocess

import pytest

from paper_2609_33051_amd import build
from test_kernel_resources import _code_objects, kernels  # noqa: F401

OBJDUMP = os.path.join(os.path.dirname(os.path.realpath(build.HIPCC)), "..", "llvm", "bin", "llvm-objdump")


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    """The instructions of the code object that holds the 8-bit products."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    if not os.path.exists(build.LIB):
        build.build()
    for elf in _code_objects(open(build.LIB, "rb").read()):
        if b"matmul_tile_kernel" in elf:
            f = tmp_path_factory.mktemp("code") / "matmul.elf"
            f.write_bytes(elf)
            text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", f], capture_output=True, text=True, check=True).stdout
            return [line.split("//")[0].strip() for line in text.split("\n") if re.match(r"^\s+[a-z]", line)]
    pytest.fail("no code object holds the 8-bit products")


def test_m0_is_settled_before_a_load_into_lds(listing):
    loads = [i for i, x in enumerate(listing) if re.match(r"(global|buffer)_load_lds_|buffer_load_\w+ .*\blds\b", x)]
    assert len(loads) > 100
    for i in loads:
        assert not re.match(r"s_\w+ m0,", listing[i - 1]), f"{listing[i - 1]} / {listing[i]}"
        assert any(re.match(r"s_\w+ m0,", x) for x in listing[i - 4:i]), listing[i - 4:i + 1]


# waves a SIMD (512 registers in eights) that the kernels' figures hang on: the scan's bf16 workgroups come two a CU
@pytest.mark.parametrize("kernel,most", [
    (r"scan_kernel<unsigned short, .*", 256), (r"scan_kernel<float, .*", 512), (r"matmul_tile_kernel<.*", 256),
    (r"conv_kernel<.*", 128), (r"conv_token_kernel<.*", 128), (r"norm_kernel<.*", 128)])
def test_mixer_kernel_registers(kernels, kernel, most):
    found = {n: v for n, v in kernels.items() if re.fullmatch(kernel, n)}
    assert found
    for name, (regs, spilled) in found.items():
        assert regs <= most and spilled == 0, (name, regs, spilled)


def test_the_loads_bases_are_settled_too(listing):
    """A scalar register that a vector instruction writes is read by a memory instruction five wait states later at the earliest."""
    for i, x in enumerate(listing):
        if "_load_lds_" not in x:
            continue
        pair = {int(n) for n in re.search(r"s\[(\d+):(\d+)\]", x).groups()}
        states = 0
        for y in reversed(listing[max(0, i - 5):i]):
            written = re.match(r"v_\w+ s(?:\[(\d+):(\d+)\]|(\d+)),", y)
            if written and states < 5:
                assert not pair & {int(n) for n in written.groups() if n}, f"{y} / {x}"
            wait = re.match(r"s_nop (\d+)", y)
            states += int(wait.group(1)) + 1 if wait else 1
