"""The instructions that gfx950 wants between a write of m0 and a load into LDS that goes by it: in code written by hand the compiler does not
put one there."""
import os
import re
import subprocess

import pytest

from paper_2510_24273_amd import build

LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")


def _instructions(tmp_path):
    bundle, code = str(tmp_path / "bundle"), str(tmp_path / "code")
    run = lambda *a: subprocess.run([os.path.join(LLVM, a[0]), *a[1:]], check=True, capture_output=True)
    run("llvm-objcopy", "--dump-section", ".hip_fatbin=" + bundle, build.LIB, os.devnull)
    data, magic = open(bundle, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__"   # (one bundle for each source)
    starts = [m.start() for m in re.finditer(magic, data)]
    for k, at in enumerate(starts):
        one = str(tmp_path / f"bundle{k}")
        open(one, "wb").write(data[at:starts[k + 1] if k + 1 < len(starts) else len(data)])
        run("clang-offload-bundler", "--unbundle", "--type=o", "--input=" + one, "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", "--output=" + code)
        out = subprocess.Popen([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", "--no-leading-addr", code], stdout=subprocess.PIPE, text=True)
        for line in out.stdout:
            yield line.split("//")[0].strip()
        assert out.wait() == 0


@pytest.mark.skipif(not os.path.exists(os.path.join(LLVM, "llvm-objdump")), reason="no LLVM tools")
def test_a_load_into_lds_does_not_follow_the_write_of_m0(tmp_path):
    if build.is_stale():
        build.build()
    loads, close, last = 0, 0, ""
    for ins in _instructions(tmp_path):
        if "_load_lds_" in ins or re.match(r"buffer_load\S* .* lds", ins):
            loads += 1
            close += bool(re.match(r"s_\w+ m0,", last))
        if ins:
            last = ins
    assert loads > 1000 and close == 0, (loads, close)
