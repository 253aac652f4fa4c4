"""The compiled kernel over rows of logits."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_16389_amd import xgemm as xg

LLVM = "/opt/rocm/llvm/bin/"


def test_what_waves_share_is_reached_as_lds(tmp_path):
    """No access through a generic address: one to LDS would wait for the
    batch of logits that is on its way."""
    if not (shutil.which("objcopy") and all(os.path.exists(LLVM + t) for t in ("clang-offload-bundler", "llvm-objdump"))):
        pytest.skip("objcopy / clang-offload-bundler / llvm-objdump not available")
    fat = tmp_path / "fat.bin"
    subprocess.run(["objcopy", "-O", "binary", "--only-section=.hip_fatbin", xg._LIB_PATH, str(fat)], check=True)
    data = fat.read_bytes()
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)]
    seen = 0
    for i, (a, b) in enumerate(zip(starts, starts[1:] + [len(data)])):
        part, co = tmp_path / ("part%d" % i), tmp_path / ("%d.co" % i)
        part.write_bytes(data[a:b])
        subprocess.run([LLVM + "clang-offload-bundler", "--unbundle", "--type=o", "--input=" + str(part),
                        "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", "--output=" + str(co)], check=True)
        text = subprocess.run([LLVM + "llvm-objdump", "-d", "--no-show-raw-insn", str(co)], check=True,
                              capture_output=True, text=True).stdout
        for name, body in re.findall(r"<(\S*logprob_rows\S*)>:\n(.*?)(?=\n\n|\Z)", text, re.S):
            seen += 1
            assert "ds_read" in body and not re.findall(r"\bflat_(?:load|store|atomic)\S*", body), name
    assert seen == 6
