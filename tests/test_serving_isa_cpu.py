"""The compiled 8-bit products: descriptors of their inline loads, as those of the other kernels, and no register of these operators' kernels in memory."""
import os
import re
import shutil
import subprocess

import pytest

import test_isa_cpu
from paper_2512_12131_amd import build as bld

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")


def test_descriptors_of_inline_loads_are_settled(tmp_path, monkeypatch):
    # (loads that pass by the caches among them)
    monkeypatch.setattr(test_isa_cpu, "LOAD", re.compile(r"buffer_load_dword(?:x4)? v\d+, s\[(\d+):(\d+)\], 0 offen (?:nt )?lds"))
    test_isa_cpu.test_descriptors_of_inline_loads_are_settled("gemm_q8.hip", tmp_path)


@pytest.mark.parametrize("src", ["gemm_q8.hip", "quant_q8.hip", "beam_select.hip", "kv_pages.hip"])
def test_registers_stay_on_the_chip(src, tmp_path):
    out = tmp_path / "k.s"
    subprocess.run(["hipcc", *bld.FLAGS, "-S", "--offload-device-only", os.path.join(bld.CSRC, src), "-o", str(out)], check=True, capture_output=True)
    assert {int(m) for m in re.findall(r"; ScratchSize: (\d+)", out.read_text())} == {0}
