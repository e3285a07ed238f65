"""The compiled kernel of attention over pages: descriptors of its inline loads, as those of the other kernels, and no register in memory."""
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
    test_isa_cpu.test_descriptors_of_inline_loads_are_settled("attention_paged.hip", tmp_path)


def test_registers_stay_on_the_chip(tmp_path):
    out = tmp_path / "k.s"
    subprocess.run(["hipcc", *bld.FLAGS, "-S", "--offload-device-only", os.path.join(bld.CSRC, "attention_paged.hip"), "-o", str(out)], check=True,
                   capture_output=True)
    assert {int(m) for m in re.findall(r"; ScratchSize: (\d+)", out.read_text())} == {0}
