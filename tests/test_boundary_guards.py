"""The guards of test_compiler_guards.py on the code of the operators at the token boundary:
no kernel spills to scratch, none needs more than 256 VGPRs, and no wide store's data
registers are rewritten closely behind it."""
import os
import subprocess

import pytest

from test_compiler_guards import CSRC, FLAGS, HIPCC, kernel_budgets, store_data_hazards

SOURCES = ("sample.hip", "embed.hip", "block_norm.hip", "block_norm_bf16.hip", "block_norm_f32.hip",
           "block_norm_mixed.hip")


@pytest.fixture(scope="module")
def device_asm(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    tmp = tmp_path_factory.mktemp("asm")
    procs = [(src, os.path.join(tmp, src + ".s")) for src in SOURCES]
    procs = [(src, out, subprocess.Popen([HIPCC, *FLAGS, os.path.join(CSRC, src), "-o", out],
                                         stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True,
                                         cwd=str(tmp))) for src, out in procs]
    asm = {}
    for src, out, p in procs:
        _, err = p.communicate(timeout=900)
        assert p.returncode == 0, err[-3000:]
        asm[src] = open(out).read()
    return asm


def test_registers(device_asm):
    seen = 0
    for src, asm in device_asm.items():
        for name, vgpr, agpr, scratch in kernel_budgets(asm):
            seen += 1
            assert vgpr <= 256 and agpr == 0 and scratch == 0, (src, name, vgpr, agpr, scratch)
    assert seen > 100


def test_wide_store_data_is_not_rewritten_early(device_asm):
    found = {src: store_data_hazards(asm) for src, asm in device_asm.items()}
    assert not any(found.values()), {s: f[:3] for s, f in found.items() if f}
