"""The loads into LDS that the compiler does not see (dma.h), in what it makes of the
kernels that use them: m0 belongs to those blocks alone, and no load takes its scalar
address from a register that a vector instruction may just have written."""

import concurrent.futures
import os
import re
import subprocess

import pytest

from paper_2506_20194_amd import build as B

USERS = ("packed.hip", "paged.hip")
# what reads m0 without naming it
READS_M0 = ("global_load_lds", "buffer_load_lds", "ds_gws", "ds_append", "ds_consume", "ds_ordered", "ds_read_addtid",
            "ds_write_addtid", "s_movrel", "v_movrel", "s_sendmsg", "v_interp")


def test_every_block_names_m0():
    text = open(os.path.join(B.CSRC, "dma.h")).read()
    blocks = re.findall(r"asm volatile\((.*?)\);", text, re.S)
    assert len(blocks) == 6
    for b in blocks:
        assert "global_load_lds" in b and '"memory", "m0"' in b, b


def test_users_are_known():
    named = {f for f in os.listdir(B.CSRC) if f.endswith((".hip", ".h")) and f != "dma.h"
             and '"dma.h"' in open(os.path.join(B.CSRC, f)).read()}
    assert named == set(USERS)


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    out = tmp_path_factory.mktemp("listing")
    jobs = [[B.HIPCC, *B.FLAGS, "-w", "--cuda-device-only", "-S", os.path.join(B.CSRC, f), "-o", str(out / (f + ".s"))]
            for f in USERS]
    with concurrent.futures.ThreadPoolExecutor(len(jobs)) as ex:
        for r in ex.map(lambda j: subprocess.run(j, capture_output=True, text=True), jobs):
            assert r.returncode == 0, r.stderr[-2000:]
    return {f: (out / (f + ".s")).read_text().splitlines() for f in USERS}


@pytest.mark.parametrize("name", USERS)
def test_blocks(listings, name):
    block, loads = None, 0
    for line in listings[name]:
        code = line.split(";")[0].strip()
        if "#ASMSTART" in line:
            block = []
        elif "#ASMEND" in line:
            block = None
        elif code and not code.startswith(".") and not code.endswith(":"):
            if block is None:
                assert not re.search(r"\bm0\b", code) and not code.startswith(READS_M0), code
                continue
            block.append(code)
            if code.startswith("global_load_lds"):
                loads += 1
                assert re.fullmatch(r"s_mov_b32 m0, \w+", block[0]), block
                address = code.split(",")[1].split()[0]
                if address == "off":
                    assert block[1] == "s_nop 0", block
                else:
                    assert block[1].startswith(f"s_mov_b64 {address},"), block
    assert loads > 50
