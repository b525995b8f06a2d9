"""The packed-prompt kernel on the host, one CTA with a thread per CUDA thread (cta_emulator/emu.h): that it walks through its
units to the end whatever comes late, and that nothing of it is under way when it leaves because a bounded wait has run out.
The latter cannot be provoked on a GPU."""
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2604_16734_b200", "csrc")
CUDA = "/usr/local/cuda/include"
KVC_ETIMEOUT = -4


@pytest.fixture(scope="module")
def emulator(tmp_path_factory):
    if not shutil.which("g++") or not os.path.exists(os.path.join(CUDA, "cuda_bf16.h")):
        pytest.skip("needs g++ and the CUDA headers")
    tmp = tmp_path_factory.mktemp("prompt_emulator")

    def source(name):
        text = open(os.path.join(CSRC, name)).read()
        text = re.sub(r"^#(include|pragma once).*$", "", text, flags=re.M)
        text = re.sub(r"asm volatile\(\"mov\.u64 %0, %%globaltimer.*$", "t = 0;", text, flags=re.M)
        return text.replace("extern __shared__ uint8_t smem_raw[];", "extern uint8_t* smem_raw;")

    ptx = source("ptx.cuh")                                       # the bounded waits are the library's, on the emulator's barriers
    waits = re.findall(r"^__device__ __forceinline__ (?:bool|void) (?:mbar_wait|mbar_wait_spin|word_wait_spin|mbar_drain)\(.*?^}\n", ptx, flags=re.M | re.S)
    limit = re.search(r"^static constexpr int kDefaultWaitLimitK.*$", ptx, flags=re.M).group(0)
    parts = ["namespace kvc {", limit, *waits, "}", source("geom.cuh"), source("kernels_tc.cuh"), source("prompt.cuh")]
    (tmp / "kernels.h").write_text("\n".join(parts))
    exe = str(tmp / "emulator")
    subprocess.run(["g++", "-std=c++20", "-O1", "-w", "-pthread", "-I", str(tmp), "-I", CUDA, "-I", os.path.join(HERE, "cta_emulator"),
                    os.path.join(HERE, "cta_emulator", "prompt.cpp"), "-o", exe], check=True)

    def run(**kw):
        r = subprocess.run(["timeout", "60", exe] + [f"{k}={v}" for k, v in kw.items()], capture_output=True, text=True)
        assert r.returncode != 124, "the kernel does not end"
        lines = r.stdout.splitlines()
        assert lines and lines[-1].startswith("status"), r.stdout + r.stderr
        return [x[len("FAULT "):] for x in lines[:-2]], int(lines[-1].split()[1]), int(lines[-2].split()[1])
    return run


UNITS = [dict(lens="1"), dict(lens="128"), dict(lens="700"), dict(lens="129,1,256,300"), dict(lens="40,70,500", G=4, Hkv=2), dict(lens="1,1,1", G=7, Hkv=3),
         dict(lens="33,900", G=3)]


@pytest.mark.parametrize("units", UNITS)
def test_every_row_of_every_unit_is_written(emulator, units):
    assert emulator(limit_ms=2000, **units) == ([], 0, 0)


@pytest.mark.parametrize("late", [dict(load_ms="0:40"), dict(load_ms="2:40,5:60,9:30"), dict(load_ms="3:50,6:50,7:50,8:50"), dict(mma_us=400), dict(load_ms="1:30,4:30,12:30", mma_us=200)])
def test_what_comes_late_only_takes_longer(emulator, late):
    assert emulator(limit_ms=2000, lens="129,1,256,300", **late) == ([], 0, 0)


@pytest.mark.parametrize("late", [dict(load_ms="0:200"), dict(load_ms="2:200"), dict(load_ms="4:200"), dict(load_ms="5:200,6:150"), dict(load_ms="9:200"), dict(load_ms="11:200,12:120"),
                                  dict(load_ms="2:60,3:60", suspend_ms="9:400,10:400"), dict(load_ms="7:60", suspend_ms="8:300,11:300")])
def test_a_wait_that_runs_out_leaves_nothing_under_way(emulator, late):
    faults, status, _ = emulator(limit_ms=20, lens="129,1,256,300", **late)
    assert status == KVC_ETIMEOUT and faults == []


def test_slow_mmas_are_waited_for(emulator):
    faults, status, _ = emulator(limit_ms=5, lens="300,200", mma_us=4000)
    assert status == KVC_ETIMEOUT and faults == []
