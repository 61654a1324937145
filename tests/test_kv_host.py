"""The key-value cache's host code under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU; tests/host_sanitize/kv_driver.cpp), and the
binding's constants against the header."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2510_23346_amd as bd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(os.path.join(ROCM, "include", "hip")),
                    reason="needs g++ and the HIP headers")
def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "kv_host")
    here = os.path.join(ROOT, "tests", "host_sanitize")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__",
           "-I", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(ROOT, "paper_2510_23346_amd", "csrc"),
           os.path.join(here, "kv_driver.cpp"), os.path.join(here, "launch_stubs.cpp"),
           os.path.join(ROOT, "paper_2510_23346_amd", "csrc", "bdl_api.cpp"),
           "-L", os.path.join(ROCM, "lib"), "-lamdhip64", f"-Wl,-rpath,{os.path.join(ROCM, 'lib')}", "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and " 0 failed checks" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "bdlora.h")).read()
    macros = dict(re.findall(r"^#define (BDLORA_KV_\w+)\s+(\d+)", text, re.M))
    assert (int(macros["BDLORA_KV_BF16"]), int(macros["BDLORA_KV_FP8_E4M3"])) == (bd.KV_BF16, bd.KV_FP8_E4M3)


def test_sizes():
    page, ws = bd.kv_bytes(4, 1, 128, 64, 1000, 64)
    assert page == 2 * 64 * 128 * 2 and ws < 16 << 20
    page8, _ = bd.kv_bytes(4, 1, 128, 64, 1000, 64, fmt=bd.KV_FP8_E4M3)
    assert 2 * page8 == page
    pagew, wsw = bd.kv_bytes(4, 1, 128, 64, 1000, 64, weights=True)
    assert pagew == page + 8 * 64 and wsw - ws >= 4 * 4 * 64 * 1000
    with pytest.raises(bd.BDLoRAError):
        bd.kv_bytes(4, 1, 80, 64, 1000, 64)


@pytest.mark.parametrize("at", range(6))
def test_sizes_that_32_bits_do_not_hold_are_refused(at):
    good = [4, 1, 128, 64, 1000, 64]
    for big in (2 ** 32 + good[at], 2 ** 31, -2 ** 32 + good[at]):
        with pytest.raises(ValueError):
            bd.kv_bytes(*good[:at], big, *good[at + 1:])
