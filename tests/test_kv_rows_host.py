"""CPU tests of the key-value cache's calls over many rows: argument checks under
AddressSanitizer and UndefinedBehaviorSanitizer (tests/host_sanitize/
kv_rows_driver.cpp), constants against the header, and the registers of the
built kernels."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2510_23346_amd as bd
from test_build_resources import kernels  # noqa: F401  (a fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(os.path.join(ROCM, "include", "hip")),
                    reason="needs g++ and the HIP headers")
def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "kv_rows_host")
    here = os.path.join(ROOT, "tests", "host_sanitize")
    csrc = os.path.join(ROOT, "paper_2510_23346_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__",
           "-I", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"), "-I", csrc,
           os.path.join(here, "kv_rows_driver.cpp"), os.path.join(here, "launch_stubs.cpp"), os.path.join(csrc, "bdl_api.cpp"),
           "-L", os.path.join(ROCM, "lib"), "-lamdhip64", f"-Wl,-rpath,{os.path.join(ROCM, 'lib')}", "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and " 0 failed checks" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])


def test_constants_and_sizes():
    text = open(os.path.join(ROOT, "include", "bdlora.h")).read()
    macros = dict(re.findall(r"^#define (BDLORA_KV_\w+)\s+(\d+)", text, re.M))
    assert (int(macros["BDLORA_KV_INT8_BLOCK"]), int(macros["BDLORA_KV_BLOCK"])) == (bd.KV_INT8, bd.KV_BLOCK)
    page, _ = bd.kv_bytes(4, 2, 128, 64, 1000, 64, fmt=bd.KV_INT8)
    assert page == 2 * 2 * 64 * 128 + 2 * (64 // 16) * 8
    with pytest.raises(bd.BDLoRAError):
        bd.kv_bytes(4, 2, 128, 64, 1000, 64, fmt=bd.KV_INT8, weights=True)


# nothing is spilled, and matrix-core results, which are read after branches, stay
# out of accumulation registers (this compiler reads those too early there)
@pytest.mark.parametrize("name,count", [("kv_attend_sinks_kernel", 20), ("kv_weigh_sinks_kernel", 1), ("kv_prompt_kernel", 16),
                                        ("kv_append_norm_kernel", 4), ("kv_store_kernel", 8), ("kv_read_kernel", 12)])
def test_kernel_registers(kernels, name, count):  # noqa: F811
    mine = {k: v for k, v in kernels.items() if re.search(rf"\d+{name}[IE]", k)}
    assert len(mine) == count, sorted(mine)
    for k, v in mine.items():
        assert v["vgpr_spill_count"] == 0 and v["private_segment_fixed_size"] == 0 and v["agpr_count"] == 0, (k, v)
