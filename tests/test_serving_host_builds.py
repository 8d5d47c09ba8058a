"""Host code of the serving entries in builds of its own: with sanitizers on the host pass, and against stand-ins for HIP that
see which LDS limits are raised on which device.  No GPU code runs."""
import os
import shutil
import subprocess

import pytest

from paper_2502_00425_amd import binding as mq
from paper_2502_00425_amd import build as hip_build
from test_sanitizers import OUT, ROOT, SAN, _run

SOURCES = ["qk_norm.hip", "paged_attention.hip", "lora.hip"]


def test_serving_host_paths_under_asan_and_ubsan():
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    os.makedirs(OUT, exist_ok=True)
    exe = os.path.join(OUT, "serving_driver")
    flags = [f for f in hip_build.HIPCC_FLAGS if f not in ("-shared", "-O3")]
    cmd = [hipcc, *flags, "-O1", "-g", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"), "-I", hip_build.CSRC,
           *[os.path.join(hip_build.CSRC, s) for s in SOURCES], "-x", "hip", os.path.join(SAN, "serving_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l)
    assert r.returncode == 0, out[-4000:]
    assert "serving host sanitizer run ok" in _run(exe)


def test_lds_limits_of_the_serving_kernels_on_every_device(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    exe = str(tmp_path / "lds_limit_serving_driver")
    subprocess.run(["gcc", "-std=gnu11", "-O1", "-rdynamic", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "tests"),
                    os.path.join(ROOT, "tests", "lds_limit_serving_driver.c"), "-o", exe, "-ldl"], check=True)
    r = subprocess.run([exe, mq.LIB_PATH], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert r.returncode == 0, r.stdout


def test_grids_and_scratch_for_any_host_bounds(tmp_path):
    """Bounds from 0 to the largest number: no empty or oversized grid, and one beyond the table is the table's."""
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    exe = str(tmp_path / "serving_grid_driver")
    subprocess.run(["gcc", "-std=gnu11", "-O1", "-rdynamic", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "tests"),
                    os.path.join(ROOT, "tests", "serving_grid_driver.c"), "-o", exe, "-ldl"], check=True)
    r = subprocess.run([exe, mq.LIB_PATH], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert r.returncode == 0, r.stdout
