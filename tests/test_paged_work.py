"""How a paged call is dealt out (csrc/burst_paged.h, integer logic that the kernels run as it stands), on the host: every unit of work once,
no page or table entry out of range whatever the arrays on the device hold, parts joined once."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_units_pages_and_parts(tmp_path):
    exe = str(tmp_path / "driver")
    cmd = [os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-g", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-I", os.path.join(ROOT, "paper_2403_09347_amd", "csrc"), os.path.join(ROOT, "tests", "paged_work_driver.cpp"), "-o", exe]
    subprocess.run(cmd, check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0")
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "work checks failed: 0" in r.stdout, r.stdout[-3000:]
