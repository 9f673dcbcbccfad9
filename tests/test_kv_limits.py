"""Steps as large as they may be: kv.hip built for the host into tests/sanitize/kv_limits.cpp."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_largest_steps_stay_within_their_lists(tmp_path):
    exe = str(tmp_path / "kv_limits")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc, "--offload-host-only", "-fuse-cuid=none", "-O1", "-std=c++17", "-pthread", "-o", exe, "-x", "hip",
                    os.path.join(ROOT, "tests", "sanitize", "kv_limits.cpp")], check=True, cwd=tmp_path, stdout=subprocess.PIPE, stderr=subprocess.PIPE)
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout == "ok\n", run.stdout + run.stderr
