"""The lists of a step never outgrow what the host makes room for: kv.hip built for the host into tests/sanitize/kv_harness.cpp."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_lists_hold_what_random_steps_put_into_them(tmp_path):
    exe = str(tmp_path / "kv_harness")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc, "--offload-host-only", "-fuse-cuid=none", "-O1", "-std=c++17", "-pthread", "-o", exe, "-x", "hip",
                    os.path.join(ROOT, "tests", "sanitize", "kv_harness.cpp")], check=True, cwd=tmp_path, stdout=subprocess.PIPE, stderr=subprocess.PIPE)
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout.startswith("ok: 4000 steps"), run.stdout + run.stderr
