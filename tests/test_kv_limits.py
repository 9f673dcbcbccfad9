"""Limits of the paged cache's calls.  Steps as large as they may be: kv.hip built for the host into tests/sanitize/kv_limits.cpp."""
import os
import subprocess

import pytest

from paper_2312_17238_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_largest_steps_stay_within_their_lists(tmp_path):
    exe = str(tmp_path / "kv_limits")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc, "--offload-host-only", "-fuse-cuid=none", "-O1", "-std=c++17", "-pthread", "-o", exe, "-x", "hip",
                    os.path.join(ROOT, "tests", "sanitize", "kv_limits.cpp")], check=True, cwd=tmp_path, stdout=subprocess.PIPE, stderr=subprocess.PIPE)
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout == "ok\n", run.stdout + run.stderr


@pytest.mark.parametrize("room", [0, -1, -2 ** 31])
def test_a_stack_without_room_is_refused(room):
    step, at = B.KvStep(2, 8, 4, 16, 32, 16, 2, 64, 8, 1, 0, 0), 0x10000
    lists = B.KvLists(*(at + 64 * i for i in range(len(B.KvLists._fields_))))
    with pytest.raises(B.MoeError, match="moe_kv_plan") as e:
        B.moe_kv_plan_within(step, lists, room, at, 0)
    assert e.value.code == B.MOE_EINVAL


def test_giving_back_nothing_is_no_error():
    """An empty list has no address."""
    at = 0x10000
    B.moe_kv_release(0, 0, 4, 32, 16, 8, at, at, at, 32, at, 0)
    for i in (0, 6, 7, 8, 10):
        args = [at, 1, 4, 32, 16, 8, at, at, at, 32, at, 0]
        args[i] += 2
        with pytest.raises(B.MoeError, match="moe_kv_release"):
            B.moe_kv_release(*args)
