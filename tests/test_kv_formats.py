"""The 8-bit half of the tensor layer where torch has no 4-bit type: in a process of its own, without a GPU."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import torch
del torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
from paper_2312_17238_amd import decode_loop, paged
assert set(paged.FORMATS) == {torch.float8_e4m3fn, torch.int8} and set(decode_loop.FORMATS) == {"e4m3", "int8"}

def refused(message, f, *a):
    try:
        f(*a)
    except ValueError as e:
        assert message in str(e), e
    else:
        raise AssertionError(message)

for t in (torch.float8_e4m3fn, torch.int8):        # as far as a cache comes without a GPU
    refused("contiguous tensors on one GPU", paged.Cache.empty, 4, 2, 64, 32, t, "cpu")
refused("codes of type", paged.Cache.empty, 4, 2, 64, 32, torch.uint8, "cpu")
refused("codes of type", paged.Cache.empty, 4, 2, 64, 32, None, "cpu")
print("fine")
"""


def test_eight_bits_without_a_four_bit_type():
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]
