"""The comparison of tensors' bytes at sizes where blocks can no longer be listed: a status, in no time, and no C++ exception out of a C entry."""
import subprocess
import sys

CODE = r"""
import ctypes
from paper_2510_12872_amd import binding
lib = binding.load_library()
T = lambda ptr, sl, sh: binding._CTensor(ptr, sl, sh, 128)
none, far = T(None, 0, 0), lambda bit: T(1 << bit, 1 << 20, 1 << 10)
c4 = lambda ptr: binding._CTensor4(binding._CTensor(ptr, 1 << 19, 1 << 9, 64), binding._CTensor(ptr + (1 << 60), 1 << 15, 1 << 5, 4))
for L, H in ((2 ** 31 - 1, 2 ** 31 - 1), (10 ** 6, 10 ** 6), (2 * 10 ** 9, 1), (1, 2 * 10 ** 9), (60000, 60000)):
    m = ctypes.byref(binding._CModel(L, H, H, 128, 1, 1e4))
    for step in (1, 2):   # strides that are the same, and others
        x, y = T(0x10000, 1 << 20, 1 << 10), T(0x20000, step << 20, step << 10)
        print(lib.kvcomm_place_qkv(m, x, none, none, 4, 0, None, None, 0, 0, 0.0, y, none, none, None),
              lib.kvcomm_quantize_kv4(m, x, far(58), 4, c4(0x18000), c4(1 << 59), None),
              lib.kvcomm_align_kv(m, 0, x, far(58), 4, None, None, none, None, 0, None, 3, None, y, far(59), None), flush=True)
"""


def test_a_status_in_no_time():
    ran = subprocess.run([sys.executable, "-c", CODE], capture_output=True, text=True, timeout=100)
    assert ran.returncode == 0, (ran.stdout, ran.stderr[-500:])
    got = ran.stdout.split()
    assert len(got) == 30 and all(int(st) in (-1, -2) for st in got), ran.stdout   # refused: shared bytes, or more than a launch holds
