"""Tiles of the dense 8-bit product, as the library chooses them on the host: sizes from one token to many, and devices whose SMs
have no room for clusters of four or eight thread blocks.  The calls run in a process of their own: a division by zero ends it."""
import json
import subprocess
import sys

import pytest

from paper_2609_07008_b200.build import LIB_PATH

CALL = """
import ctypes, json, sys
lib = ctypes.CDLL(sys.argv[1])
i64, i32 = ctypes.c_int64, ctypes.c_int32
lib.rk_matmul8_plan.restype = None
lib.rk_matmul8_plan.argtypes = [i64, i64, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32)]
out = []
for n_out, n_tok, k_pad, sms, slots in json.loads(sys.argv[2]):
    rows, split = i32(-1), i32(-1)
    lib.rk_matmul8_plan(n_out, n_tok, k_pad, sms, (i32 * 2)(*slots), ctypes.byref(rows), ctypes.byref(split))
    out.append([rows.value, split.value])
print(json.dumps(out))
"""

SIZES = [(4096, 5, 8192), (1001, 333, 784), (7168, 8192, 16384), (1, 1, 16), (4096, 256, 8192), (256, 2, 131072), (100000, 1, 4096),
         (129, 1000000, 64), (2**31 - 2048, 1, 16), (1, 2**31 - 2048, 16)]


def plans(cases):
    r = subprocess.run([sys.executable, "-c", CALL, LIB_PATH, json.dumps(cases)], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])
    return json.loads(r.stdout)


@pytest.mark.parametrize("slots", [[37, 18], [0, 0], [37, 0], [0, 18], [1, 1]])
@pytest.mark.parametrize("sms", [148, 132, 2])
def test_every_size_has_tiles(slots, sms):
    for (n_out, n_tok, k_pad), (rows, split) in zip(SIZES, plans([(*size, sms, slots) for size in SIZES])):
        assert rows in (32, 64, 128, 256) and split in (1, 2, 4)
        tiles = -(-n_out // 256) * -(-n_tok // rows)
        if split > 1:                                   # all clusters run at once, and every pair has four steps of k or more
            assert tiles <= slots[split // 4] and -(-k_pad // 128) >= 4 * split
        assert tiles < 2**31


def test_k_is_shared_where_there_is_room():
    size = (4096, 5, 8192)
    assert [p[1] for p in plans([(*size, 148, s) for s in ([37, 18], [37, 0], [0, 0])])] == [4, 2, 1]
