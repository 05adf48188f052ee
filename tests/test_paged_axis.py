"""Calls on batches whose keys, over all row tiles and heads, are more than the wavefronts of a launch count: refused before anything is launched."""
import ctypes

import paper_2510_12872_amd as kv
from paper_2510_12872_amd import binding


def test_runs_longer_than_the_kernels_walk():
    """36 row tiles of up to 2^25 halves for each of L * Hkv (layer, kv head) pairs: 1.2e9 fit 31 bits, a wavefront's share of all of them goes up to 2^31."""
    lib = kv.load_library()
    T, P = (lambda p: binding._CTensor(p, 1 << 20, 1 << 12, 128)), (lambda p: binding._CPages(p, 1 << 30, 1 << 28, 1 << 24, 128))
    batch = binding._CBatch(0x1000, 0x2000, 0x3000, 16384, 16384, 35, 16, 65536, 1, 1)   # 2^30 tokens a sequence, 16 rows of 35 sequences
    for dtype, D, waves in ((1, 64, 4096), (1, 128, 2048), (1, 256, 1024), (0, 64, 2048), (0, 128, 2048), (0, 256, 1024)):
        tiles = 16 // 16 + 35
        for pairs in (waves, waves * 3 // 2):   # the share of a wavefront: 1.2e9, 1.8e9
            m = binding._CModel(2, pairs // 2, pairs // 2, D, dtype, 1e4)
            share = tiles * (2 ** 25 + 1) * pairs / waves
            assert 1e9 < share < 2147483000 and tiles * (2 ** 25 + 1) < 2 ** 31 - 1 and 16 * pairs < 67000000
            st = lib.kvcomm_paged_attn(ctypes.byref(m), T(0x10000), P(0x100000000), P(0x200000000), ctypes.byref(batch), 0.0, T(0x300000000), None, None, 0, None)
            assert st == -2, (dtype, D, pairs, st)
