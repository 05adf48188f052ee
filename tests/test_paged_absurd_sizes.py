"""Calls on batches with absurd sizes: a status, no trap and no exception, and nothing launched."""
import ctypes
import itertools

import paper_2510_12872_amd as kv
from paper_2510_12872_amd import binding

BIG = 2 ** 31 - 1


def test_a_status_for_every_size():
    lib = kv.load_library()
    T, P = (lambda p: binding._CTensor(p, 2 ** 62, 2 ** 61, 2 ** 40)), (lambda p: binding._CPages(p, 2 ** 62, 2 ** 61, 2 ** 60, 2 ** 40))
    refused = 0
    for L, H, G, dtype, n_seqs, n_rows, width, n_pages, page, n_prefix in itertools.product(
            (1, BIG), (1, BIG), (1, 2), (0, 1), (1, 8192), (1, BIG), (0, 2 ** 10, BIG), (0, BIG), (16, 65536), (1, BIG)):
        Hq = min(BIG // H * H, H * G)
        m = binding._CModel(L, H, Hq, 128, dtype, 1e4)
        starts = 0x3000 if n_rows != n_seqs else None
        b = binding._CBatch(0x1000, 0x2000, starts, 2 ** 60, width, n_seqs, n_rows, page, n_pages, BIG)
        lib.kvcomm_paged_attn_workspace(ctypes.byref(m), ctypes.byref(b))
        lib.kvcomm_paged_attn_prefix_workspace(ctypes.byref(m), n_prefix, ctypes.byref(b))
        if L * Hq * n_rows < 67000000 and not (width * page > 2 ** 30 or width * page + n_prefix > 2 ** 30):
            continue   # (a call that might be launched)
        for st in (lib.kvcomm_paged_attn_prefix(ctypes.byref(m), T(0x10000), T(0x20000), T(0x30000), n_prefix, P(0x40000), P(0x50000), ctypes.byref(b), 0.0, T(0x60000), None, None,
                                                0, None),):
            assert st in (-1, -2), (L, H, G, n_seqs, n_rows, width, n_pages, page, n_prefix, st)
            refused += 1
        if L * (Hq + 2 * H) * n_rows * 128 >= 2 ** 35 or width * page > 2 ** 30:
            assert lib.kvcomm_place_qkv_paged(ctypes.byref(m), T(0x10000), T(0x20000), T(0x30000), ctypes.byref(b), 0, None, None, 0, 0, 0.0, T(0x60000), P(0x40000),
                                              P(0x50000), None) in (-1, -2)
    assert refused > 100


def test_workspaces_of_what_is_refused():
    lib = kv.load_library()
    b = binding._CBatch(0x1000, 0x2000, None, 8, 8, 3, 3, 16, 4, 0)
    good = binding._CModel(1, 1, 1, 128, 1, 1e4)
    assert lib.kvcomm_paged_attn_workspace(ctypes.byref(good), ctypes.byref(b)) > 0
    assert lib.kvcomm_paged_attn_prefix_workspace(ctypes.byref(good), 0, ctypes.byref(b)) == 0
    assert lib.kvcomm_paged_attn_workspace(None, ctypes.byref(b)) == 0 and lib.kvcomm_paged_attn_workspace(ctypes.byref(good), None) == 0
    for bad in (binding._CModel(1, 1, 1, 96, 1, 1e4), binding._CModel(0, 1, 1, 128, 1, 1e4), binding._CModel(BIG, 1, 1, 128, 1, 1e4)):
        assert lib.kvcomm_paged_attn_workspace(ctypes.byref(bad), ctypes.byref(b)) == 0
