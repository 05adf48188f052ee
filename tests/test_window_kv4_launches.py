"""What the attention through windows and over 4-bit caches launches (CPU only, see launches.py)."""
import re

import pytest

from launches import BF16, F32, DRIVER, record
from test_attn_window_kv4 import COMPACT, WINDOWS
from test_gpu_window_kv4_tiles import COMPACT_TILES, WINDOW_TILES

CALLS = DRIVER[:DRIVER.index("res = []")] + r"""
class Tensor4(ctypes.Structure):
    _fields_ = [("codes", Tensor), ("scales", Tensor)]
tail = [i32, i32, f32, Tensor, vp, vp, sz, vp]
lib.kvcomm_suffix_attn_window.argtypes = [vp, Tensor, Tensor, Tensor, i32, i32, i32, i32, f32, Tensor, vp, vp, sz, vp]
lib.kvcomm_suffix_attn_kv4.argtypes = [vp, Tensor, Tensor4, Tensor4, i32, i32, f32, Tensor, vp, vp, sz, vp]
lib.kvcomm_suffix_attn_window_workspace.argtypes = [vp, i32, i32, i32, i32]
lib.kvcomm_suffix_attn_window_workspace.restype = sz
lib.kvcomm_suffix_attn_kv4_workspace.argtypes = [vp, i32, i32]
lib.kvcomm_suffix_attn_kv4_workspace.restype = sz
res = []
for L, hkv, G, D, dtype, n_ctx, tq, window, sinks, scratch in json.load(sys.stdin):
    m = Model(L, hkv, hkv * G, D, dtype, 1e4)
    t = lambda h, n, d: Tensor(0x1000, h * n * d, n * d, d)
    N = n_ctx + tq
    if window:
        need = lib.kvcomm_suffix_attn_window_workspace(ctypes.byref(m), n_ctx, tq, window, sinks)
        cache, more = t(hkv, N, D), (window, sinks)
    else:
        need = lib.kvcomm_suffix_attn_kv4_workspace(ctypes.byref(m), n_ctx, tq)
        cache, more = Tensor4(t(hkv, N, D // 2), t(hkv, N, D // 32)), ()
    ws = (0x1000, need) if scratch and need else (None, 0)
    shim.rec_clear()
    q = t(hkv * G, tq, D)
    call = lib.kvcomm_suffix_attn_window if window else lib.kvcomm_suffix_attn_kv4
    st = call(ctypes.byref(m), q, cache, cache, n_ctx, tq, *more, 0.0, q, None, *ws, None)
    res.append(dict(status=st, workspace=need,
                    launches=[(shim.rec_name(i).decode(), [shim.rec_grid(i, k) for k in range(3)], shim.rec_block(i, 0)) for i in range(shim.rec_count())]))
json.dump(res, sys.stdout)
"""


def launches(tmp_path, calls):
    """calls: (L, Hkv, G, D, dtype code, n_ctx, tq, window (0: 4-bit cache), sinks, with scratch)."""
    return record(tmp_path, CALLS, calls)


def _kind(name):
    """(kernel, template arguments) of a mangled name."""
    kernel = re.search(r"attn_\w+?_kernel(16)?(?=I)", name)[0]
    return kernel, re.findall(r"L(?:[ib]|N\w+?E)(\d+)E", name[name.index(kernel) + len(kernel):])


def _of(cases, compact):
    dt = lambda t: F32 if "float32" in str(t) else BF16
    for c in cases:
        L, hkv, G, D = c[:4]
        if compact:
            yield L, hkv, G, D, dt(c[6]) if len(c) > 6 else BF16, c[4], c[5], 0, 0
        else:
            yield L, hkv, G, D, dt(c[4]), c[5], c[6], c[7], c[8]


def test_the_shapes_of_the_gpu_tests_reach_every_kernel(tmp_path):
    seen = set()
    tiles = lambda cases, compact: [c[:4] + (BF16,) + (c[4:] if not compact else c[4:] + (0, 0)) for c in cases]
    for compact, cases in ((False, list(_of(WINDOWS, False)) + tiles(WINDOW_TILES, False)), (True, list(_of(COMPACT, True)) + tiles(COMPACT_TILES, True))):
        calls = [c + (ws,) for c in cases for ws in (True, False)]
        for c, r in zip(calls, launches(tmp_path, calls)):
            assert r["status"] == 0, c
            kernel, args = _kind(r["launches"][0][0])
            cut = len(r["launches"]) > 1
            assert cut == (r["workspace"] > 0 and c[-1])
            if "rows" in kernel and args[1] == "1":
                seen.add((compact, kernel, "non-temporal"))
            seen.add((compact, kernel, int(args[0]), r["launches"][0][2], cut))
    want = {(False, "attn_rows_kernel16", D, 256 if D == 256 else 512, cut) for D in (64, 128, 256) for cut in (False, True)}
    want |= {(False, "attn_rows_kernel", D, 512, False) for D in (64, 128)} | {(False, "attn_rows_kernel", 256, 256, False)}
    want |= {(False, "attn_mfma_kernel", 128, t, cut) for t in (256, 512) for cut in (False, True)}
    want |= {(False, "attn_mfma_kernel", D, 256, cut) for D in (64, 256) for cut in (False, True)}
    want |= {(c, "attn_f32_kernel", D, 512, False) for c in (False, True) for D in (64, 128, 256)}
    want |= {(True, "attn_kv4_rows_kernel", D, 512, cut) for D in (64, 128, 256) for cut in (False, True)}
    want |= {(True, "attn_mfma_kernel", D, t, cut) for D in (64, 128, 256) for t in ((256,) if D == 256 else (256, 512)) for cut in (False, True)}
    want |= {(False, "attn_rows_kernel16", "non-temporal"), (True, "attn_kv4_rows_kernel", "non-temporal")}
    assert want <= seen, sorted(want - seen)
