"""Sizes beyond all arithmetic: every attention call and query answers with a status, on the host, before anything is launched."""
from launches import BF16, F32, attention_launches
from test_window_kv4_launches import launches

MOST = 2 ** 31 - 1
SHAPES = [(L, H, G, D, dt, n_ctx, tq) for L, H, G in ((MOST, MOST, 1), (2 ** 30, 2 ** 30, 1), (2 ** 20, 2 ** 16, 2), (1, 1, 2 ** 20), (MOST, 1, 1))
          for D, dt in ((64, BF16), (256, BF16), (128, F32)) for n_ctx, tq in ((0, 33), (5000, 64), (700, 2 ** 20), (2 ** 30, 2 ** 30 + 5), (0, MOST), (MOST, 1))]


def _refused(calls, results):
    for c, r in zip(calls, results):
        assert r["status"] in (-1, -2) and not r["launches"] and r["workspace"] == 0, (c, r)   # (-1: strides that have overflowed)


def test_attention_of_whole_caches(tmp_path):
    calls = [s + (blocks, ws) for s in SHAPES if (s[0], s[5:]) != (1, (5000, 64)) and (s[0], s[5:]) != (1, (0, 33)) for blocks in (0, 64) for ws in (True, False)]
    calls = [c for c in calls if c[0] * c[1] * c[2] * c[6] >= 2 ** 40 or c[2] * c[6] > MOST - 511 or c[5] + c[6] > MOST - 511]
    assert len(calls) > 150
    _refused(calls, attention_launches(tmp_path, calls))


def test_short_f32_caches_of_many_heads(tmp_path):
    """Their launch has a block for four (head, query) rows."""
    most = (2 ** 20, 4, 15, 64, F32, 0, 1, 0, False)   # 15.7 M blocks of 256 threads
    beyond = [(2 ** 20, 4, 16, 64, F32, 0, 1, 0, False), (2 ** 20, 2 ** 12, 8, 64, F32, 0, 1, 0, False), (2 ** 20, 8, 8, 128, F32, 0, 2, 64, False)]
    ok, *rest = attention_launches(tmp_path, [most] + beyond)
    assert ok["status"] == 0 and ok["launches"][0][1] == [15 * 2 ** 20, 1, 1]
    _refused(beyond, rest)


def test_windows_and_compact_caches(tmp_path):
    calls = [s + (w, 0, ws) for s in SHAPES for w in (0, 100) for ws in (True, False) if s[0] > 1 or s[6] > 2 ** 12]
    _refused(calls, launches(tmp_path, calls))
