"""A step over a compact cache that fails leaves the cache as it was, so that it can be made again."""
import pytest
import torch

import paper_2510_12872_amd as kv
from paper_2510_12872_amd import hotpath

M = kv.Model(1, 2, 4, 64, torch.bfloat16, 1e4)


def test_a_failed_attention_gives_its_tokens_back(monkeypatch):
    """(CPU: the calls are stand-ins, the last one fails.)"""
    fails = [kv.KVCommError(kv.binding.EINVAL, "out"), torch.OutOfMemoryError("no room"), KeyboardInterrupt()]
    done = []

    def attend(*args, **kw):
        if fails:
            raise fails.pop()
        return "out"
    monkeypatch.setattr(hotpath.kv, "kvcomm_place_qkv", lambda m, q, k, v, first, **kw: (q, k, v))
    monkeypatch.setattr(hotpath.kv, "kvcomm_quantize_kv4", lambda m, k, v, out_k, out_v, **kw: done.append(out_k[0].storage_offset()))
    monkeypatch.setattr(hotpath.kv, "kvcomm_suffix_attn_kv4", attend)
    cache = hotpath.CompactCache(M, 20, "cpu")
    cache.length = 7
    x = lambda h: torch.zeros((1, h, 5, 64), dtype=torch.bfloat16)
    while fails:
        with pytest.raises(type(fails[-1])):
            hotpath.suffix_step(M, x(4), x(2), x(2), cache, 7)
        assert cache.length == 7
    assert hotpath.suffix_step(M, x(4), x(2), x(2), cache, 7) == "out" and cache.length == 12
    assert done == [7 * 32] * 4   # each time at the same rows


@pytest.mark.gpu
def test_a_step_made_again():
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = lambda h, n: torch.randn((1, h, n, 64), generator=g, device="cuda").bfloat16()
    first, parts = [x(2, 9), x(2, 9)], (x(4, 5), x(2, 5), x(2, 5))
    outs = []
    for bad in (False, True):
        cache = hotpath.CompactCache(M, 20, "cuda")
        cache.append(*first)
        if bad:
            for out in (torch.empty((1, 4, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((1, 4, 5, 64), device="cuda")):
                with pytest.raises(kv.KVCommError):
                    hotpath.suffix_step(M, *parts, cache, 9, out=out)
                assert cache.length == 9
        outs.append(hotpath.suffix_step(M, *parts, cache, 9))
        assert cache.length == 14
    assert torch.equal(*outs)
