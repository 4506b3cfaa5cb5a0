"""KVCache keeps what it was made of (no GPU: what describes its tensors is not made)."""
import pytest
import torch


def test_a_cache_does_not_change_under_its_descriptor(monkeypatch):
    from paper_2407_16990_amd import KVCache, binding
    monkeypatch.setitem(binding._seq.__dict__, "kv_desc", lambda *a: b"made once")
    k, v, s = torch.zeros(3, 4, 2, 32), torch.ones(3, 4, 2, 32), torch.zeros(3, 2, 4)
    cache = KVCache(k, v, s, s)
    assert cache.k is k and cache.v is v and cache.k_scale is s and cache.v_scale is s
    assert (cache.n_pages, cache.page, cache.heads, cache.dim) == (3, 4, 2, 32)
    for name in ("k", "v", "k_scale", "v_scale", "n_pages", "page", "heads", "dim"):
        with pytest.raises(AttributeError):
            setattr(cache, name, torch.zeros(3, 4, 2, 32))
    assert cache.k is k and cache.desc == b"made once"
