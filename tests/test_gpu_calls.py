"""Calls around a step at the ends of what they take, through the bindings."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_no_tokens():
    from paper_2509_21081_b200 import binding as b
    bf = torch.bfloat16
    cache = b.PagedCache(torch.zeros(2, 64, 512, dtype=bf, device="cuda"), torch.zeros(2, 64, 64, dtype=bf, device="cuda"))
    rope = b.typhoon_mla_rope_init()
    kv = torch.zeros(0, 576, dtype=bf, device="cuda")
    slots, pos = torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    b.typhoon_mla_cache_append(cache, kv[:, :512], kv[:, 512:], slots, rope, pos)
    b.typhoon_mla_cache_append(cache, kv[:, :512], kv[:, 512:], slots)
    q = torch.zeros(0, 16, 192, dtype=bf, device="cuda")
    b.typhoon_mla_rope_queries(rope, q[..., 128:], pos, torch.empty(0, 16, 64, dtype=bf, device="cuda"), q[..., :128],
                               torch.empty(0, 16, 128, dtype=bf, device="cuda"))
    assert not cache.ckv_pages.any() and not cache.kpe_pages.any()
