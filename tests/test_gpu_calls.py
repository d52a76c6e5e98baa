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


@pytest.mark.parametrize("sizes", [dict(max_drafts=65), dict(max_drafts=-1), dict(max_batch=1 << 15, max_drafts=33), dict(max_pages=0, max_drafts=2),
                                   dict(max_pages=(1 << 23) + 1, max_drafts=2)])
def test_decoder_of_steps_that_are_refused(sizes):
    """Refused where it is built, not at the first step that does not fit."""
    from paper_2509_21081_b200.decoder import TyphoonMLADecoder
    bf = torch.bfloat16
    a = dict(max_batch=2, max_pages=4, max_drafts=2)
    a.update(sizes)
    prefix = torch.zeros(64, 512, dtype=bf, device="cuda"), torch.zeros(64, 64, dtype=bf, device="cuda")
    w = torch.zeros(16, 128, 512, dtype=bf, device="cuda")
    with pytest.raises(ValueError, match="drafts"):
        TyphoonMLADecoder(16, *prefix, w, w, 0.1, **a)
    TyphoonMLADecoder(16, *prefix, w, w, 0.1, 2, 4, max_drafts=64).close()
    TyphoonMLADecoder(16, *prefix, w, w, 0.1, 2, 0).close()


def test_misaligned_arrays_are_refused():
    """Arrays of 32-bit words at odd addresses: an error, no launch."""
    from paper_2509_21081_b200 import binding as b
    from paper_2509_21081_b200.decoder import TyphoonMLADecoder
    bf = torch.bfloat16
    w = torch.zeros(16, 128, 512, dtype=bf, device="cuda")
    dec = TyphoonMLADecoder(16, torch.zeros(64, 512, dtype=bf, device="cuda"), torch.zeros(64, 64, dtype=bf, device="cuda"), w, w, 0.1, 2, 1,
                            max_drafts=2)
    cache = b.PagedCache(torch.zeros(2, 64, 512, dtype=bf, device="cuda"), torch.zeros(2, 64, 64, dtype=bf, device="cuda"))
    q, qp, out = (torch.zeros(4, 16, n, dtype=bf, device="cuda") for n in (128, 64, 128))
    words = torch.zeros(64, dtype=torch.int32, device="cuda")
    at, c, ws = words.data_ptr(), cache.struct, dec.workspace
    stream = torch.cuda.current_stream().cuda_stream

    def draft(table=at, lens=at, counts=at, lse=None):
        return b._lib.typhoon_mla_decode_draft(dec.shared.handle, q.data_ptr(), qp.data_ptr(), 2, 2, c, table, 1, lens, counts, None, 0.1, 0,
                                               out.data_ptr(), lse, ws.data_ptr(), ws.numel(), stream)

    def decode(table=at, lens=at, lse=None):
        return b._lib.typhoon_mla_decode(dec.shared.handle, q.data_ptr(), qp.data_ptr(), 2, c.ckv_pages, c.kpe_pages, 512, 64, 64, 2, table, 1, lens,
                                         0.1, 0, out.data_ptr(), lse, ws.data_ptr(), ws.numel(), stream)

    assert draft() == 0 and decode() == 0
    for odd in (1, 2, 3):
        for kw in (dict(table=at + odd), dict(lens=at + odd), dict(counts=at + odd), dict(lse=at + odd)):
            assert draft(**kw) == 1
            assert "counts" in kw or decode(**kw) == 1
    assert b._lib.typhoon_mla_combine_partials(at, at + 2, 1, 1, 1, at, None, stream) == 1
    assert b._lib.typhoon_mla_combine_partials(at, at, 1, 1, 1, at, at + 1, stream) == 1
    torch.cuda.synchronize()
    dec.close()
