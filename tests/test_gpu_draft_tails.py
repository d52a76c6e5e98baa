"""One dominant token beside a long tail of small weights: what the tail adds up to has to reach the result, over either cache.

Every weight of the second product is rounded by itself; a rounding with a fixed smallest step takes the same away from each of N tokens,
N half steps in all, to one side (two E4M3 terms with 2^4 at the reference: half of 2^-9 over 2^4, 2^-14 of the largest for each token).  So the
tail is kept only if a weight's error is small next to the weight itself: 2^-8 of it over a 16-bit cache (bf16), less than that over an
8-bit one (three terms of 3 bits) down to 2^-19 of the row's largest contribution.  The tails here have weights of 2^-7 to 2^-18 of the dominant
one.  So the roundings are those that the ordinary tolerances count, and the tolerances are the ordinary ones."""
import math

import pytest
import torch

from tests.draft_harness import SCALE, Problem, check

pytestmark = pytest.mark.gpu


def tailed(H, S, tokens, bits, share, spread, at, seed):
    """Two requests whose rows put `share` of their weight on the token at place `at`.  Latent rows have a common part as large as their
    spread, so that what is lost of the tail does not average out.  spread 0: a flat tail, the dominant token's logit comes from the
    rope keys alone; else the tail's logits have that standard deviation."""
    p = Problem(H, S, 0, [tokens] * 2, bits=bits, seed=seed)
    g = torch.Generator().manual_seed(seed + 1)
    common = torch.randn(512, generator=g)
    for b in range(p.B):
        x = common + torch.randn(tokens, 512, generator=g)
        if bits == 8:
            e = torch.ceil(torch.log2(x.abs().amax(-1) / 440.0))
            p.ckv_pages.view(-1, 512)[p.slot[b]] = (x * torch.exp2(-e)[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
            p.exponents.view(-1)[p.slot[b]] = (e + 127).to(torch.uint8)
        else:
            p.ckv_pages.view(-1, 512)[p.slot[b]] = x.to(torch.bfloat16)
        # the rope keys: zero but for the dominant token's
        p.kpe_pages.view(-1, 64)[p.slot[b]] = 0
        p.kpe_pages.view(-1, 64)[p.slot[b][at], 0] = 16.0
    # the spread of q_lat . c over tokens is |q_lat| for standard normal rows
    size = torch.linalg.norm(torch.einsum("rhd,hdc->rhc", p.q_nope.double(), p.w_uk.double()), dim=-1, keepdim=True)
    p.q_nope = (p.q_nope.double() * (spread / SCALE / size)).to(torch.bfloat16)
    q_lat = torch.einsum("rhd,hdc->rhc", p.q_nope.double(), p.w_uk.double())
    p.q_pe = torch.zeros_like(p.q_pe)
    for b in range(p.B):
        c, _ = p.latent(b)
        rest = torch.ones(tokens, dtype=torch.bool)
        rest[at] = False
        for j in range(S):
            logits = q_lat[b * S + j] @ c.T * SCALE
            want = torch.logsumexp(logits[:, rest], -1) + math.log(share / (1 - share))
            p.q_pe[b * S + j, :, 0] = ((want - logits[:, at]) / (SCALE * 16.0)).to(torch.bfloat16)
    return p


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("tokens,at", [(4096, 0), (4096, 3000), (16384, 0), (16384, 16000)])
@pytest.mark.parametrize("share", [0.45, 0.8, 0.9])
@pytest.mark.parametrize("S,spread", [(1, 0.0), (1, 1.0), (6, 0.0), (6, 0.6)])
def test_dominant_token_before_a_long_tail(bits, tokens, at, share, S, spread):
    p = tailed(16, S, tokens, bits, share, spread, at, seed=40 + S)
    want, want_lse = p.reference()
    # a request per pair of SMs: the plan leaves such suffixes in one piece
    copies = torch.cuda.get_device_properties(0).multi_processor_count // 4
    q = Problem(16, S, 0, [1] * 2, bits=bits, seed=0)
    q.w_uk, q.w_uv = p.w_uk, p.w_uv
    q.B, q.lens, q.max_pages = 2 * copies, p.lens * copies, p.max_pages
    q.table = p.table.repeat(copies, 1)
    q.q_nope, q.q_pe = p.q_nope.repeat(copies, 1, 1), p.q_pe.repeat(copies, 1, 1)
    q.ckv_pages, q.kpe_pages, q.exponents = p.ckv_pages, p.kpe_pages, p.exponents
    dec = q.decoder()
    mask = torch.ones(q.B, 1, dtype=torch.int64) if S == 1 else None     # (with a mask: the kernel of drafted tokens for S = 1 as well)
    got, lse, status = q.step(dec, mask=mask)
    assert status == 0
    assert torch.equal(got.view(copies, 2 * S, 16, 128), got[:2 * S].expand(copies, -1, -1, -1))
    check(got[:2 * S], want, lse[:2 * S], want_lse)


@pytest.mark.parametrize("bits", [8, 16])
def test_dominant_token_before_a_quarter_of_a_million(bits):
    """The longest tail here: 2^18 tokens in one piece, each worth 2^-18 of the dominant one."""
    p = tailed(16, 1, 1 << 18, bits, 0.5, 0.0, 0, seed=47)
    p.B, p.lens, p.table, p.slot = 1, p.lens[:1], p.table[:1], p.slot[:1]
    p.q_nope, p.q_pe = p.q_nope[:1], p.q_pe[:1]
    want, want_lse = p.reference()
    copies = torch.cuda.get_device_properties(0).multi_processor_count // 2
    dec = p.decoder(max_batch=copies)
    p.B, p.lens, p.table = copies, p.lens * copies, p.table.repeat(copies, 1)
    p.q_nope, p.q_pe = p.q_nope.repeat(copies, 1, 1), p.q_pe.repeat(copies, 1, 1)
    got, lse, status = p.step(dec, mask=torch.ones(copies, 1, dtype=torch.int64))
    assert status == 0 and torch.equal(got, got[:1].expand_as(got))
    check(got[:1], want, lse[:1], want_lse)
