"""Rotary positions, cache writes, drafted steps and moves of accepted drafts together, as a serving program runs them: two rounds of
speculative decoding against the definition in 64 bits over the tokens that were kept."""
import math

import pytest
import torch

from oracle import fp8_oracle as F
from tests.draft_harness import SCALE, check, random_tree
from tests.test_gpu_rope_cache import rotated64
from tests.test_rope_host import frequencies

pytestmark = pytest.mark.gpu
ROPE = dict(layout="interleaved", base=10000.0, scaling="yarn", factor=40.0, original_length=4096.0)
FREQS = frequencies(64, 10000.0, "yarn", 40.0, 4096.0, 32.0, 1.0)


def stored(latent, bits):
    """The values that the cache keeps of latent rows (float64)."""
    x = latent.double().numpy()
    if bits == 16:
        return torch.from_numpy(x)
    rows = []
    for r in x:
        s = F.pow2_scale(abs(r).max())
        rows.append(F.e4m3_decode_table()[F.e4m3_encode(r / s)] * s)
    return torch.stack([torch.as_tensor(r, dtype=torch.float64) for r in rows])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H", [16, 128])
def test_two_rounds_of_speculative_decoding(bits, H):
    from paper_2509_21081_b200 import binding as b
    from paper_2509_21081_b200.decoder import TyphoonMLADecoder
    g = torch.Generator().manual_seed(bits + H)
    B, S, page, max_pages, prompt, prefix = 5, 6, 64, 5, [70, 1, 128, 200, 63], 300

    def normal(*shape, mul=1.0):
        return (torch.randn(*shape, generator=g) * mul).to(torch.bfloat16)

    w_uk, w_uv = normal(H, 128, 512, mul=512 ** -0.5), normal(H, 128, 512, mul=512 ** -0.5)
    rope = b.typhoon_mla_rope_init(64, **ROPE)

    # the cache, the page tables, and what the definition keeps beside them: float64 latent rows and rotated keys per request
    n_pages = B * max_pages + 6
    latent_pages = torch.zeros(n_pages, page, 512, dtype=torch.uint8 if bits == 8 else torch.bfloat16, device="cuda")
    cache = b.PagedCache(latent_pages, torch.zeros(n_pages, page, 64, dtype=torch.bfloat16, device="cuda"),
                         torch.zeros(n_pages, page, dtype=torch.uint8, device="cuda") if bits == 8 else None)
    perm = torch.randperm(n_pages, generator=g)
    table = perm[:B * max_pages].view(B, max_pages).to(torch.int32)
    prefix_slots = torch.cat([perm[-6 + i] * page + torch.arange(page) for i in range(5)])[:prefix]
    kept = [(torch.zeros(0, 512, dtype=torch.float64), torch.zeros(0, 64, dtype=torch.float64)) for _ in range(B)]

    def slot_of(r, pos):
        return int(table[r, pos // page]) * page + pos % page

    def write(tokens, slots, positions):
        """tokens [T, 576] as a projection leaves them; returns what the definition has of them."""
        t = tokens.cuda()
        b.typhoon_mla_cache_append(cache, t[:, :512], t[:, 512:], torch.tensor(slots).cuda(), rope,
                                   torch.tensor(positions, dtype=torch.int32).cuda())
        keys = rotated64(tokens[:, None, 512:].double().numpy(), torch.tensor(positions).numpy(), 64, "interleaved", FREQS)[:, 0]
        return stored(tokens[:, :512], bits), torch.from_numpy(keys)

    # the prefix enters the cache, and is read back to become a shared prefix
    pre_c, pre_k = write(normal(prefix, 576), prefix_slots.tolist(), list(range(prefix)))
    ckv, kpe = b.typhoon_mla_cache_read(cache, prefix_slots.cuda())
    assert torch.equal(ckv.double().cpu(), pre_c)
    dec = TyphoonMLADecoder(H, ckv, kpe, w_uk.cuda(), w_uv.cuda(), SCALE, B, max_pages, page, max_drafts=S)
    # the prompts of the requests
    for r in range(B):
        kept[r] = write(normal(prompt[r], 576), [slot_of(r, i) for i in range(prompt[r])], [prefix + i for i in range(prompt[r])])
    length = list(prompt)

    for round_ in range(2):
        mask = random_tree(S, B, seed=round_)
        # drafts sit at the end of the suffixes; their position is their depth in the tree
        depth = [[bin(int(mask[r, j])).count("1") - 1 for j in range(S)] for r in range(B)]
        slots = [slot_of(r, length[r] + j) for r in range(B) for j in range(S)]
        positions = [prefix + length[r] + depth[r][j] for r in range(B) for j in range(S)]
        draft_c, draft_k = write(normal(B * S, 576), slots, positions)
        # queries of the drafts, from a projection of 192 per head
        q = normal(B * S, H, 192)
        q_nope, q_pe = torch.empty(B * S, H, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(B * S, H, 64, dtype=torch.bfloat16, device="cuda")
        qg = q.cuda()
        b.typhoon_mla_rope_queries(rope, qg[..., 128:], torch.tensor(positions, dtype=torch.int32).cuda(), q_pe, qg[..., :128], q_nope)
        lens = torch.tensor([n + S for n in length], dtype=torch.int32).cuda()
        out = dec.decode_draft(q_nope, q_pe, cache, table.cuda(), lens, tree_mask=mask.cuda())
        # one row at a time
        want = torch.zeros(B * S, H, 128, dtype=torch.float64)
        rot = torch.from_numpy(rotated64(q[..., 128:].double().numpy(), torch.tensor(positions).numpy(), 64, "interleaved", FREQS))
        for r in range(B):
            for j in range(S):
                row = r * S + j
                see = [i for i in range(S) if (int(mask[r, j]) >> i) & 1]
                c = torch.cat([pre_c, kept[r][0], draft_c[[r * S + i for i in see]]])
                k = torch.cat([pre_k, kept[r][1], draft_k[[r * S + i for i in see]]])
                q_lat = torch.einsum("hd,hdc->hc", q[row, :, :128].double(), w_uk.double())
                p = torch.softmax((q_lat @ c.T + rot[row] @ k.T) * SCALE, -1)
                want[row] = torch.einsum("hc,hdc->hd", p @ c, w_uv.double())
        # (keys and rope queries are rounded to 16 bits here, which the definition's are not: two more roundings of a third of the logit)
        check(out.double().cpu(), want, tensor_tol=6e-3)
        # a path of each tree is accepted: its drafts move to the front, in order, the rest is dropped
        source, target = [], []
        for r in range(B):
            tip = S - 1 - (r + round_) % 3
            path = [i for i in range(S) if (int(mask[r, tip]) >> i) & 1]
            for n, i in enumerate(path):
                source.append(slots[r * S + i])
                target.append(slot_of(r, length[r] + n))
            pick = [r * S + i for i in path]
            kept[r] = (torch.cat([kept[r][0], draft_c[pick]]), torch.cat([kept[r][1], draft_k[pick]]))
            length[r] += len(path)
        moved_c, moved_k = b.typhoon_mla_cache_read(cache, torch.tensor(source).cuda())
        b.typhoon_mla_cache_append(cache, moved_c, moved_k, torch.tensor(target).cuda())
    for r in range(B):
        at = torch.tensor([slot_of(r, i) for i in range(length[r])]).cuda()
        c, _ = b.typhoon_mla_cache_read(cache, at)
        assert torch.equal(c.double().cpu(), kept[r][0])
    assert b.typhoon_mla_check_status(dec.shared) == 0
    dec.close()
