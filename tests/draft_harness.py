"""Steps of drafted tokens: problems, pages in either format, and the definition in 64 bits (one softmax per row over what it sees)."""
import math

import torch

SCALE = (128 + 64) ** -0.5


class Problem:
    """Random queries, weights, prefix and suffixes; `lens` per request.  With bits = 8 the latent rows are exactly representable:
    codes under a power of two per token."""

    def __init__(self, H, S, Ls, lens, bits=16, page=64, seed=0, spread=0, poison=True, peak=1.0):
        g = torch.Generator().manual_seed(seed * 1009 + 7 * H + S)
        B = len(lens)
        self.H, self.S, self.Ls, self.B, self.lens, self.bits, self.page = H, S, Ls, B, list(lens), bits, page

        def normal(*shape, mul=1.0):
            return (torch.randn(*shape, generator=g) * mul).to(torch.bfloat16)

        self.ckv, self.kpe = normal(Ls, 512), normal(Ls, 64)
        self.w_uk, self.w_uv = normal(H, 128, 512, mul=512 ** -0.5), normal(H, 128, 512, mul=512 ** -0.5)
        self.q_nope, self.q_pe = normal(B * S, H, 128, mul=peak), normal(B * S, H, 64, mul=peak)
        need = [(n + page - 1) // page for n in lens]
        self.max_pages = max(max(need), 1)
        n_pages = sum(need) + 2
        perm = torch.randperm(n_pages, generator=g).tolist()
        self.table = torch.full((B, self.max_pages), -1, dtype=torch.int32)
        # every slot nobody owns holds NaN
        nan = float("nan") if poison else 0.0
        self.kpe_pages = torch.full((n_pages, page, 64), nan, dtype=torch.bfloat16)
        self.exponents = None
        if bits == 8:
            self.ckv_pages = torch.full((n_pages, page, 512), 0x7F if poison else 0, dtype=torch.uint8)
            self.exponents = torch.full((n_pages, page), 255 if poison else 127, dtype=torch.uint8)
        else:
            self.ckv_pages = torch.full((n_pages, page, 512), nan, dtype=torch.bfloat16)
        self.slot = []                      # per request: physical slot of every suffix token
        for b, n in enumerate(lens):
            ids = [perm.pop() for _ in range(need[b])]
            self.table[b, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
            at = torch.tensor([ids[t // page] * page + t % page for t in range(n)], dtype=torch.long)
            self.slot.append(at)
            if not n:
                continue
            x = torch.randn(n, 512, generator=g)
            if spread:
                x = x * torch.exp2(torch.randint(-spread, spread + 1, (n, 1), generator=g).float())
            if bits == 8:
                e = torch.ceil(torch.log2(x.abs().amax(-1) / 440.0))
                codes = (x * torch.exp2(-e)[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
                self.ckv_pages.view(-1, 512)[at] = codes
                self.exponents.view(-1)[at] = (e + 127).to(torch.uint8)
            else:
                self.ckv_pages.view(-1, 512)[at] = x.to(torch.bfloat16)
            self.kpe_pages.view(-1, 64)[at] = normal(n, 64)

    def latent(self, b):
        """float64 latent rows and rope keys of request b's suffix."""
        at = self.slot[b]
        c = self.ckv_pages.view(-1, 512)[at]
        if self.bits == 8:
            byte = self.exponents.view(-1)[at].double()
            c = c.view(torch.float8_e4m3fn).double() * torch.where(byte == 255, torch.full_like(byte, math.nan), torch.exp2(byte - 127))[:, None]
        return c.double(), self.kpe_pages.view(-1, 64)[at].double()

    def visible(self, b, mask=None, draft_lens=None, max_tokens=None):
        """bool [S, L]"""
        S = self.S
        L = self.lens[b] if max_tokens is None else min(self.lens[b], max_tokens)
        n = S if draft_lens is None else min(max(int(draft_lens[b]), 0), S)
        see = torch.zeros(S, L, dtype=torch.bool)
        for j in range(S):
            m = (1 << (j + 1)) - 1 if mask is None else int(mask[b, j]) & (2 ** 64 - 1)
            for p in range(L):
                see[j, p] = p < L - n or bool((m >> (p - (L - n))) & 1)
        return see

    def reference(self, mask=None, draft_lens=None):
        """float64 (out [B * S, H, 128], lse [B * S, H]) on the GPU."""
        S, H, B = self.S, self.H, self.B
        qn, qp, w_uk, w_uv, ckv, kpe = (x.cuda().double() for x in (self.q_nope, self.q_pe, self.w_uk, self.w_uv, self.ckv, self.kpe))
        q_lat = torch.einsum("rhd,hdc->rhc", qn, w_uk)
        out, lse = torch.zeros(B * S, H, 128, dtype=torch.float64, device="cuda"), torch.empty(B * S, H, dtype=torch.float64, device="cuda")
        for b in range(B):
            c, k = (x.cuda() for x in self.latent(b))
            see = self.visible(b, mask, draft_lens)
            for j in range(S):
                r = b * S + j
                own_c, own_k = c[see[j]], k[see[j]]
                keys_c, keys_k = torch.cat([ckv, own_c]), torch.cat([kpe, own_k])
                if not len(keys_c):
                    lse[r] = -math.inf
                    continue
                logits = (q_lat[r] @ keys_c.T + qp[r] @ keys_k.T) * SCALE
                lse[r] = torch.logsumexp(logits, -1)
                out[r] = torch.einsum("hc,hdc->hd", torch.softmax(logits, -1) @ keys_c, w_uv)
        return out, lse

    def decoder(self, fp8_shared=False, max_batch=None, max_drafts=None, max_pages=None):
        from paper_2509_21081_b200.decoder import TyphoonMLADecoder
        return TyphoonMLADecoder(self.H, self.ckv.cuda(), self.kpe.cuda(), self.w_uk.cuda(), self.w_uv.cuda(), SCALE,
                                 max_batch or self.B, max_pages or self.max_pages, self.page, fp8_shared=fp8_shared,
                                 max_drafts=max_drafts or self.S)

    def cache(self):
        from paper_2509_21081_b200 import binding as b
        return b.PagedCache(self.ckv_pages.cuda(), self.kpe_pages.cuda(), None if self.exponents is None else self.exponents.cuda())

    def step(self, dec=None, mask=None, draft_lens=None, mode=0, want_lse=True):
        """(out float64, lse float64, status word) on the GPU; the status is that of the prefix's handle."""
        from paper_2509_21081_b200 import binding as b
        dec = dec or self.decoder()
        lse = torch.full((self.B * self.S, self.H), 77.0, device="cuda") if want_lse else None
        out = dec.decode_draft(self.q_nope.cuda(), self.q_pe.cuda(), self.cache(), self.table.cuda(),
                               torch.tensor(self.lens, dtype=torch.int32, device="cuda"),
                               tree_mask=None if mask is None else mask.cuda(),
                               draft_lens=None if draft_lens is None else torch.as_tensor(draft_lens, dtype=torch.int32).cuda(), mode=mode,
                               lse_out=lse)
        status = b.typhoon_mla_check_status(dec.shared, raise_on_error=False)
        return out.double(), None if lse is None else lse.double(), status


def random_tree(S, B, seed=0):
    """int64 [B, S]: draft j hangs under an earlier draft or the last committed token, and sees its ancestors and itself."""
    g = torch.Generator().manual_seed(seed)
    mask = torch.zeros(B, S, dtype=torch.int64)
    for b in range(B):
        rows = []
        for j in range(S):
            parent = int(torch.randint(-1, j, (1,), generator=g)) if j else -1
            rows.append((rows[parent] if parent >= 0 else 0) | (1 << j))
        mask[b] = torch.tensor([r - (1 << 64) if r >= 1 << 63 else r for r in rows], dtype=torch.int64)
    return mask


# Four roundings to bf16 stand between the inputs and the result (absorbed query, probabilities, latent output, result), each off by at
# most half a step, 2^-8, and evenly spread below that: 2^-8 / sqrt(3) = 2.3e-3 in the 2-norm.  Independent: 4.5e-3 over a tensor.  A single
# row of 128 values depends on few independent errors where a few tokens or a sharp softmax make it: their sum, four times 2^-8.
TENSOR_TOL, ROW_TOL, LSE_TOL = 5e-3, 4 * 2.0 ** -8, 2e-2


def check(got, want, got_lse=None, want_lse=None, tensor_tol=TENSOR_TOL, row_tol=ROW_TOL, lse_tol=LSE_TOL):
    assert torch.isfinite(got).all()
    norm = torch.linalg.norm(want)
    if norm > 0:
        assert (torch.linalg.norm(got - want) / norm).item() <= tensor_tol, (torch.linalg.norm(got - want) / norm).item()
    rows, ref = got.reshape(-1, 128), want.reshape(-1, 128)
    rn = torch.linalg.norm(ref, dim=1)
    off = torch.linalg.norm(rows - ref, dim=1)
    assert (off[rn == 0] == 0).all()
    assert (off[rn > 0] <= row_tol * rn[rn > 0]).all(), (off[rn > 0] / rn[rn > 0]).max().item()
    if got_lse is not None:
        inf = torch.isinf(want_lse)
        assert torch.equal(torch.isinf(got_lse), inf)
        if (~inf).any():
            # logits carry the absorbed query's rounding, 2^-8 of values of a few units
            assert (got_lse[~inf] - want_lse[~inf]).abs().max().item() <= lse_tol * max(1.0, want_lse[~inf].abs().max().item() / 10)
