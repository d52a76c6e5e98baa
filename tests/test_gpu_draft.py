"""Decode attention for drafted tokens (chains, trees, any mask) over 16- and 8-bit caches, against the definition in 64 bits."""
import random

import pytest
import torch

from tests.draft_harness import Problem, check, random_tree

pytestmark = pytest.mark.gpu
MODES = {"auto": 0, "absorb": 1, "hybrid": 2}


@pytest.fixture(scope="module")
def b():
    from paper_2509_21081_b200 import binding
    return binding


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H,S", [(128, 1), (16, 1), (64, 2), (16, 4), (48, 3), (128, 2), (128, 5), (32, 33), (16, 64)])
def test_chain_without_prefix(b, bits, H, S):
    """One tile, tile borders, several chunks; rows of more than one request tile."""
    p = Problem(H, S, 0, [S, S + 1, 64, 127 + S, 128, 700], bits=bits, seed=1)
    got, lse, status = p.step()
    assert status == 0
    check(got, p.reference()[0], lse, p.reference()[1])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("mode", ["auto", "absorb", "hybrid"])
@pytest.mark.parametrize("H,S,Ls,page", [(128, 1, 300, 64), (16, 4, 256, 64), (128, 3, 1111, 128), (64, 8, 640, 64), (32, 2, 77, 128)])
def test_tree_beside_a_prefix(b, bits, mode, H, S, Ls, page):
    p = Problem(H, S, Ls, [300, S, 65, 190, 1030], bits=bits, page=page, seed=2)
    mask = random_tree(S, p.B, seed=3)
    got, lse, status = p.step(mask=mask, mode=MODES[mode])
    assert status == 0
    want, want_lse = p.reference(mask)
    check(got, want, lse, want_lse)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("length", [0, 1, 2, 3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 130, 255, 256, 257])
def test_lengths(b, bits, length):
    """Every end of a tile, a token group and a page; suffixes shorter than the drafts they should hold, and empty ones."""
    p = Problem(16, 3, 0, [length, length + 1], bits=bits, seed=length)
    got, lse, status = p.step()
    assert status == 0
    want, want_lse = p.reference()
    check(got, want, lse, want_lse)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("S", [1, 7, 64])
@pytest.mark.parametrize("Ls", [0, 200])
def test_any_mask_and_ragged_counts(b, bits, S, Ls):
    """Masks that are no trees (empty rows, bits of later drafts, bits past the last draft), fewer drafts than S, none at all, counts
    outside 0 .. S, requests without a token."""
    p = Problem(32, S, Ls, [S + 5, 64 + S // 2, 130, 0, S, 1, 300], bits=bits, seed=5)
    g = torch.Generator().manual_seed(9)
    mask = torch.randint(-(1 << 62), 1 << 62, (p.B, S), generator=g) * 2 + torch.randint(0, 2, (p.B, S), generator=g)
    mask[0] = 0
    mask[4, S // 2] = 0
    mask[2, -1] = -1
    counts = [S, S // 2, 0, 3, S + 9, 1, -4]
    got, lse, status = p.step(mask=mask, draft_lens=counts)
    assert status == 0
    want, want_lse = p.reference(mask, counts)
    check(got, want, lse, want_lse)


@pytest.mark.parametrize("bits", [16, 8])
def test_rows_that_see_nothing(b, bits):
    """No prefix, no committed token, an empty mask: zeros and -inf, whatever the drafts hold."""
    p = Problem(128, 4, 0, [4, 4, 200], bits=bits, seed=6)
    mask = random_tree(4, 3)
    mask[0] = 0
    mask[1, 2] = 0
    for slot in p.slot[0].tolist():
        p.kpe_pages.view(-1, 64)[slot] = float("nan")
    got, lse, status = p.step(mask=mask)
    assert status == 0
    want, want_lse = p.reference(mask)
    assert not got[:4].any() and torch.isinf(lse[:4]).all() and not got[6].any()
    check(got, want, lse, want_lse)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("mode", ["absorb", "hybrid"])
@pytest.mark.parametrize("what", ["nan", "inf", "-inf"])
def test_hidden_values_stay_hidden(b, bits, mode, what):
    """Drafts that some rows do not see hold values that are not finite: those rows are as without them, the rows that see them are NaN."""
    H, S = 16, 6
    p = Problem(H, S, 150, [140, 131, 64 + S, 400], bits=bits, seed=7)
    mask = random_tree(S, p.B, seed=1)
    bad = [2, 5, 0, 3]
    mask &= ~torch.tensor([1 << i for i in bad])[:, None]
    for r, i in enumerate(bad):
        mask[r, i] |= 1 << i                                   # only the draft itself sees it
    clean, _ = p.reference(mask)
    v = float(what)
    for r, i in enumerate(bad):
        slot = int(p.slot[r][p.lens[r] - S + i])
        if bits == 8:
            p.ckv_pages.view(-1, 512)[slot] = 0x7F if r % 2 else 0          # as another program may leave them, or as they are written here
            p.exponents.view(-1)[slot] = 255
        else:
            p.ckv_pages.view(-1, 512)[slot, 40 * r:40 * r + 40] = v
        p.kpe_pages.view(-1, 64)[slot, 3] = v
    got, lse, status = p.step(mask=mask, mode=MODES[mode])
    assert status == 0
    sees = torch.zeros(p.B, S, dtype=torch.bool)
    for r, i in enumerate(bad):
        sees[r, i] = True
    sees = sees.view(-1)
    if what == "nan" or bits == 8:
        assert torch.isnan(got[sees.cuda()]).all() and torch.isnan(lse[sees.cuda()]).all()
    rest = ~sees.cuda()
    check(got[rest], clean[rest])


@pytest.mark.parametrize("spread", [0, 3, 12])
@pytest.mark.parametrize("peak", [1.0, 6.0])
def test_8_bit_tokens_of_different_sizes(b, spread, peak):
    """Powers of two that differ by up to 2^24 between tokens, flat and sharp softmaxes.  A weight is good to 2^-14 of the row's largest
    contribution, which adds to the bf16 roundings where many small contributions make up a row: at most 2^-14 / 2 per token of 512,
    2^-6 of the largest together if all fell to one side; evenly spread, as they are, sqrt(512) 2^-15 = 7e-4."""
    p = Problem(64, 2, 0, [512, 300, 129], bits=8, seed=8, spread=spread, peak=peak)
    got, lse, status = p.step()
    assert status == 0
    want, want_lse = p.reference()
    # sharp logits carry the absorbed query's rounding times their size: |logit| 2^-8 / sqrt(3) each
    size = max(1.0, float(want_lse.abs().max()) / 10)
    check(got, want, lse, want_lse, tensor_tol=5e-3 * size, row_tol=4 * 2.0 ** -8 * size)


def test_8_bit_rows_of_zeros_and_extreme_exponents(b):
    """Rows of zeros as they are written here (byte 1, 2^-126), alone and among others, also where one of them takes nearly all the
    weight; powers of two up to 2^100 apart; bytes 0.  The row sums have all of them, the output what is not negligible."""
    H, S = 16, 2
    p = Problem(H, S, 0, [40, 200, 131, 200, 140, 300], bits=8, seed=21)
    codes, ex, kpe = p.ckv_pages.view(-1, 512), p.exponents.view(-1), p.kpe_pages.view(-1, 64)
    codes[p.slot[0]], ex[p.slot[0]] = 0, 1                                 # nothing but zeros
    codes[p.slot[1][::3]], ex[p.slot[1][::3]] = 0, 1                       # zeros among others
    at = p.slot[2][100]
    codes[at], ex[at] = 0, 1
    kpe[at] = 40.0 * torch.sign(p.q_pe[2 * S, 0].float()).to(torch.bfloat16)     # a row of zeros that is worth 2^150 of the others for one row
    ex[p.slot[3][50:60]] = 200                                             # values of 2^70 and more: their logits decide
    ex[p.slot[4]] = torch.randint(20, 110, (140,), dtype=torch.uint8)      # down to 2^-107
    codes[p.slot[5][7]], ex[p.slot[5][7]] = 0, 0
    got, lse, status = p.step()
    assert status == 0 and torch.isfinite(got).all() and not got[:S].any()
    want, want_lse = p.reference()
    rows = [r for r in range(12) if r // S not in (2, 3)]
    check(got[rows], want[rows], lse[rows], want_lse[rows])
    # one row per head may be all weight on a row of zeros: nothing there but what is below 2^-90
    big = want[4:6].norm(dim=-1) > 1e-3
    off = (got[4:6] - want[4:6]).norm(dim=-1)
    assert (off[big] <= 4 * 2.0 ** -8 * want[4:6].norm(dim=-1)[big]).all() and (off[~big] <= 1e-5).all()
    assert (lse[4:6] - want_lse[4:6]).abs().max().item() <= 2e-2 * max(1.0, float(want_lse[4:6].abs().max()) / 10)


def test_8_and_16_bits_agree(b):
    """The same values in either cache: the two kernels differ by their roundings alone."""
    p = Problem(128, 2, 500, [640, 100, 333], bits=8, seed=9, poison=False)
    q = Problem(128, 2, 500, [640, 100, 333], bits=16, seed=9, poison=False)
    q.q_nope, q.q_pe, q.ckv, q.kpe, q.w_uk, q.w_uv = p.q_nope, p.q_pe, p.ckv, p.kpe, p.w_uk, p.w_uv
    q.table, q.slot, q.kpe_pages = p.table, p.slot, p.kpe_pages
    byte = p.exponents.float()
    q.ckv_pages = (p.ckv_pages.view(torch.float8_e4m3fn).float() * torch.exp2(byte - 127)[..., None]).to(torch.bfloat16)
    got8, lse8, _ = p.step()
    got16, lse16, _ = q.step()
    want, want_lse = p.reference()
    check(got8, want, lse8, want_lse)
    check(got16, want, lse16, want_lse)
    assert (torch.linalg.norm(got8 - got16) / torch.linalg.norm(want)).item() <= 5e-3


def test_single_tokens_are_the_decode_step(b):
    """S = 1 without a mask over a 16-bit cache is typhoon_mla_decode, to the bit; with the mask of a token that sees itself it is the
    same attention."""
    p = Problem(128, 1, 700, [300, 1, 129, 64], seed=10)
    dec = p.decoder()
    lens = torch.tensor(p.lens, dtype=torch.int32, device="cuda")
    cache = p.cache()
    want = dec.decode(p.q_nope.cuda(), p.q_pe.cuda(), cache.ckv_pages, cache.kpe_pages, p.table.cuda(), lens)
    got = dec.decode_draft(p.q_nope.cuda(), p.q_pe.cuda(), cache, p.table.cuda(), lens)
    assert torch.equal(got, want)
    masked, lse, _ = p.step(dec, mask=torch.ones(4, 1, dtype=torch.int64))
    check(masked, p.reference()[0], lse, p.reference()[1])


def test_chain_is_the_expanded_rows(b):
    """S = 3 without a mask gives what typhoon_mla_expand_query_rows and typhoon_mla_decode give."""
    p = Problem(128, 3, 400, [300, 3, 129, 64], seed=11)
    got, lse, _ = p.step()
    bt, sl = b.typhoon_mla_expand_query_rows(p.table.cuda(), torch.tensor(p.lens, dtype=torch.int32, device="cuda"), 3)
    dec = p.decoder(max_batch=12)
    cache = p.cache()
    want = dec.decode(p.q_nope.cuda(), p.q_pe.cuda(), cache.ckv_pages, cache.kpe_pages, bt, sl).double()
    ref, ref_lse = p.reference()
    check(got, ref, lse, ref_lse)
    assert (torch.linalg.norm(got - want) / torch.linalg.norm(ref)).item() <= 5e-3


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("mode", ["absorb", "hybrid"])
def test_8_bit_prefix_and_many_rows(b, bits, mode):
    """More than 128 query rows over the prefix; a prefix expanded in 8 bits (E4M3 rounds to 2^-4 of a value at most, evenly spread
    2^-4 / sqrt(3) = 3.6 % of keys and values, averaged over the tokens a row sees)."""
    p = Problem(16, 8, 900, [200 + 7 * i for i in range(20)], bits=bits, seed=12)
    mask = random_tree(8, p.B, seed=2)
    want, want_lse = p.reference(mask)
    got, lse, _ = p.step(mask=mask, mode=MODES[mode])
    check(got, want, lse, want_lse)
    got8, _, _ = p.step(p.decoder(fp8_shared=True), mask=mask, mode=MODES[mode])
    assert (torch.linalg.norm(got8 - want) / torch.linalg.norm(want)).item() <= 2.0 ** -4


@pytest.mark.parametrize("bits", [16, 8])
def test_many_requests_and_long_suffixes(b, bits):
    """More items than pairs of SMs, several chunks, launch order by length; bitwise the same on every run."""
    lens = [4 + (i * 389) % 3000 for i in range(90)]
    p = Problem(16, 4, 64, lens, bits=bits, seed=13)
    mask = random_tree(4, p.B, seed=4)
    dec = p.decoder()
    got, lse, status = p.step(dec, mask=mask)
    again, _, _ = p.step(dec, mask=mask)
    assert status == 0 and torch.equal(got, again)
    want, want_lse = p.reference(mask)
    check(got, want, lse, want_lse)


@pytest.mark.parametrize("bits", [16, 8])
def test_bad_pages(b, bits):
    """A page id outside the cache inside a request's length: reported, not dereferenced, the other requests as they are."""
    p = Problem(16, 2, 100, [150, 200, 70], bits=bits, seed=14)
    want, _ = p.reference()
    for bad in (-1, p.kpe_pages.shape[0], 1 << 30):
        table = p.table.clone()
        p.table[1, 1] = bad
        got, _, status = p.step()
        assert status == b.STATUS_BAD_PAGE
        check(torch.cat([got[:2], got[4:]]), torch.cat([want[:2], want[4:]]))
        p.table = table


@pytest.mark.parametrize("bits", [16, 8])
def test_clamped_lengths(b, bits):
    """Lengths past the table are the table's, negative ones zero."""
    p = Problem(32, 2, 64, [128, 128], bits=bits, seed=15)
    q = Problem(32, 2, 64, [128, 128], bits=bits, seed=15)
    q.lens = [1 << 30, -5]
    got, lse, _ = q.step()
    want, want_lse = p.reference()
    check(got[:2], want[:2], lse[:2], want_lse[:2])
    empty = Problem(32, 2, 64, [128, 0], bits=bits, seed=15)
    empty.q_nope, empty.q_pe, empty.ckv, empty.kpe, empty.w_uk, empty.w_uv = p.q_nope, p.q_pe, p.ckv, p.kpe, p.w_uk, p.w_uv
    check(got[2:], empty.reference()[0][2:])


@pytest.mark.parametrize("bits", [16, 8])
def test_strided_cache(b, bits):
    """Latent rows and rope keys as slices of wider rows."""
    p = Problem(64, 2, 50, [300, 77], bits=bits, seed=16)
    if bits == 8:
        wide = torch.zeros(*p.ckv_pages.shape[:2], 528, dtype=torch.uint8)
        wide[..., :512] = p.ckv_pages
        keys = torch.zeros(*p.kpe_pages.shape[:2], 72, dtype=torch.bfloat16)
        keys[..., 8:] = p.kpe_pages
        cache = b.PagedCache(wide.cuda()[..., :512], keys.cuda()[..., 8:], p.exponents.cuda())
    else:
        wide = torch.cat([p.ckv_pages, p.kpe_pages], -1).cuda()
        cache = b.PagedCache(wide[..., :512], wide[..., 512:])
    p.cache = lambda: cache
    got, lse, _ = p.step()
    check(got, p.reference()[0], lse, p.reference()[1])


@pytest.mark.parametrize("bits", [16, 8])
def test_smaller_steps_in_one_workspace(b, bits):
    """A workspace for a batch, drafts and a table serves every smaller step, and nothing behind it is written."""
    big = Problem(32, 8, 300, [500] * 6, bits=bits, seed=17)
    dec = big.decoder()
    n = dec.workspace.numel()
    guard = torch.full((n + 4096,), 0x5C, dtype=torch.uint8, device="cuda")
    dec.workspace = guard[:n]
    for B, S, L, mode in ((6, 8, 500, 0), (5, 8, 64, 1), (1, 1, 500, 1), (1, 8, 500, 1), (3, 2, 130, 2), (6, 1, 500, 2), (2, 7, 448, 1)):
        p = Problem(32, S, 300, [L] * B, bits=bits, seed=18)
        p.ckv, p.kpe, p.w_uk, p.w_uv = big.ckv, big.kpe, big.w_uk, big.w_uv
        got, lse, status = p.step(dec, mode=mode)
        want, want_lse = p.reference()
        assert status == 0
        check(got, want, lse, want_lse)
        assert (guard[n:] == 0x5C).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_streams_and_graphs(b, bits):
    """Another stream; a captured step replayed with other contents, beside eager steps that use a workspace of their own."""
    p = Problem(16, 4, 200, [300, 100, 50], bits=bits, seed=19)
    mask = random_tree(4, 3, seed=5)
    want, _ = p.reference(mask)
    dec, other = p.decoder(), p.decoder()
    cache, table, lens, gm = p.cache(), p.table.cuda(), torch.tensor(p.lens, dtype=torch.int32, device="cuda"), mask.cuda()
    qn, qp = p.q_nope.cuda(), p.q_pe.cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = dec.decode_draft(qn, qp, cache, table, lens, tree_mask=gm)
    torch.cuda.current_stream().wait_stream(s)
    check(out.double(), want)
    graph = torch.cuda.CUDAGraph()
    held = torch.empty_like(out)
    with torch.cuda.graph(graph, stream=s):
        dec.decode_draft(qn, qp, cache, table, lens, tree_mask=gm, out=held)
    eager = other.decode_draft(qn, qp, cache, table, lens, tree_mask=gm)
    graph.replay()
    assert torch.equal(held, out) and torch.equal(eager, out)
    gm.fill_(15)
    qn.neg_()
    graph.replay()
    p.q_nope = -p.q_nope
    check(held.double(), p.reference(torch.full((3, 4), 15))[0])


def test_refusals(b):
    p = Problem(16, 2, 64, [100, 70])
    dec = p.decoder()
    cache, table, lens = p.cache(), p.table.cuda(), torch.tensor(p.lens, dtype=torch.int32, device="cuda")
    qn, qp = p.q_nope.cuda(), p.q_pe.cuda()
    out = torch.empty_like(qn)

    def call(**kw):
        a = dict(q_nope=qn, q_pe=qp, cache=cache, block_table=table, seq_lens=lens, softmax_scale=0.1, out=out, workspace=dec.workspace)
        a.update(kw)
        b.typhoon_mla_decode_draft(dec.shared, **a)

    call()
    for kw in (dict(mode=3), dict(mode=4), dict(mode=-1), dict(softmax_scale=0.0), dict(softmax_scale=float("nan")),
               dict(workspace=dec.workspace[:4096]), dict(workspace=dec.workspace[1:]), dict(block_table=table[:, :0].contiguous())):
        with pytest.raises(b.TyphoonMLAError):
            call(**kw)
    for kw in (dict(q_nope=qn[:3]), dict(q_pe=qp[:2]), dict(q_nope=qn.float()), dict(block_table=table.long()), dict(seq_lens=lens[:1]),
               dict(tree_mask=torch.zeros(2, 3, dtype=torch.int64, device="cuda")), dict(tree_mask=torch.zeros(2, 2, dtype=torch.int32, device="cuda")),
               dict(draft_lens=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(out=out[:2]), dict(q_nope=qn.cpu()),
               dict(lse_out=torch.empty(4, 15, device="cuda"))):
        with pytest.raises(ValueError):
            call(**kw)
    b.typhoon_mla_set_kernel_path(b.PATH_WARP_MMA)
    try:
        with pytest.raises(b.TyphoonMLAError, match="unsupported"):
            call()
    finally:
        b.typhoon_mla_set_kernel_path(b.PATH_TCGEN05)
    with pytest.raises(ValueError):
        dec.decode_draft(torch.cat([qn, qn]), torch.cat([qp, qp]), cache, table, lens)      # four drafts per request: sized for two
    q65 = torch.zeros(65, 16, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(b.TyphoonMLAError):
        call(q_nope=q65, q_pe=torch.zeros(65, 16, 64, dtype=torch.bfloat16, device="cuda"), block_table=table[:1], seq_lens=lens[:1],
             out=torch.empty_like(q65))
    assert b.typhoon_mla_draft_workspace_bytes(dec.shared, 2, 65, 2, 64) == 0
    assert b.typhoon_mla_draft_workspace_bytes(dec.shared, 2, 2, 0, 64) == 0
    assert b.typhoon_mla_draft_workspace_bytes(dec.shared, 2, 2, (1 << 23) + 1, 64) == 0 < b.typhoon_mla_draft_workspace_bytes(dec.shared, 2, 2, 1 << 23, 128)
    assert b.typhoon_mla_draft_workspace_bytes(dec.shared, 2, 2, 2, 32) == 0
    assert b.typhoon_mla_draft_workspace_bytes(dec.shared, 2, 2, 2, 64, 3) == 0


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("mode", ["absorb", "hybrid"])
@pytest.mark.parametrize("H,S,masked", [(16, 1, False), (16, 1, True), (16, 3, False), (128, 3, True), (128, 16, False)])
@pytest.mark.parametrize("where", ["query", "query rope", "committed", "prefix"])
def test_nan_reaches_the_rows_that_see_it_and_no_others(b, bits, mode, H, S, masked, where):
    p = Problem(H, S, 150, [140, 131, 64 + S, 400, 0, S], bits=bits, seed=22)
    mask = torch.zeros(p.B, S, dtype=torch.int64) if masked else None       # (no row sees a draft)
    clean, _ = p.reference(mask)
    hit = torch.zeros(p.B * S, H, dtype=torch.bool)
    if where.startswith("query"):
        q = p.q_nope if where == "query" else p.q_pe
        q[S, 3, 5] = float("nan")
        q[2 * S, 15, 0] = float("inf")
        hit[S, 3] = hit[2 * S, 15] = True
    elif where == "committed":
        slot = int(p.slot[1][20])
        if bits == 8:
            p.ckv_pages.view(-1, 512)[slot], p.exponents.view(-1)[slot] = 0, 255
        else:
            p.ckv_pages.view(-1, 512)[slot, 100] = float("nan")
        hit[S:2 * S] = True
    else:
        p.ckv[77, 9] = float("nan")
        hit[:] = True
    got, lse, status = p.step(mask=mask, mode=MODES[mode])
    assert status == 0
    hit = hit.cuda()
    assert torch.isnan(got[hit]).all() and torch.isnan(lse[hit]).all()
    check(got[~hit][None], clean[~hit][None])


@pytest.mark.parametrize("bits", [16, 8])
def test_more_requests_than_are_ordered(b, bits):
    """More than 4096 requests: no launch order, no descriptors."""
    p = Problem(16, 2, 100, [2 + (i * 37) % 70 for i in range(4100)], bits=bits, seed=23)
    got, lse, status = p.step()
    assert status == 0
    rows = [0, 1, 2, 3, 200, 201, 4098, 4099, 8190, 8191, 8198, 8199]
    part = [r // 2 for r in rows[::2]]
    q = Problem(16, 2, 100, [p.lens[r] for r in part], bits=bits, seed=23)
    q.q_nope, q.q_pe, q.ckv, q.kpe, q.w_uk, q.w_uv = p.q_nope[rows], p.q_pe[rows], p.ckv, p.kpe, p.w_uk, p.w_uv
    q.slot, q.ckv_pages, q.kpe_pages, q.exponents = [p.slot[r] for r in part], p.ckv_pages, p.kpe_pages, p.exponents
    want, want_lse = q.reference()
    check(got[rows], want, lse[rows], want_lse)


@pytest.mark.parametrize("seed", range(32))
def test_drawn_steps(b, seed):
    """Sizes, masks, counts, modes and library settings at random; half of the steps are captured and replayed."""
    g = random.Random(seed)
    H, S, B = g.choice([16, 32, 48, 64, 80, 112, 128]), g.choice([1, 1, 2, 3, 5, 8, 13, 33, 64]), g.randint(1, 9)
    if H * S > 2048:
        H = 16
    Ls = g.choice([0, 1, 63, 129, 500, 1500])
    lens = [max(0, g.choice([S, S + 1, g.randint(0, 130), g.randint(100, 900)])) for _ in range(B)]
    bits = g.choice([8, 16])
    p = Problem(H, S, Ls, lens, bits=bits, page=g.choice([64, 128]), seed=100 + seed)
    kind = g.choice(["chain", "tree", "any"])
    mask = None if kind == "chain" else random_tree(S, B, seed) if kind == "tree" else \
        torch.tensor([[g.getrandbits(64) - (1 << 63) for _ in range(S)] for _ in range(B)], dtype=torch.int64)
    counts = None if g.random() < 0.5 else [g.randint(-1, S + 1) for _ in range(B)]
    mode = g.choice([0, 1, 2])
    want, want_lse = p.reference(mask, counts)
    b.typhoon_mla_set_overlap(g.random() < 0.7)
    b.typhoon_mla_set_programmatic_launch(g.random() < 0.7)
    b.typhoon_mla_set_stacked_absorb(g.random() < 0.7)
    b.typhoon_mla_set_naive_schedule(g.choice([0, 1, 2]))
    try:
        dec = p.decoder()
        got, lse, status = p.step(dec, mask, counts, mode)
        assert status == 0
        check(got, want, lse, want_lse)
        if seed % 2:
            a = [x.cuda() for x in (p.q_nope, p.q_pe, p.table, torch.tensor(p.lens, dtype=torch.int32))]
            kw = dict(tree_mask=None if mask is None else mask.cuda(),
                      draft_lens=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"), mode=mode)
            cache, out = p.cache(), torch.empty_like(a[0])
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                dec.decode_draft(a[0], a[1], cache, a[2], a[3], out=out, **kw)
            for _ in range(3):
                out.zero_()
                graph.replay()
                assert torch.equal(out.double(), got)
    finally:
        b.typhoon_mla_set_overlap(True)
        b.typhoon_mla_set_programmatic_launch(True)
        b.typhoon_mla_set_stacked_absorb(True)
        b.typhoon_mla_set_naive_schedule(0)


def test_steps_at_once(b):
    """Four decoders on four streams, both caches and both modes, many steps in flight: each gives what it gives alone."""
    runs = []
    for i, (bits, mode) in enumerate([(16, 1), (8, 1), (16, 2), (8, 2)]):
        p = Problem(32, 5, 700, [5 + 97 * k % 600 for k in range(20)], bits=bits, seed=30 + i)
        a = [x.cuda() for x in (p.q_nope, p.q_pe)] + [p.cache(), p.table.cuda(), torch.tensor(p.lens, dtype=torch.int32, device="cuda")]
        dec, s = p.decoder(), torch.cuda.Stream()
        runs.append((dec, a, mode, s, dec.decode_draft(*a, mode=mode)))
    torch.cuda.synchronize()
    got = [[] for _ in runs]
    for _ in range(25):
        for k, (dec, a, mode, s, _) in enumerate(runs):
            with torch.cuda.stream(s):
                got[k].append(dec.decode_draft(*a, mode=mode))
    torch.cuda.synchronize()
    for k, (dec, _, _, _, want) in enumerate(runs):
        assert all(torch.equal(x, want) for x in got[k])
        assert b.typhoon_mla_check_status(dec.shared, raise_on_error=False) == 0


@pytest.mark.parametrize("bits", [16, 8])
def test_offsets_past_32_bits(b, bits):
    """A cache of more than 2^32 bytes whose last pages are used: written, read back and attended there."""
    p = Problem(16, 3, 100, [200, 3, 130], bits=bits, seed=24, poison=False)
    n = p.kpe_pages.shape[0]
    pages = (2 ** 32) // (64 * (1024 if bits == 16 else 512)) + 1000
    first = pages - n
    big = b.PagedCache(torch.zeros(pages, 64, 512, dtype=torch.bfloat16 if bits == 16 else torch.uint8, device="cuda"),
                       torch.zeros(pages, 64, 64, dtype=torch.bfloat16, device="cuda"),
                       None if bits == 16 else torch.zeros(pages, 64, dtype=torch.uint8, device="cuda"))
    small = p.cache()
    slots = torch.cat(p.slot).cuda()
    ckv, kpe = b.typhoon_mla_cache_read(small, slots)
    b.typhoon_mla_cache_append(big, ckv, kpe, slots + first * 64)
    again, keys = b.typhoon_mla_cache_read(big, slots + first * 64)
    assert torch.equal(again, ckv) and torch.equal(keys, kpe)
    assert not big.kpe_pages[:first].any()
    want, want_lse = p.reference()
    p.cache, p.table = lambda: big, torch.where(p.table >= 0, p.table + first, p.table)
    for mode in (1, 2):
        got, lse, status = p.step(mode=mode)
        assert status == 0
        check(got, want, lse, want_lse)
