"""Rotary positions, cache writes and reads on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as F
from tests.test_rope_host import frequencies

pytestmark = pytest.mark.gpu
EPS = torch.finfo(torch.bfloat16).eps / 2      # half a step of the result


@pytest.fixture(scope="module")
def b():
    from paper_2509_21081_b200 import binding
    return binding


def rotated64(x, positions, d, layout, freqs, scale=1.0):
    """x float64 [T, H, 64] -> the definition, pair by pair."""
    y = x.copy()
    ang = positions.astype(np.float64)[:, None] * np.array(freqs)[None]          # off by 2^-52 of the angle: 1e-9 at 2^22 radians
    c, s = scale * np.cos(ang)[:, None], scale * np.sin(ang)[:, None]
    a = slice(0, d, 2) if layout == "interleaved" else slice(0, d // 2)
    e = slice(1, d, 2) if layout == "interleaved" else slice(d // 2, d)
    y[..., a], y[..., e] = x[..., a] * c - x[..., e] * s, x[..., a] * s + x[..., e] * c
    return y


def close(got, want, x, scale=1.0):
    """Half a step of bf16, and in 32 bits: the angle (its top 32 bits rounded to 24 and times pi: 2^-23 pi = 3.8e-7), the fast sine and
    cosine (2^-21.2 = 4.2e-7 within +-pi), two products and a sum (3 * 2^-24 = 1.8e-7): 1e-6 of each element of the pair."""
    got, mag = got.double().cpu().numpy(), np.abs(x).max() * 2 * abs(scale)
    tol = EPS * np.abs(want) + 1e-6 * mag
    assert (np.abs(got - want) <= tol * (1 + 1e-6)).all(), np.abs(got - want).max()


POSITIONS = [0, 1, -1, 5, 4095, 32768, 1 << 20, (1 << 31) - 1, -(1 << 31), 12345679]


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("d", [16, 32, 48, 64])
@pytest.mark.parametrize("T,H", [(1, 1), (1, 128), (10, 3), (37, 16), (700, 1), (301, 33), (650, 128)])
def test_rope_queries(b, layout, d, T, H):
    g = torch.Generator().manual_seed(d + T)
    q = torch.randn(T, H, 192, generator=g).to(torch.bfloat16).cuda()
    pos = torch.tensor((POSITIONS * (T // 10 + 1))[:T], dtype=torch.int32) if T <= 40 else torch.randint(0, 1 << 21, (T,), generator=g, dtype=torch.int32)
    rope = b.typhoon_mla_rope_init(d, layout, 10000.0, "yarn", 40.0, 4096.0, 32.0, 1.0, 1.25)
    nope, pe = torch.full((T + 1, H, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T + 1, H, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    b.typhoon_mla_rope_queries(rope, q[..., 128:], pos.cuda(), pe[:T], q[..., :128], nope[:T])
    assert b.typhoon_mla_last_launch_count() == 1
    x = q[..., 128:].double().cpu().numpy()
    want = rotated64(x, pos.numpy(), d, layout, frequencies(d, 10000.0, "yarn", 40.0, 4096.0, 32.0, 1.0), 1.25)
    close(pe[:T, :, :d], want[..., :d], x, 1.25)
    assert torch.equal(pe[:T, :, d:], q[..., 128 + d:]) and torch.equal(nope[:T], q[..., :128])
    assert (pe[T] == 7).all() and (nope[T] == 7).all()            # nothing behind the last row


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_rope_in_place_and_keys(b, layout):
    """Contiguous rows rotated in place; keys are rows with one head, here a slice of a projection; head-major inputs."""
    g = torch.Generator().manual_seed(3)
    rope = b.typhoon_mla_rope_init(64, layout)
    pos = torch.randint(0, 100000, (517,), generator=g, dtype=torch.int32).cuda()
    q = torch.randn(517, 24, 64, generator=g).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)
    b.typhoon_mla_rope_queries(rope, q, pos, out)
    headmajor = q.transpose(0, 1).contiguous().transpose(0, 1)
    out2 = torch.empty_like(q)
    b.typhoon_mla_rope_queries(rope, headmajor, pos, out2)
    assert torch.equal(out, out2)
    kv = torch.randn(517, 576, generator=g).to(torch.bfloat16).cuda()
    kv[:, 512:] = q[:, 5]
    k = torch.empty(517, 1, 64, dtype=torch.bfloat16, device="cuda")
    b.typhoon_mla_rope_queries(rope, kv[:, None, 512:], pos, k)
    assert torch.equal(k[:, 0], out[:, 5])
    b.typhoon_mla_rope_queries(rope, q, pos, q)
    assert torch.equal(q, out)


def test_rope_special_values(b):
    """A value that is not finite stays within its pair."""
    q = torch.ones(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    q[1, 1, 6], q[2, 0, 63] = float("nan"), float("inf")
    out = torch.empty_like(q)
    b.typhoon_mla_rope_queries(b.typhoon_mla_rope_init(64, "interleaved"), q, torch.arange(4, dtype=torch.int32, device="cuda"), out)
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[1, 1, 6:8] = want[2, 0, 62:64] = True
    assert torch.equal(bad, want)


def _pages(pages, page, bits, wide=False):
    """Pages full of a pattern; with `wide` the rows are slices of longer ones."""
    dt = torch.uint8 if bits == 8 else torch.bfloat16
    if bits == 8:
        base = torch.full((pages, page, 528 if wide else 512), 0x5A, dtype=dt, device="cuda")
        kpe = torch.full((pages, page, 72 if wide else 64), 3.0, dtype=torch.bfloat16, device="cuda")
        return base[..., :512], kpe[..., :64], torch.full((pages, page), 77, dtype=torch.uint8, device="cuda")
    base = torch.full((pages, page, 576), 3.0, dtype=dt, device="cuda")
    if wide:
        return base[..., :512], base[..., 512:], None
    return base[..., :512].contiguous(), base[..., 512:].contiguous(), None


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("page,wide", [(64, False), (128, True)])
@pytest.mark.parametrize("T", [1, 2, 7, 64, 331])
def test_append_and_read(b, bits, page, wide, T):
    g = torch.Generator().manual_seed(T + bits)
    pages = T // page + 3
    ckv, kpe, ex = _pages(pages, page, bits, wide)
    cache = b.PagedCache(ckv, kpe, ex)
    kv = torch.randn(T, 576, generator=g) * torch.exp2(torch.randint(-20, 20, (T, 1), generator=g).float())
    kv = kv.to(torch.bfloat16)
    slots = torch.randperm(pages * page, generator=g)[:T]
    skipped = torch.zeros(T, dtype=torch.bool)
    if T > 2:
        skipped[::5] = True
    slots[skipped] = -1 - slots[skipped]
    pos = torch.randint(0, 200000, (T,), generator=g, dtype=torch.int32)
    rope = b.typhoon_mla_rope_init(64, "half" if wide else "interleaved")
    before = [t.clone() for t in (ckv, kpe) + ((ex,) if bits == 8 else ())]
    kvg, status = kv.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    b.typhoon_mla_cache_append(cache, kvg[:, :512], kvg[:, 512:], slots.cuda(), rope, pos.cuda(), status)
    live = ~skipped
    at = slots[live]
    x = kv[live, 512:].double().numpy()[:, None]
    want_k = rotated64(x, pos[live].numpy(), 64, "half" if wide else "interleaved", frequencies(64, 10000.0, "none", 1, 1, 1, 1))[:, 0]
    flat = lambda t: t.reshape(-1, *t.shape[2:]).cpu()
    got_k = flat(kpe)[at].double().numpy()
    tol = EPS * np.abs(want_k) + 2e-6 * np.abs(x[:, 0]).max(-1, keepdims=True)
    assert (np.abs(got_k - want_k) <= tol).all()
    latent = kv[live, :512].double().numpy()
    if bits == 16:
        assert torch.equal(flat(ckv)[at], kv[live, :512])
    else:
        scale = np.array([F.pow2_scale(r) for r in np.abs(latent).max(-1)])
        assert np.array_equal(flat(ex)[at].numpy().astype(int), np.log2(scale).astype(int) + 127)
        assert np.array_equal(flat(ckv)[at].numpy(), F.e4m3_encode(latent / scale[:, None]))
    # everything else is as it was
    rest = torch.ones(pages * page, dtype=torch.bool)
    rest[at] = False
    for t, o in zip((ckv, kpe) + ((ex,) if bits == 8 else ()), before):
        assert torch.equal(flat(t)[rest], flat(o)[rest])
    assert status.item() == 0

    c, k = b.typhoon_mla_cache_read(cache, slots.cuda(), status=status)
    assert torch.equal(k.cpu()[live], flat(kpe)[at]) and not k.cpu()[skipped].any() and not c.cpu()[skipped].any()
    values = latent if bits == 16 else F.e4m3_decode_table()[flat(ckv)[at].numpy()] * scale[:, None]
    assert np.array_equal(c.cpu()[live].double().numpy(), values) and status.item() == 0
    # what was read back is written without change: codes may double with a smaller exponent, values stay
    ckv2, kpe2, ex2 = _pages(pages, page, bits)
    cache2 = b.PagedCache(ckv2, kpe2, ex2)
    b.typhoon_mla_cache_append(cache2, c, k, slots.cuda())
    c2, k2 = b.typhoon_mla_cache_read(cache2, slots.cuda())
    assert torch.equal(c2, c) and torch.equal(k2, k)


def test_read_repeats_and_strides(b):
    ckv, kpe, _ = _pages(4, 64, 16)
    ckv.normal_(), kpe.normal_()
    cache = b.PagedCache(ckv, kpe)
    slots = torch.tensor([5, 5, -3, 255, 0, 5], device="cuda")
    rows = torch.full((6, 640), 9.0, dtype=torch.bfloat16, device="cuda")
    b.typhoon_mla_cache_read(cache, slots, rows[:, :512], rows[:, 512:576])
    for i, s in enumerate(slots.tolist()):
        want_c = ckv.view(-1, 512)[s] if s >= 0 else torch.zeros_like(ckv.view(-1, 512)[0])
        want_k = kpe.view(-1, 64)[s] if s >= 0 else torch.zeros_like(kpe.view(-1, 64)[0])
        assert torch.equal(rows[i, :512], want_c) and torch.equal(rows[i, 512:576], want_k)
    assert (rows[:, 576:] == 9).all()


@pytest.mark.parametrize("bits", [8, 16])
def test_slots_outside_the_cache(b, bits):
    """Not dereferenced; reported through the status word, which keeps its other bits."""
    ckv, kpe, ex = _pages(2, 64, bits)
    before = [ckv.clone(), kpe.clone()]
    cache = b.PagedCache(ckv, kpe, ex)
    kv = torch.randn(3, 576, device="cuda").to(torch.bfloat16)
    status = torch.full((1,), 2, dtype=torch.int32, device="cuda")
    slots = torch.tensor([128, 1 << 40, -(1 << 62)], device="cuda")
    b.typhoon_mla_cache_append(cache, kv[:, :512], kv[:, 512:], slots, status=status)
    assert status.item() == 2 | b.STATUS_BAD_PAGE and torch.equal(ckv, before[0]) and torch.equal(kpe, before[1])
    status.fill_(0)
    c, k = b.typhoon_mla_cache_read(cache, slots, status=status)
    assert status.item() == b.STATUS_BAD_PAGE and not c.any() and not k.any()
    b.typhoon_mla_cache_append(cache, kv[:, :512], kv[:, 512:], slots)          # without a status word
    torch.cuda.synchronize()


def test_encoding_at_the_borders(b):
    """Rows at the scale's borders, of zeros, of subnormal values, with values that are not finite."""
    rows = torch.zeros(14, 512)
    rows[1, 3] = 448.0
    rows[2, 3] = 450.0
    rows[3, 9] = -0.875
    rows[4, 9] = 0.87890625                 # the next bf16 value: one octave up
    rows[5] = torch.linspace(-448, 448, 512)
    rows[6, 0], rows[6, 1:9] = 1.0, torch.tensor([2.0 ** -k for k in range(12, 20)])
    rows[7, 511] = 3.3e38
    rows[8] = 2.0 ** -126
    rows[9, 5] = 2.0 ** -130
    rows[10, 100] = float("inf")
    rows[11, 511] = float("nan")
    rows[12, 0] = float("-inf")
    rows[13] = -0.0
    rows = rows.to(torch.bfloat16)
    ckv, kpe, ex = _pages(1, 64, 8)
    cache = b.PagedCache(ckv, kpe, ex)
    slots = torch.arange(14, device="cuda")
    b.typhoon_mla_cache_append(cache, rows.cuda(), torch.zeros(14, 64, dtype=torch.bfloat16, device="cuda"), slots)
    x = rows.double().numpy()
    for i in range(14):
        byte, codes = ex[0, i].item(), ckv[0, i].cpu().numpy()
        if i in (10, 11, 12):
            assert byte == 255 and not codes.any()
            continue
        amax = np.abs(x[i]).max()
        e = max(int(np.log2(F.pow2_scale(amax))), -126) if amax else -126
        assert byte == e + 127, i
        y = np.minimum(np.abs(x[i]) / 2.0 ** e, 240.0 if e == 120 else 448.0)      # 2^128 is no bf16 value: 1.875 * 2^127 then
        assert np.array_equal(codes & 0x7F, F.e4m3_encode(y)), i
    c, _ = b.typhoon_mla_cache_read(cache, slots)
    for i in (10, 11, 12):
        assert torch.isnan(c[i]).all()
    table = F.e4m3_decode_table()
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 13):
        v = table[ckv[0, i].cpu().numpy()] * 2.0 ** (ex[0, i].item() - 127)
        got = c[i].double().cpu().numpy()
        if i not in (8, 9):
            assert np.array_equal(got, v), i
        else:                               # below 2^-126: bf16's own grid of 2^-133
            assert (np.abs(got - v) <= 2.0 ** -134).all(), i


def test_other_stream_and_capture(b):
    """The calls follow the current stream and replay from a graph."""
    g = torch.Generator().manual_seed(8)
    q = torch.randn(33, 16, 64, generator=g).to(torch.bfloat16).cuda()
    pos = torch.arange(33, dtype=torch.int32, device="cuda")
    rope = b.typhoon_mla_rope_init()
    want, got = torch.empty_like(q), torch.empty_like(q)
    b.typhoon_mla_rope_queries(rope, q, pos, want)
    ckv, kpe, ex = _pages(2, 64, 8)
    cache = b.PagedCache(ckv, kpe, ex)
    kv = torch.randn(33, 576, generator=g).to(torch.bfloat16).cuda()
    slots = torch.arange(33, device="cuda")
    c, k = torch.empty(33, 512, dtype=torch.bfloat16, device="cuda"), torch.empty(33, 64, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        b.typhoon_mla_rope_queries(rope, q, pos, got)
        b.typhoon_mla_cache_append(cache, kv[:, :512], kv[:, 512:], slots, rope, pos)
        b.typhoon_mla_cache_read(cache, slots, c, k)
    pos += 7
    graph.replay()
    b.typhoon_mla_rope_queries(rope, q, pos, want)
    c2, k2 = b.typhoon_mla_cache_read(cache, slots)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(c, c2) and torch.equal(k, k2)
    k3 = torch.empty(33, 1, 64, dtype=torch.bfloat16, device="cuda")
    b.typhoon_mla_rope_queries(rope, kv[:, None, 512:], pos, k3)
    assert torch.equal(k3[:, 0], k)


def test_binding_refusals(b):
    bf = torch.bfloat16
    q, pos = torch.zeros(4, 2, 64, dtype=bf, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    rope = b.typhoon_mla_rope_init()
    with pytest.raises(ValueError):
        b.typhoon_mla_rope_queries(rope, q, pos.long(), torch.empty_like(q))
    with pytest.raises(ValueError):
        b.typhoon_mla_rope_queries(rope, q, pos[:3], torch.empty_like(q))
    with pytest.raises(ValueError):
        b.typhoon_mla_rope_queries(rope, q.float(), pos, torch.empty_like(q))
    with pytest.raises(ValueError):
        b.typhoon_mla_rope_queries(rope, q, pos, torch.empty_like(q), q_nope=torch.zeros(4, 2, 128, dtype=bf, device="cuda"))
    with pytest.raises(ValueError):
        b.typhoon_mla_rope_queries(rope, q[..., ::2], pos, torch.empty_like(q))
    with pytest.raises(b.TyphoonMLAError):      # rows that do not start on 16 bytes
        b.typhoon_mla_rope_queries(rope, torch.zeros(4, 2, 68, dtype=bf, device="cuda")[..., 4:], pos, torch.empty_like(q))
    with pytest.raises(ValueError):
        b.PagedCache(torch.zeros(2, 64, 512, dtype=torch.uint8, device="cuda"), torch.zeros(2, 64, 64, dtype=bf, device="cuda"))
    with pytest.raises(ValueError):
        b.PagedCache(torch.zeros(2, 64, 512, dtype=bf, device="cuda"), torch.zeros(2, 128, 64, dtype=bf, device="cuda"))
    with pytest.raises(ValueError):             # pages that do not follow one another at the tokens' stride
        b.PagedCache(torch.zeros(2, 65, 512, dtype=bf, device="cuda")[:, :64], torch.zeros(2, 64, 64, dtype=bf, device="cuda"))
    cache = b.PagedCache(torch.zeros(2, 64, 512, dtype=bf, device="cuda"), torch.zeros(2, 64, 64, dtype=bf, device="cuda"))
    kv = torch.zeros(3, 576, dtype=bf, device="cuda")
    with pytest.raises(ValueError):
        b.typhoon_mla_cache_append(cache, kv[:, :512], kv[:, 512:], torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        b.typhoon_mla_cache_append(cache, kv[:, :512], kv[:, 512:], torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        b.typhoon_mla_cache_append(cache, kv[:, :512], kv[:, 512:], torch.zeros(3, dtype=torch.int64, device="cuda"), rope=rope)
    with pytest.raises(b.TyphoonMLAError):
        b.typhoon_mla_cache_read(cache, torch.zeros(3, dtype=torch.int64, device="cuda"), torch.empty(3, 514, dtype=bf, device="cuda")[:, :512])
    assert b.typhoon_mla_cache_read(cache, torch.zeros(0, dtype=torch.int64, device="cuda"))[0].shape == (0, 512)
