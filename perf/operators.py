"""Operators that a serving program runs next to the decode step, as measurable cases: rotary positions of the query projection,
writing new tokens into the paged latent cache (16-bit, or 8-bit codes with one power of two per token), reading cached tokens
back as 16-bit rows, and decode attention for drafted tokens (chains or trees) over a prepared prefix and either cache.

With ``own`` false ``run`` computes them in elementary torch operations in 32 bits, with ``own`` true by the package's entry
points.  Shapes follow ``paper_2509_21081_b200/inputs.py``: 128 nope + 64 rope dims per query head, latent width 512, activations
N(0, 1), projection weights N(0, 1/512), physical pages in random order.
"""
import math

import torch

own = False

SCALE = (128 + 64) ** -0.5
# rotary settings of the cases: (base, scaling, factor, original length); beta_fast 32, beta_slow 1
ROPES = {"plain": (10000.0, "none", 1.0, 4096.0), "linear": (10000.0, "linear", 4.0, 4096.0), "ntk": (10000.0, "ntk", 8.0, 8192.0),
         "yarn": (10000.0, "yarn", 40.0, 4096.0)}


def _rope(name, tokens, heads, layout, scaling, dims=64, far=32768):
    return {"name": name, "kind": "rope", "tokens": tokens, "heads": heads, "layout": layout, "scaling": scaling, "dims": dims, "far": far}


def _append(name, tokens, bits, page=64, layout="interleaved", scaling="yarn", far=32768):
    return {"name": name, "kind": "append", "tokens": tokens, "bits": bits, "page": page, "layout": layout, "scaling": scaling, "dims": 64,
            "far": far}


def _read(name, tokens, bits, page=64):
    return {"name": name, "kind": "read", "tokens": tokens, "bits": bits, "page": page}


def _draft(name, heads, batch, drafts, prefix, lo, hi, bits=16, tree=True, ragged=False, page=64):
    return {"name": name, "kind": "draft", "heads": heads, "batch": batch, "drafts": drafts, "prefix": prefix, "suffix_lo": lo,
            "suffix_hi": hi, "bits": bits, "tree": tree, "ragged": ragged, "page": page}


def listed():
    return [
        # the queries of one decode step of 64 chats, long-context scaling, pairs side by side as the projection leaves them
        _rope("rope_step", 64, 128, "interleaved", "yarn"),
        # the queries of a prompt
        _rope("rope_prompt", 4759, 128, "half", "plain"),
        # the new tokens of one decode step, into an 8-bit cache
        _append("append_step_8bit", 64, 8),
        # a long prompt enters the 16-bit cache
        _append("append_prompt", 26624, 16),
        # the prompts of a full batch enter the 8-bit cache
        _append("append_prompts_8bit", 70001, 8, 128, "half", "ntk"),
        # accepted drafts of a batch, on their way to their final places
        _read("read_accepted", 311, 16),
        # a cached prompt is read back to become a shared prefix
        _read("read_prompt_8bit", 16384, 8),
        # a small tree for a few requests on one of eight devices that share the heads: launches and latency
        _draft("draft_tiny", 16, 4, 4, 256, 64, 64),
        # two drafted tokens per request on one of eight devices, odd sizes
        _draft("draft_chain_shard", 16, 83, 2, 7069, 3, 1537, tree=False, page=128),
        # trees of eight drafts, every head on this device, trees of different sizes
        _draft("draft_tree", 128, 32, 8, 4096, 100, 700, ragged=True),
        # the ordinary step of single tokens over an 8-bit cache
        _draft("step_8bit", 128, 64, 1, 4096, 512, 512, bits=8, tree=False),
        # large trees over long ragged suffixes in an 8-bit cache
        _draft("draft_tree_long_8bit", 64, 64, 16, 8192, 128, 4096, bits=8),
    ]


def _plain_flops(case):
    return 2176.0 * case["heads"] * case["batch"] * case["drafts"] * (case["prefix"] + case["suffix_hi"])


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["rope", "append", "read", "draft", "draft", "draft", "draft"])
    layout, scaling = rng.choice(["interleaved", "half"]), rng.choice(sorted(ROPES))
    bits, page = rng.choice([8, 16]), rng.choice([64, 64, 128])
    far = log_int(1000, 1 << 20)
    if kind == "rope":
        heads = rng.choice([128, 64, 32, 16, 1])
        case = _rope("", log_int(1, 4759 * 128 // max(heads, 16)), heads, layout, scaling, rng.choice([64, 64, 32, 48]), far)
    elif kind == "append":
        case = _append("", log_int(1, 70001), bits, page, layout, scaling, far)
    elif kind == "read":
        case = _read("", log_int(1, 70001), bits, page)
    else:
        heads, batch, drafts = rng.choice([128, 128, 64, 32, 16]), log_int(1, 256), rng.choice([1, 1, 2, 3, 4, 5, 8, 16, 33, 64])
        prefix, hi = rng.choice([0, 1, 1]) * log_int(128, 16384), log_int(16, 4096)
        hi = max(hi, drafts)
        lo = rng.randint(drafts, hi)
        tree = drafts > 1 and rng.random() < 0.7
        case = _draft("", heads, batch, drafts, prefix, lo, hi, bits, tree, tree and rng.random() < 0.5, page)
        most = max(_plain_flops(c) for c in listed() if c["kind"] == "draft")
        while case["batch"] > 1 and _plain_flops(case) > most:
            case["batch"] = case["batch"] * 3 // 4
        while _plain_flops(case) > most:
            case["prefix"] //= 2
    del case["name"]
    return case


# ---------------------------------------------------------------- inputs
class State:
    pass


def _normal(gen, *shape, mul=1.0):
    return torch.empty(*shape, dtype=torch.float32, device="cuda").normal_(generator=gen).mul_(mul).to(torch.bfloat16)


def prepare(case, seed):
    gen, cpu = torch.Generator(device="cuda"), torch.Generator()
    gen.manual_seed(seed * 7919 + 29)
    cpu.manual_seed(seed * 104729 + 11)
    st = State()
    st.case = case
    kind = case["kind"]
    if kind in ("rope", "append"):
        # positions of tokens of several sequences, somewhere up to the longest context
        n = case["tokens"]
        starts = torch.randint(0, case["far"], ((n + 63) // 64,), generator=cpu).repeat_interleave(64)[:n]
        st.positions = (starts + torch.arange(n) % 64).to(torch.int32).cuda()
    if kind == "rope":
        st.q = _normal(gen, case["tokens"], case["heads"], 192)   # the projection's rows: 128 nope | 64 rope
        st.rope = _rope_handle(case)
    elif kind in ("append", "read"):
        n, page = case["tokens"], case["page"]
        pages = (n + page - 1) // page + 2
        # consecutive tokens of one sequence in pages of random order
        order = torch.randperm(pages, generator=cpu)
        at = torch.arange(n)
        st.slots = (order[at // page] * page + at % page).cuda()
        if kind == "append":
            st.kv = _normal(gen, n, 576)                          # the projection's rows: 512 latent | 64 rope
            st.rope = _rope_handle(case)
        _cache(st, gen, pages, page, case["bits"])
    else:
        H, B, S, page = case["heads"], case["batch"], case["drafts"], case["page"]
        st.ckv, st.kpe = _normal(gen, case["prefix"], 512), _normal(gen, case["prefix"], 64)
        st.w_uk, st.w_uv = _normal(gen, H, 128, 512, mul=512 ** -0.5), _normal(gen, H, 128, 512, mul=512 ** -0.5)
        st.q_nope, st.q_pe = _normal(gen, B * S, H, 128), _normal(gen, B * S, H, 64)
        lens = torch.randint(case["suffix_lo"], case["suffix_hi"] + 1, (B,), generator=cpu)
        need, st.max_pages = (lens + page - 1) // page, (case["suffix_hi"] + page - 1) // page
        total = int(need.sum())
        table = torch.full((B, st.max_pages), -1, dtype=torch.int32)
        table[torch.arange(st.max_pages)[None, :] < need[:, None]] = torch.randperm(total + 2, generator=cpu)[:total].to(torch.int32)
        _cache(st, gen, total + 2, page, case["bits"])
        st.table, st.lens = table.cuda(), lens.to(torch.int32).cuda()
        st.counts = torch.randint(1, S + 1, (B,), generator=cpu).to(torch.int32).cuda() if case["ragged"] else None
        st.mask = None
        if case["tree"]:
            # draft j hangs under an earlier one (or under the last committed token) and sees its ancestors and itself
            sees = torch.zeros(B, S + 1, S, dtype=torch.bool)
            for j in range(S):
                parent = torch.randint(-1, j, (B,), generator=cpu)
                sees[:, j] = sees[torch.arange(B), parent]        # -1: the empty row at the end
                sees[:, j, j] = True
            st.mask = (sees[:, :S].to(torch.int64) << torch.arange(S)).sum(-1).cuda()
        if own:
            # the handle that a serving program keeps: the expanded prefix and the workspace
            from paper_2509_21081_b200.decoder import TyphoonMLADecoder
            st.decoder = TyphoonMLADecoder(H, st.ckv, st.kpe, st.w_uk, st.w_uv, SCALE, B, st.max_pages, page, max_drafts=S)
    torch.cuda.synchronize()
    return st


def _rope_handle(case):
    """The rotary settings as the program keeps them: the library's structure, or nothing."""
    if not own:
        return None
    from paper_2509_21081_b200 import binding as b
    base, scaling, factor, length = ROPES[case["scaling"]]
    return b.typhoon_mla_rope_init(case["dims"], layout=case["layout"], base=base, scaling=scaling, factor=factor, original_length=length,
                                   beta_fast=32.0, beta_slow=1.0)


def _cache(st, gen, pages, page, bits):
    """Pages filled with tokens: 16-bit latent rows, or codes of random latent rows under a power of two per token."""
    latent = torch.empty(pages, page, 512, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    st.kpe_pages = torch.empty(pages, page, 64, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    st.exponents = None
    if bits == 8:
        st.exponents = torch.randint(116, 123, (pages, page), generator=gen, device="cuda", dtype=torch.uint8)
        latent = latent.float().mul_(100.0).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    st.ckv_pages = latent
    if own:
        from paper_2509_21081_b200 import binding as b
        st.cache = b.PagedCache(st.ckv_pages, st.kpe_pages, st.exponents)


# ---------------------------------------------------------------- plain forms
def _frequencies(case):
    """Radians per position of every rotated pair, in 64 bits."""
    base, scaling, factor, length = ROPES[case["scaling"]]
    d = case["dims"]
    i = torch.arange(d // 2, dtype=torch.float64, device="cuda")
    if scaling == "ntk":
        base = base * factor ** (d / (d - 2))
    f = base ** (-2.0 * i / d)
    if scaling == "linear":
        f = f / factor
    if scaling == "yarn":
        # pairs that turn more than 32 times over the original length keep their frequency, fewer than once: interpolated
        low = max(math.floor(d * math.log(length / (32.0 * 2 * math.pi)) / (2 * math.log(base))), 0)
        high = min(math.ceil(d * math.log(length / (1.0 * 2 * math.pi)) / (2 * math.log(base))), d - 1)
        ramp = ((i - low) / max(high - low, 0.001)).clamp(0.0, 1.0)
        f = f / factor * ramp + f * (1.0 - ramp)
    return f


def _rotated(case, x, positions):
    """x [tokens, .., 64] in 32 (64) bits, its first `dims` dims rotated; angles in 64 bits."""
    d, one = case["dims"], x.shape[1:-1]
    angle = (positions.double()[:, None] * _frequencies(case)).reshape(-1, *[1] * len(one), d // 2)
    c, s = torch.cos(angle).to(x.dtype), torch.sin(angle).to(x.dtype)
    if case["layout"] == "half":
        a, b = x[..., :d // 2], x[..., d // 2:d]
        y = torch.cat([a * c - b * s, a * s + b * c], -1)
    else:
        a, b = x[..., 0:d:2], x[..., 1:d:2]
        y = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    return torch.cat([y, x[..., d:]], -1)


def _power(n):
    """2^n exactly (torch.ldexp and torch.pow round on the GPU), -127 < n < 128."""
    return (n.int() + 127 << 23).view(torch.float32)


def _encoded(latent):
    """Codes and exponent bytes of latent rows: the smallest power of two under which a row fits +-448."""
    m, e = torch.frexp(latent.float().abs().amax(-1))
    byte = (e + 127 - 8 - (m <= 0.875).int()).clamp(min=1)
    byte = torch.where(m == 0, torch.ones_like(byte), byte)
    codes = (latent.float() * _power(127 - byte)[:, None]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), byte.to(torch.uint8)


def _values(codes, exponents):
    return codes.view(torch.float8_e4m3fn).float() * _power(exponents.int() - 127)[..., None]


def _visible(st, tokens):
    """[batch, drafts, tokens]: what every drafted token sees of its request's cached tokens."""
    B, S = st.case["batch"], st.case["drafts"]
    j = torch.arange(S, device="cuda")
    counts = torch.full((B,), S, device="cuda") if st.counts is None else st.counts.long()
    mask = ((2 << j) - 1).expand(B, S) if st.mask is None else st.mask
    t = torch.arange(tokens, device="cuda")
    draft = t - (st.lens.long() - counts)[:, None, None]                        # [batch, 1, tokens], < 0: committed
    sees = (draft < 0) | ((mask[..., None] >> draft.clamp(0, 63)) & 1 != 0)
    return sees & (t < st.lens[:, None, None])


def _plain_draft(st):
    c = st.case
    B, S, H, tokens = c["batch"], c["drafts"], c["heads"], st.max_pages * c["page"]
    q = torch.cat([torch.einsum("rhd,hdc->rhc", st.q_nope.float(), st.w_uk.float()), st.q_pe.float()], -1) * SCALE
    q = q.reshape(B, S * H, 576)
    ids = st.table.clamp(min=0).long()
    latent = st.ckv_pages[ids].float() if c["bits"] == 16 else _values(st.ckv_pages[ids], st.exponents[ids])
    latent = latent.reshape(B, tokens, 512)
    keys = torch.cat([latent, st.kpe_pages[ids].float().reshape(B, tokens, 64)], -1)
    logits = (q @ keys.transpose(1, 2)).view(B, S, H, tokens)
    logits.masked_fill_(~_visible(st, tokens)[:, :, None], -math.inf)
    logits = logits.view(B, S * H, tokens)
    top = logits.amax(-1, keepdim=True)
    prefix = None
    if c["prefix"]:
        prefix = q @ torch.cat([st.ckv, st.kpe], -1).float().T
        top = torch.maximum(top, prefix.amax(-1, keepdim=True))
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    weights = logits.sub_(top).exp_()
    total, o = weights.sum(-1, keepdim=True), weights @ latent
    if prefix is not None:
        weights = prefix.sub_(top).exp_()
        total, o = total + weights.sum(-1, keepdim=True), o + weights @ st.ckv.float()
    o = torch.where(total > 0, o / total, torch.zeros_like(o)).view(B * S, H, 512)
    return torch.einsum("rhc,hdc->rhd", o, st.w_uv.float()).to(torch.bfloat16)


# ---------------------------------------------------------------- one pass
def run(st):
    c = st.case
    if c["kind"] == "rope":
        if own:
            from paper_2509_21081_b200 import binding as b
            q_nope = torch.empty(c["tokens"], c["heads"], 128, dtype=torch.bfloat16, device="cuda")
            q_pe = torch.empty(c["tokens"], c["heads"], 64, dtype=torch.bfloat16, device="cuda")
            b.typhoon_mla_rope_queries(st.rope, st.q[..., 128:], st.positions, q_pe, st.q[..., :128], q_nope)
            return q_nope, q_pe
        return st.q[..., :128].contiguous(), _rotated(c, st.q[..., 128:].float(), st.positions).to(torch.bfloat16)
    if c["kind"] == "append":
        latent, key = st.kv[:, :512], st.kv[:, 512:]
        if own:
            from paper_2509_21081_b200 import binding as b
            b.typhoon_mla_cache_append(st.cache, latent, key, st.slots, rope=st.rope, positions=st.positions)
        else:
            rows = latent
            if c["bits"] == 8:
                rows, byte = _encoded(latent)
                st.exponents.view(-1)[st.slots] = byte
            st.ckv_pages.view(-1, 512)[st.slots] = rows
            st.kpe_pages.view(-1, 64)[st.slots] = _rotated(c, key.float(), st.positions).to(torch.bfloat16)
        if c["bits"] == 8:
            return st.ckv_pages.view(torch.float8_e4m3fn), st.exponents, st.kpe_pages
        return st.ckv_pages, st.kpe_pages
    if c["kind"] == "read":
        if own:
            from paper_2509_21081_b200 import binding as b
            return b.typhoon_mla_cache_read(st.cache, st.slots)
        latent = st.ckv_pages.view(-1, 512)[st.slots]
        if c["bits"] == 8:
            latent = _values(latent, st.exponents.view(-1)[st.slots]).to(torch.bfloat16)
        return latent, st.kpe_pages.view(-1, 64)[st.slots]
    if own:
        return st.decoder.decode_draft(st.q_nope, st.q_pe, st.cache, st.table, st.lens, tree_mask=st.mask, draft_lens=st.counts)
    return _plain_draft(st)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Every input read once and every output written once, at 2 operations per multiply-add; of attention over the prefix the
    cheaper formulation (expanded per-head keys and values, or the latent rows)."""
    if case["kind"] == "rope":
        return {"bytes": 768.0 * case["tokens"] * case["heads"] + 4.0 * case["tokens"], "flops": 3.0 * case["tokens"] * case["heads"] * case["dims"]}
    if case["kind"] != "draft":
        token = 1152 if case["bits"] == 16 else 641
        return {"bytes": (1152.0 + token + 8 + (4 if case["kind"] == "append" else 0)) * case["tokens"], "flops": 512.0 * case["tokens"]}
    H, rows = case["heads"], case["batch"] * case["drafts"]
    suffix = case["batch"] * (case["suffix_lo"] + case["suffix_hi"]) / 2
    flops = 262144.0 * H * rows + 2176.0 * H * case["drafts"] * suffix
    bytes_ = 640.0 * H * rows + 262144.0 * H + (1152.0 if case["bits"] == 16 else 641.0) * suffix
    n = case["prefix"]
    if n:
        expanded = {"flops": 640.0 * H * rows * n, "bytes": (512.0 * H + 128.0) * n}
        latent = {"flops": 2176.0 * H * rows * n, "bytes": 1152.0 * n}
        best = min((expanded, latent), key=lambda w: max(w["bytes"] / 6.5e12, w["flops"] / 1.6e15))
        flops, bytes_ = flops + best["flops"], bytes_ + best["bytes"]
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    two = lambda n: (n.to(torch.int64) + 1023 << 52).view(torch.float64)   # noqa: E731  (2^n; torch.pow rounds on the GPU)
    if kind in ("rope", "append"):
        # pair i of a row is the complex number (x_a, x_b), turned by positions * frequency
        x = (st.q[..., 128:] if kind == "rope" else st.kv[:, None, 512:]).double()
        d = case["dims"]
        base, scaling, factor, length = ROPES[case["scaling"]]
        freq = []
        for i in range(d // 2):
            b = base * factor ** (d / (d - 2.0)) if scaling == "ntk" else base
            f = math.exp(-2.0 * i / d * math.log(b))
            if scaling == "linear":
                f /= factor
            if scaling == "yarn":
                lo = max(0, math.floor(d / 2 * math.log(length / 32 / (2 * math.pi), base)))
                hi = min(d - 1, math.ceil(d / 2 * math.log(length / (2 * math.pi), base)))
                keep = 1.0 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3)))
                f = f * keep + f / factor * (1.0 - keep)
            freq.append(f)
        turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"),
                           torch.outer(st.positions.double(), torch.tensor(freq, dtype=torch.float64, device="cuda")))[:, None]
        a, b = (list(range(0, d, 2)), list(range(1, d, 2))) if case["layout"] == "interleaved" else (list(range(d // 2)), list(range(d // 2, d)))
        z = torch.complex(x[..., a], x[..., b]) * turn
        y = x.clone()
        y[..., a], y[..., b] = z.real, z.imag
        if kind == "rope":
            return st.q[..., :128].double(), y
        kpe = st.kpe_pages.double()
        kpe.view(-1, 64)[st.slots] = y[:, 0]
        if case["bits"] == 16:
            ckv = st.ckv_pages.double()
            ckv.view(-1, 512)[st.slots] = st.kv[:, :512].double()
            return ckv, kpe
        # smallest power of two with amax / 2^e <= 448, then E4M3: steps of 2^-3 of the value's own power of two, at least 2^-9
        v = st.kv[:, :512].double()
        amax = v.abs().amax(-1)
        e = torch.floor(torch.log2(amax / 448.0)) - 1
        e = e + (amax > 448.0 * two(e))
        e = e + (amax > 448.0 * two(e))
        e = e + (amax > 448.0 * two(e))
        v = v / two(e)[:, None]
        _, above = torch.frexp(v.abs().clamp(min=2.0 ** -6))
        step = two(above - 4)
        ckv, byte = st.ckv_pages.view(torch.float8_e4m3fn).double(), st.exponents.clone()
        ckv.view(-1, 512)[st.slots] = (torch.round(v / step) * step).clamp(-448.0, 448.0)
        byte.view(-1)[st.slots] = (e + 127).to(torch.uint8)
        return ckv, byte, kpe
    if kind == "read":
        latent = st.ckv_pages.view(-1, 512)[st.slots]
        if case["bits"] == 8:
            scale = two(st.exponents.view(-1)[st.slots].long() - 127)
            latent = latent.view(torch.float8_e4m3fn).double() * scale[:, None]
        return latent.double(), st.kpe_pages.view(-1, 64)[st.slots].double()
    # attention: every request by itself, keys and values decompressed for a group of heads at a time
    B, S, H, page = case["batch"], case["drafts"], case["heads"], case["page"]
    out = torch.zeros(B, S, H, 128, dtype=torch.float64, device="cuda")
    qn, qp = st.q_nope.double().view(B, S, H, 128), st.q_pe.double().view(B, S, H, 64)
    w_uk, w_uv = st.w_uk.double(), st.w_uv.double()
    q_lat = torch.einsum("bshd,hdc->bshc", qn, w_uk)
    lens, counts = st.lens.tolist(), [S] * B if st.counts is None else st.counts.tolist()
    masks = [[(2 << j) - 1 for j in range(S)]] * B if st.mask is None else st.mask.tolist()
    ckv, kpe = st.ckv.double(), st.kpe.double()
    for r in range(B):
        n = lens[r]
        ids = st.table[r, :(n + page - 1) // page].long()
        c = st.ckv_pages[ids]
        c = c.double() if case["bits"] == 16 else c.view(torch.float8_e4m3fn).double() * two(st.exponents[ids].long() - 127)[..., None]
        c, k = c.reshape(-1, 512)[:n], st.kpe_pages[ids].double().reshape(-1, 64)[:n]
        own_logits = (torch.einsum("shc,tc->sht", q_lat[r], c) + torch.einsum("shd,td->sht", qp[r], k)) * SCALE
        hidden = torch.zeros(S, n, dtype=torch.bool)
        for j in range(S):
            for i in range(counts[r]):
                if n - counts[r] + i >= 0 and not (masks[r][j] >> i) & 1:
                    hidden[j, n - counts[r] + i] = True
        own_logits.masked_fill_(hidden.cuda()[:, None], -math.inf)
        logits = torch.cat([(torch.einsum("shc,tc->sht", q_lat[r], ckv) + torch.einsum("shd,td->sht", qp[r], kpe)) * SCALE, own_logits], -1)
        seen = torch.isfinite(logits).any(-1, keepdim=True)
        p = torch.where(seen, torch.softmax(logits, -1), torch.zeros_like(logits))
        out[r] = torch.einsum("shc,hdc->shd", torch.einsum("sht,tc->shc", p, torch.cat([ckv, c])), w_uv)
    return out.view(B * S, H, 128)
