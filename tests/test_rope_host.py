"""CPU tests of the rotary settings and of what the calls around a step refuse (no kernel runs)."""
import ctypes as C
import math

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2509_21081_b200 import build
    build.build()
    from paper_2509_21081_b200 import binding
    return binding


def frequencies(d, base, scaling, factor, length, beta_fast, beta_slow):
    """From the definitions, one pair at a time."""
    out = []
    for i in range(d // 2):
        if scaling == "ntk":
            out.append((base * factor ** (d / (d - 2))) ** (-2 * i / d))
            continue
        f = base ** (-2 * i / d)
        if scaling == "linear":
            f /= factor
        elif scaling == "yarn":
            def pair(beta):
                return d * math.log(length / (2 * math.pi * beta)) / (2 * math.log(base))
            low, high = max(math.floor(pair(beta_fast)), 0), min(math.ceil(pair(beta_slow)), d - 1)
            ramp = min(max((i - low) / max(high - low, 0.001), 0), 1)
            f = f / factor * ramp + f * (1 - ramp)
        out.append(f)
    return out


@pytest.mark.parametrize("d", [16, 32, 48, 64])
@pytest.mark.parametrize("scaling,factor,length", [("none", 1.0, 4096), ("linear", 4.0, 4096), ("ntk", 8.0, 8192), ("yarn", 40.0, 4096),
                                                    ("yarn", 1.0, 1), ("yarn", 32.0, 131072)])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_turns(b, d, scaling, factor, length, base):
    r = b.typhoon_mla_rope_init(d, "half", base, scaling, factor, length, 32.0, 1.0, 1.25)
    assert (r.d_rot, r.layout, r.scale) == (d, 1, 1.25)
    want = frequencies(d, base, scaling, factor, length, 32.0, 1.0)
    for i, f in enumerate(want):
        # both sides form f in 64 bits (a few 2^-53 each, pow and the ramp among them); the table adds half of 2^-64
        assert abs(r.turns[i] / 2 ** 64 - f / (2 * math.pi)) <= 1e-14 * f + 2.0 ** -63
    assert all(r.turns[i] == 0 for i in range(d // 2, 32))


@pytest.mark.parametrize("args", [dict(d_rot=0), dict(d_rot=8), dict(d_rot=24), dict(d_rot=80), dict(base=1.0), dict(base=math.inf),
                                  dict(base=math.nan), dict(scaling="linear", factor=0.5), dict(scaling="ntk", factor=math.nan),
                                  dict(scaling="yarn", factor=2.0, original_length=0.0), dict(scaling="yarn", factor=2.0, beta_slow=0.0),
                                  dict(scaling="yarn", factor=2.0, beta_fast=0.5), dict(scale=math.nan), dict(scale=math.inf)])
def test_rope_init_refuses(b, args):
    with pytest.raises(b.TyphoonMLAError, match="invalid argument"):
        b.typhoon_mla_rope_init(**args)


def test_rope_init_refuses_codes(b):
    r = b.Rope()
    for layout, scaling in ((2, 0), (-1, 0), (0, 4), (0, -1)):
        assert b._lib.typhoon_mla_rope_init(C.byref(r), 64, layout, 1e4, scaling, 1.0, 4096.0, 32.0, 1.0, 1.0) == 1
    assert b._lib.typhoon_mla_rope_init(None, 64, 0, 1e4, 0, 1.0, 4096.0, 32.0, 1.0, 1.0) == 1
    assert r.d_rot == 0                       # a refused call leaves the structure alone


A = 4096          # an aligned address that no refused call reads


def _rope_queries(b, **kw):
    a = dict(rope=b.typhoon_mla_rope_init(), nope=A, nt=24576, nh=192, pe=A, pt=24576, ph=192, pos=A, T=3, H=2, no=A, po=A)
    a.update(kw)
    return b._lib.typhoon_mla_rope_queries(None if a["rope"] is None else C.byref(a["rope"]), a["nope"], a["nt"], a["nh"], a["pe"], a["pt"],
                                           a["ph"], a["pos"], a["T"], a["H"], a["no"], a["po"], None)


@pytest.mark.parametrize("kw", [dict(rope=None), dict(T=-1), dict(H=0), dict(H=70000), dict(nope=None), dict(no=None), dict(pe=None),
                                dict(po=None), dict(pos=None), dict(pe=A + 2), dict(po=A + 8), dict(nope=A + 8), dict(no=A + 4), dict(pos=A + 1),
                                dict(pt=100), dict(ph=4), dict(nt=100), dict(nh=190), dict(T=1 << 41)])
def test_rope_queries_refuses(b, kw):
    assert _rope_queries(b, **kw) == 1


def test_rope_queries_refuses_bad_settings(b):
    for change in (dict(d_rot=20), dict(d_rot=128), dict(layout=2), dict(scale=math.nan)):
        r = b.typhoon_mla_rope_init()
        for k, v in change.items():
            setattr(r, k, v)
        assert _rope_queries(b, rope=r) == 1
        assert b._lib.typhoon_mla_cache_append(C.byref(_cache(b)), A, 512, A, 64, C.byref(r), A, A, 3, None, None) == 1


def test_no_tokens_is_no_work(b):
    assert _rope_queries(b, T=0, pe=None, po=None, pos=None, nope=None, no=None) == 0
    c = _cache(b)
    assert b._lib.typhoon_mla_cache_append(C.byref(c), None, 512, None, 64, None, None, None, 0, None, None) == 0
    assert b._lib.typhoon_mla_cache_read(C.byref(c), None, 0, None, 512, None, 64, None, None) == 0
    assert b.typhoon_mla_last_launch_count() == 0


def _cache(b, **kw):
    a = dict(ckv_pages=A, kpe_pages=A, ckv_exponents=None, ckv_token_stride=512, kpe_token_stride=64, page_size=64, num_pages=4)
    a.update(kw)
    return b.Cache(**a)


@pytest.mark.parametrize("kw", [dict(ckv_pages=None), dict(kpe_pages=None), dict(ckv_pages=A + 8), dict(kpe_pages=A + 8), dict(page_size=32),
                                dict(page_size=0), dict(num_pages=0), dict(ckv_token_stride=504), dict(ckv_token_stride=516),
                                dict(kpe_token_stride=56), dict(kpe_token_stride=68), dict(ckv_exponents=A + 8),
                                dict(ckv_exponents=A, ckv_token_stride=520)])
def test_cache_refuses(b, kw):
    c = _cache(b, **kw)
    assert b._lib.typhoon_mla_cache_append(C.byref(c), A, 512, A, 64, None, None, A, 3, None, None) == 1
    assert b._lib.typhoon_mla_cache_read(C.byref(c), A, 3, A, 512, A, 64, None, None) == 1


@pytest.mark.parametrize("at,value", [(0, None), (1, None), (1, A + 8), (2, 504), (2, 516), (3, None), (3, A + 4), (4, 32), (4, 68),
                                      (6, A), (7, None), (7, A + 4), (8, -1), (9, A + 2)])
def test_append_refuses(b, at, value):
    args = [C.byref(_cache(b)), A, 512, A, 64, None, None, A, 3, None, None]
    args[at] = value
    assert b._lib.typhoon_mla_cache_append(*args) == 1


@pytest.mark.parametrize("at,value", [(0, None), (1, None), (1, A + 4), (2, -1), (3, None), (3, A + 8), (4, 500), (5, None), (5, A + 8),
                                      (6, 56), (7, A + 2)])
def test_read_refuses(b, at, value):
    args = [C.byref(_cache(b)), A, 3, A, 512, A, 64, None, None]
    args[at] = value
    assert b._lib.typhoon_mla_cache_read(*args) == 1


def test_bindings_check_their_tensors(b):
    import torch
    x = torch.zeros(4, 6, dtype=torch.int32)                       # get_device() of a CPU tensor: -1
    assert b._need(x, "x", torch.int32, (4, 6), -1) == x.data_ptr()
    assert b._need(x[:, :3], "x", torch.int32, (4, 3), -1, contiguous=False) == x.data_ptr()
    for t, dtype, shape, dev, contiguous, match in ((x, torch.int32, (4, 6), 0, True, "CUDA device"), (x, torch.int64, (4, 6), -1, True, "int64"),
                                                    (x, torch.int32, (4, 5), -1, True, "shape"), (x[:, :3], torch.int32, (4, 3), -1, True, "contiguous"),
                                                    (x[:, ::2], torch.int32, (4, 3), -1, False, "dense")):
        with pytest.raises(ValueError, match=match):
            b._need(t, "x", dtype, shape, dev, contiguous)
    with pytest.raises(ValueError, match="dimensions"):
        b._sizes(x, 3, "x")
    assert b._steps(torch.zeros(1, 5, 64)) == (0, 64) and b._steps(torch.zeros(5, 1, 64)) == (64, 0)
