"""CPU tests of calls around a step at the ends of what they take (no kernel runs)."""
import ctypes as C

import pytest

from tests.test_rope_host import A, _cache


@pytest.fixture(scope="module")
def b():
    from paper_2509_21081_b200 import build
    build.build()
    from paper_2509_21081_b200 import binding
    return binding


def test_append_of_no_tokens_with_rotation(b):
    """An empty tensor of positions has no address: no tokens is no work with rotary settings as well."""
    c, r = _cache(b), b.typhoon_mla_rope_init()
    assert b._lib.typhoon_mla_cache_append(C.byref(c), None, 512, None, 64, C.byref(r), None, None, 0, None, None) == 0
    assert b.typhoon_mla_last_launch_count() == 0
    # with tokens the two go together, and the cache and the settings are checked either way
    assert b._lib.typhoon_mla_cache_append(C.byref(c), A, 512, A, 64, C.byref(r), None, A, 3, None, None) == 1
    assert b._lib.typhoon_mla_cache_append(C.byref(c), A, 512, A, 64, None, A, A, 3, None, None) == 1
    bad = _cache(b, page_size=32)
    assert b._lib.typhoon_mla_cache_append(C.byref(bad), None, 512, None, 64, C.byref(r), None, None, 0, None, None) == 1
    r.d_rot = 20
    assert b._lib.typhoon_mla_cache_append(C.byref(c), None, 512, None, 64, C.byref(r), None, None, 0, None, None) == 1


def test_rope_init_refuses_a_scale_that_is_infinite_in_32_bits(b):
    """What rope_init accepts, the calls that take it accept."""
    for scale in (1e39, -1e39):
        with pytest.raises(b.TyphoonMLAError, match="invalid argument"):
            b.typhoon_mla_rope_init(scale=scale)
    assert b.typhoon_mla_rope_init(scale=3.4e38).scale > 3.3e38
