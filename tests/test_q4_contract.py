"""The limits that include/vd.h states for the calls on a 4-bit cache: each is refused just
beyond it (CPU only, before any launch)."""
import ctypes

import pytest

INVALID, UNSUPPORTED = 1, 3


@pytest.fixture(scope="module")
def lib():
    from paper_2609_23314_gb300 import build, load_library
    build.build()
    return load_library()


def q4(n_seq=1, n_layer=1, n_kv_head=2, head_dim=64, capacity=128):
    from paper_2609_23314_gb300 import _VdQ4Cache
    return ctypes.byref(_VdQ4Cache(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, n_seq, n_layer,
                                   n_kv_head, head_dim, capacity))


def attend(lib, cache, heads=4, B=1, scale=1.0):
    return lib.vd_q4_attend(cache, 0, 0x100, heads, None, None, B, scale, 0x200, None, None)


@pytest.mark.parametrize("scale", [0.0, -0.0, -1e-30, 3.4028234e38, float("inf"), float("nan")])
def test_scale(lib, scale):
    assert attend(lib, q4(), scale=scale) == INVALID


def test_tokens_and_query_rows(lib):
    assert attend(lib, q4(), B=0) == INVALID
    assert attend(lib, q4(), B=-1) == INVALID
    assert attend(lib, q4(n_kv_head=1), heads=1, B=(1 << 24) + 1) == UNSUPPORTED
    assert attend(lib, q4(n_kv_head=1), heads=3, B=(1 << 24) // 3 + 1) == UNSUPPORTED
    # 2^27 query rows in all, 2^23 of each KV head
    assert attend(lib, q4(n_seq=8, n_kv_head=2), heads=2, B=1 << 23) == UNSUPPORTED
    assert attend(lib, q4(n_seq=2, n_kv_head=2), heads=16, B=1 << 22) == UNSUPPORTED


def test_append_of_no_rows(lib):
    assert lib.vd_q4_append(q4(), 0x100, 0x200, 0, None) == 0
    assert lib.vd_q4_append(q4(), None, 0x200, 0, None) == INVALID


def test_cache_size(lib):
    for bad in (dict(capacity=(1 << 30) + 8), dict(n_seq=1 << 20, n_layer=64),
                dict(n_seq=134217728, n_kv_head=1)):
        assert attend(lib, q4(**bad), heads=2) == UNSUPPORTED


def test_projection_size(lib):
    def call(n_seq=1, B=1, n_q=4, n_kv=2):
        return lib.vd_qkv_norm_rope(0x100, n_seq, B, n_q, n_kv, 64, None, None, 1e-6, 0x40, 64, 0,
                                    0x80, 0x200, 0x300, 0x400, 0, 1, None)

    assert call(n_seq=1 << 16, B=1 << 15) == UNSUPPORTED
    assert call(n_q=65536) == UNSUPPORTED
