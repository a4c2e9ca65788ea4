"""Calls on a paged cache refuse bad arguments before any launch (CPU only), in C and in the
binding."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2609_23314_gb300 import build, load_library
    build.build()
    return load_library()


def _paged(k=0x1000, v=0x2000, ks=0, vs=0, table=0x3000, ln=0x4000, layer=1 << 20, page=2048,
           head=1024, slot=64, type=0, n_seq=1, n_layer=2, n_kv_head=2, head_dim=64, page_size=16,
           n_page=8, max_pages=4):
    from paper_2609_23314_gb300 import _VdPagedCache
    return ctypes.byref(_VdPagedCache(k, v, ks, vs, table, ln, layer, page, head, slot, type,
                                      n_seq, n_layer, n_kv_head, head_dim, page_size, n_page,
                                      max_pages))


def _cache(n_seq=1, n_layer=1, n_kv_head=2, head_dim=64, capacity=128, k=0x1000):
    from paper_2609_23314_gb300 import _VdCache
    return ctypes.byref(_VdCache(k, 0x2000, 0x3000, n_seq, n_layer, n_kv_head, head_dim,
                                 capacity))


def _append(lib, c, layer=0, qkv=0x100, B=1, n_q=4, new=None, qw=None, kw=None, eps=1e-6,
            freq=0x40, rd=64, inter=0, pos=None, q=0x200):
    return lib.vd_paged_append(c, layer, qkv, B, n_q, new, qw, kw, eps, freq, rd, inter, pos, q,
                               None)


def _attend(lib, c, layer=0, q=0x100, B=1, n_q=4, new=None, causal=1, scale=1.0, out=0x200,
            work=0x300, size=1 << 40):
    return lib.vd_paged_attend(c, layer, q, B, n_q, new, causal, scale, out, None, work, size, None)


@pytest.mark.parametrize("fields,code", [
    (dict(k=0), 1), (dict(v=0), 1), (dict(table=0), 1), (dict(ln=0), 1), (dict(type=2), 1),
    (dict(type=-1), 1), (dict(ks=0x500), 1), (dict(vs=0x500), 1), (dict(n_seq=0), 1),
    (dict(n_layer=0), 1), (dict(n_kv_head=0), 1), (dict(head_dim=0), 1), (dict(page_size=0), 1),
    (dict(n_page=0), 1), (dict(max_pages=0), 1), (dict(slot=56), 1), (dict(head=0), 1),
    (dict(page=-2048), 1), (dict(layer=8), 1),
    (dict(k=0x1008), 2), (dict(v=0x2001), 2), (dict(head_dim=60), 2), (dict(slot=68), 2),
    (dict(type=1, head_dim=56), 2), (dict(type=1, slot=72), 2), (dict(page=2052), 2),
    (dict(head_dim=264, slot=264, head=1 << 14, page=1 << 16), 3),
    (dict(page_size=1 << 16, max_pages=(1 << 14) + 1), 3), (dict(n_seq=(1 << 20) + 1), 3),
    (dict(n_kv_head=65537), 3), (dict(n_seq=1 << 20, n_layer=2048), 3),
])
def test_bad_cache(lib, fields, code):
    c = _paged(**fields)
    assert _append(lib, c, rd=0, freq=None) == code
    assert _attend(lib, c, n_q=65537 if "n_kv_head" in fields else 4) == code
    assert lib.vd_paged_attend_workspace(c, 4, 1) == 0
    assert lib.vd_paged_advance(c, None, 1, None) == code
    assert lib.vd_paged_pack(c, 0, _cache(), None) == code
    assert lib.vd_paged_unpack(c, 0, _cache(), None) == code


def test_strides_of_an_extent_of_one_do_not_count(lib):
    c = _paged(layer=0, n_layer=1, head=3, n_kv_head=1, slot=0, page_size=1, page=-1, n_page=1)
    assert _append(lib, c, layer=1) == 1  # refused for its layer, behind the cache's checks
    assert _append(lib, c, qkv=0x108, n_q=4) == 2


def test_bad_arguments(lib):
    c = _paged()
    for bad in (dict(layer=2), dict(layer=-1), dict(qkv=None), dict(q=None), dict(B=0), dict(n_q=0),
                dict(rd=-16), dict(rd=80), dict(freq=None), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=2.0)):
        assert _append(lib, c, **bad) == 1, bad
    for bad in (dict(qkv=0x108), dict(q=0x208), dict(qw=0x8), dict(kw=0x2)):
        assert _append(lib, c, **bad) == 2, bad
    for bad in (dict(rd=40), dict(rd=2), dict(n_q=1 << 20)):
        assert _append(lib, c, **bad) == 3, bad
    for bad in (dict(layer=2), dict(layer=-1), dict(q=None), dict(out=None), dict(work=None),
                dict(B=0), dict(n_q=0), dict(n_q=3), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("nan")), dict(scale=float("inf"))):
        assert _attend(lib, c, **bad) == 1, bad
    for bad in (dict(q=0x108), dict(out=0x208), dict(work=0x308)):
        assert _attend(lib, c, **bad) == 2, bad
    for bad in (dict(B=1 << 24), dict(n_q=1 << 26)):
        assert _attend(lib, c, **bad) == 3, bad
        assert lib.vd_paged_attend_workspace(c, bad.get("n_q", 4), bad.get("B", 1)) == 0
    assert lib.vd_paged_advance(c, None, -1, None) == 1
    assert lib.vd_paged_advance(None, None, 1, None) == 1
    for f in (lib.vd_paged_pack, lib.vd_paged_unpack):
        assert f(None, 0, _cache(), None) == 1
        assert f(c, 0, None, None) == 1
        for bad in (dict(n_seq=2), dict(n_kv_head=3), dict(head_dim=32), dict(n_layer=3),
                    dict(n_layer=0), dict(capacity=0), dict(k=0)):
            assert f(c, 0, _cache(**bad), None) == 1, bad
        assert f(c, 2, _cache(), None) == 1
        assert f(c, -1, _cache(), None) == 1
        assert f(c, 0, _cache(k=0x1008), None) == 2


def bf(*s):
    return torch.zeros(s, dtype=torch.bfloat16)


def test_the_binding_checks_its_tensors():
    import paper_2609_23314_gb300 as vd
    c = vd.PagedCache.empty(2, 3, 2, 64, n_page=5, page_size=16, max_pages=4, device="cpu")
    assert (c.n_seq, c.n_layer, c.n_kv_head, c.head_dim, c.n_page, c.page_size, c.max_pages) == \
        (2, 3, 2, 64, 5, 16, 4)
    assert bool((c.page_table == -1).all())
    new = lambda **kw: vd.PagedCache(**dict(dict(k=c.k, v=c.v, page_table=c.page_table, len=c.len),
                                            **kw))
    tok = torch.zeros((3, 5, 16, 2, 64), dtype=torch.bfloat16).transpose(2, 3)
    assert new(k=tok, v=tok)._s.slot_stride == 128
    f8 = c.k.to(torch.float8_e4m3fn)
    assert new(k=f8, v=f8, k_scale=torch.ones(3, 2)).type == vd.VD_PAGED_E4M3
    for error, match, kw in (
            (ValueError, "strides", dict(v=tok)),
            (ValueError, "strides", dict(k=c.k.transpose(3, 4), v=c.v.transpose(3, 4))),
            (ValueError, "shape", dict(v=c.v[:2])),
            (TypeError, "v must be", dict(v=f8)),
            (TypeError, "k must be", dict(k=c.k.half(), v=c.v.half())),
            (TypeError, "page_table", dict(page_table=c.page_table.long())),
            (ValueError, "page_table", dict(page_table=c.page_table[0])),
            (ValueError, "shape", dict(len=c.len[:1])),
            (ValueError, "shape", dict(k=f8, v=f8, k_scale=torch.ones(3, 3))),
            (TypeError, "v_scale", dict(k=f8, v=f8, v_scale=torch.ones(3, 2).double()))):
        with pytest.raises(error, match=match):
            new(**kw)
    q, work = bf(2, 1, 8, 64), torch.zeros(64, dtype=torch.uint8)
    count = torch.ones(2, dtype=torch.int32)
    for error, match, call in (
            (ValueError, "shape", lambda: vd.vd_paged_attend(c, q, bf(2, 1, 4, 64), work)),
            (ValueError, "shape", lambda: vd.vd_paged_attend(c, bf(1, 1, 8, 64), q, work)),
            (TypeError, "q must", lambda: vd.vd_paged_attend(c, q.float(), q, work)),
            (TypeError, "workspace", lambda: vd.vd_paged_attend(c, q, bf(2, 1, 8, 64), work.int())),
            (ValueError, "dim", lambda: vd.vd_paged_attend(c, q[0], q, work)),
            (TypeError, "n_new", lambda: vd.vd_paged_attend(c, q, q, work, n_new=count.long())),
            (ValueError, "shape", lambda: vd.vd_paged_append(c, bf(2, 1, 12, 64), bf(2, 1, 9, 64))),
            (ValueError, "shape", lambda: vd.vd_paged_append(c, bf(2, 1, 12, 32), q)),
            (ValueError, "contiguous",
             lambda: vd.vd_paged_append(c, bf(2, 1, 12, 128)[..., :64], q)),
            (ValueError, "dimensions", lambda: vd.vd_paged_append(c, bf(2, 12, 64), q)),
            (ValueError, "shape", lambda: vd.vd_paged_advance(c, 1, count[:1]))):
        with pytest.raises(error, match=match):
            call()


def test_tensors_that_are_not_on_a_gpu_are_refused(lib):
    import paper_2609_23314_gb300 as vd
    c = vd.PagedCache.empty(2, 3, 2, 64, n_page=5, page_size=16, max_pages=4, device="cpu")
    q, work = bf(2, 1, 8, 64), torch.zeros(64, dtype=torch.uint8)
    cache = vd.Cache.empty(2, 3, 2, 16, 64, device="cpu")
    for call in (lambda: vd.vd_paged_attend(c, q, torch.empty_like(q), work),
                 lambda: vd.vd_paged_append(c, bf(2, 1, 12, 64), q),
                 lambda: vd.vd_paged_advance(c), lambda: vd.vd_paged_pack(c, cache),
                 lambda: vd.vd_paged_unpack(c, cache)):
        with pytest.raises(ValueError, match="must live on a CUDA device, got cpu"):
            call()
