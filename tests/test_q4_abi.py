"""Calls on a 4-bit cache and vd_qkv_norm_rope refuse bad arguments before any launch
(CPU only), in C and in the binding."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2609_23314_gb300 import build, load_library
    build.build()
    return load_library()


def _q4(k=0x1000, v=0x2000, ks=0x3000, vs=0x4000, ln=0x5000, n_seq=1, n_layer=2, n_kv_head=2,
        head_dim=64, capacity=128):
    from paper_2609_23314_gb300 import _VdQ4Cache
    return ctypes.byref(_VdQ4Cache(k, v, ks, vs, ln, n_seq, n_layer, n_kv_head, head_dim,
                                   capacity))


def _cache(n_seq=1, n_layer=1, n_kv_head=2, head_dim=64, capacity=128, k=0x1000):
    from paper_2609_23314_gb300 import _VdCache
    return ctypes.byref(_VdCache(k, 0x2000, 0x3000, n_seq, n_layer, n_kv_head, head_dim,
                                 capacity))


@pytest.mark.parametrize("fields,code", [
    (dict(k=0), 1), (dict(vs=0), 1), (dict(ln=0), 1), (dict(n_layer=0), 1), (dict(capacity=0), 1),
    (dict(head_dim=0), 1), (dict(head_dim=48), 2), (dict(capacity=129), 2), (dict(k=0x1008), 2),
    (dict(vs=0x4001), 2), (dict(head_dim=288), 3), (dict(capacity=(1 << 30) + 8), 3), (dict(n_seq=1 << 20, n_layer=64), 3),
])
def test_bad_cache(lib, fields, code):
    c = _q4(**fields)
    assert lib.vd_q4_append(c, 0x100, 0x200, 4, None) == code
    assert lib.vd_q4_attend(c, 0, 0x100, 4, None, None, 1, 1.0, 0x200, None, None) == code
    assert lib.vd_q4_pack(c, 0, _cache(), None) == code
    assert lib.vd_q4_unpack(c, 0, _cache(), None) == code


def test_bad_arguments(lib):
    c = _q4()
    assert lib.vd_q4_append(None, 0x100, 0x200, 4, None) == 1
    assert lib.vd_q4_append(c, None, 0x200, 4, None) == 1
    assert lib.vd_q4_append(c, 0x100, 0x200, -1, None) == 1
    assert lib.vd_q4_append(c, 0x100, 0x200, 129, None) == 1
    assert lib.vd_q4_append(c, 0x108, 0x200, 4, None) == 2
    assert lib.vd_q4_append(c, 0x100, 0x200, 0, None) == 0       # nothing to do
    for f in (lib.vd_q4_pack, lib.vd_q4_unpack):
        assert f(c, 0, None, None) == 1
        for bad in (dict(n_seq=2), dict(n_kv_head=3), dict(head_dim=32), dict(n_layer=3),
                    dict(n_layer=0), dict(capacity=0), dict(k=0)):
            assert f(c, 0, _cache(**bad), None) == 1
        assert f(c, 2, _cache(), None) == 1                       # layers 2 .. 2 of 2
        assert f(c, -1, _cache(), None) == 1
        assert f(c, 0, _cache(k=0x1008), None) == 2

    def attend(layer=0, q=0x100, heads=4, kn=0x300, vn=0x400, B=1, scale=1.0, out=0x200):
        return lib.vd_q4_attend(c, layer, q, heads, kn, vn, B, scale, out, None, None)

    for bad in (dict(q=None), dict(out=None), dict(kn=None), dict(vn=None), dict(layer=2),
                dict(layer=-1), dict(heads=3), dict(heads=0), dict(B=0), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attend(**bad) == 1, bad
    for bad in (dict(q=0x108), dict(out=0x208), dict(kn=0x302), dict(vn=0x404)):
        assert attend(**bad) == 2, bad
    assert attend(B=1 << 28) == 3


def test_bad_projection_arguments(lib):
    def call(qkv=0x100, n_seq=1, B=1, n_q=4, n_kv=2, d=64, qw=None, kw=None, eps=1e-6, freq=0x40,
             rd=64, inter=0, pos=0x80, q=0x200, k=0x300, v=0x400, layer=0, n_layer=1):
        return lib.vd_qkv_norm_rope(qkv, n_seq, B, n_q, n_kv, d, qw, kw, eps, freq, rd, inter, pos,
                                    q, k, v, layer, n_layer, None)

    for bad in (dict(qkv=None), dict(q=None), dict(k=None), dict(v=None), dict(n_seq=0), dict(B=0),
                dict(n_q=0), dict(n_kv=0), dict(d=0), dict(layer=1), dict(layer=-1),
                dict(n_layer=0), dict(rd=-16), dict(rd=80), dict(freq=None), dict(pos=None),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=2.0)):
        assert call(**bad) == 1, bad
    for bad in (dict(d=68, rd=64), dict(qkv=0x108), dict(qw=0x8), dict(kw=0x2), dict(q=0x208),
                dict(k=0x302), dict(v=0x404)):
        assert call(**bad) == 2, bad
    for bad in (dict(d=264, rd=64), dict(rd=40), dict(rd=2)):
        assert call(**bad) == 3, bad


def test_the_binding_checks_its_tensors():
    import paper_2609_23314_gb300 as vd
    c = vd.Q4Cache.empty(2, 3, 2, 16, 64, device="cpu")
    assert c.units == 12 and c.unit_shape() == (2, 3, 2) and c.head_dim == 64
    with pytest.raises(ValueError, match="shape"):
        vd.Q4Cache(c.k, c.v, c.k_scale[..., :2].contiguous(), c.v_scale, c.len)
    with pytest.raises(TypeError):
        vd.Q4Cache(c.k.to(torch.int8), c.v, c.k_scale, c.v_scale, c.len)
    with pytest.raises(ValueError, match="contiguous"):
        vd.Q4Cache(c.k, c.v.transpose(0, 1).contiguous().transpose(0, 1), c.k_scale, c.v_scale,
                   c.len)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    q, new = bf(2, 1, 8, 64), bf(2, 3, 2, 1, 64)
    with pytest.raises(ValueError, match="shape"):
        vd.vd_q4_attend(c, q, bf(2, 1, 4, 64), new, new)
    with pytest.raises(TypeError):
        vd.vd_q4_attend(c, q.float(), q, new, new)
    with pytest.raises(ValueError, match="shape"):
        vd.vd_q4_attend(c, q, torch.empty_like(q), bf(2, 1, 2, 1, 64), new)
    with pytest.raises(ValueError, match="dim"):
        vd.vd_q4_attend(c, q[0], q, new, new)
    with pytest.raises(ValueError, match="shape"):
        vd.vd_q4_append(c, new, new, 2)
    qkv = bf(2, 1, 12, 64)
    with pytest.raises(ValueError, match="heads"):
        vd.vd_qkv_norm_rope(bf(2, 1, 11, 64), q, new, new)
    with pytest.raises(ValueError, match="shape"):
        vd.vd_qkv_norm_rope(qkv, q, bf(2, 3, 1, 1, 64), new)
    with pytest.raises(ValueError, match="contiguous"):
        vd.vd_qkv_norm_rope(bf(2, 1, 12, 128)[..., :64], q, new, new)


def test_tensors_of_another_device_are_refused(monkeypatch):
    """A call launches on the current device; tensors of another one do not reach it."""
    import paper_2609_23314_gb300 as vd
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 77 + i, raising=False)
    assert vd._launch_stream(torch.device("cuda", 0), None) == 77
    assert vd._launch_stream(torch.device("cpu"), None) is None
    with pytest.raises(ValueError, match="current device"):
        vd._launch_stream(torch.device("cuda", 1), None)
