"""Rows into a 4-bit cache and back (vd_q4_append, vd_q4_pack, vd_q4_unpack): codes,
scales and values equal the 64-bit form bit for bit.  Needs a GB300."""
from __future__ import annotations

import pytest
import torch

import paper_2609_23314_gb300 as vd
import q4_ref as ref
from paper_2609_23314_gb300 import build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    vd.load_library()
    torch.cuda.set_device(0)
    vd.vd_get_device_status()
    yield
    assert vd.vd_get_device_status() == 0


def rows(shape, seed, kind="gauss"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g, dtype=torch.float64)
    if kind == "wide":      # magnitudes over the whole range of scales, and beyond
        x = x * torch.exp2(torch.randint(-24, 19, shape[:-1] + (1,), generator=g).double())
    elif kind == "ties":    # small integers: quotients on the code grid's edges, zero groups
        x = torch.randint(-12, 13, shape, generator=g).double()
        x[torch.rand(shape[:-1], generator=g) < 0.2] = 0.0
    return x.to(torch.bfloat16)


def q4_filled(n_seq, L, H, cap, d, seed=5):
    c = vd.Q4Cache.empty(n_seq, L, H, cap, d)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    return c


def snapshot(c):
    return [t.cpu().clone() for t in (c.k, c.v, c.k_scale, c.v_scale, c.len)]


@pytest.mark.parametrize("kind", ["gauss", "wide", "ties"])
@pytest.mark.parametrize("d,B,lens", [(32, 1, [0, 3, 31]), (64, 5, [0, 1, 9]), (96, 33, [7, 0, 6]),
                                      (128, 40, [0, 8, 1]), (160, 3, [5, 0, 2]),
                                      (192, 31, [1, 2, 3]), (224, 1, [39, 0, 0]),
                                      (256, 32, [8, 0, 5])])
def test_append(d, B, lens, kind):
    c = q4_filled(3, 2, 3, 48, d)
    c.len.copy_(torch.tensor(lens, dtype=torch.int32))
    kn, vn = (rows((3, 2, 3, B, d), s, kind) for s in (1, 2))
    want = snapshot(c)
    for s, n in enumerate(lens):
        for x, codes, scales in ((kn, want[0], want[2]), (vn, want[1], want[3])):
            codes[s, :, :, n:n + B], scales[s, :, :, n:n + B] = ref.quantise(x[s])
    want[4] += B
    vd.vd_q4_append(c, kn.cuda(), vn.cuda(), B)
    for got, w in zip(snapshot(c), want):
        assert torch.equal(got, w)


@pytest.mark.parametrize("kind", ["gauss", "wide", "ties"])
@pytest.mark.parametrize("d,lens,caps", [(32, [0, 24, 7], (24, 31)), (96, [33, 0, 17], (48, 33)),
                                         (128, [100, 64, 1], (104, 100)),
                                         (256, [5, 31, 0], (32, 57))])
def test_pack_and_unpack(d, lens, caps, kind):
    cap4, cap = caps
    cache = vd.Cache.empty(3, 2, 2, cap, d)
    for t, seed in ((cache.k, 3), (cache.v, 4)):
        t.copy_(rows(t.shape, seed, kind))
    cache.len.copy_(torch.tensor(lens, dtype=torch.int32))
    c = q4_filled(3, 2, 2, cap4, d)
    want = snapshot(c)
    for s, n in enumerate(lens):
        for x, codes, scales in ((cache.k, want[0], want[2]), (cache.v, want[1], want[3])):
            codes[s, :, :, :n], scales[s, :, :, :n] = ref.quantise(x[s, :, :, :n].cpu())
    want[4] = cache.len.cpu()
    vd.vd_q4_pack(c, cache)
    for got, w in zip(snapshot(c), want):
        assert torch.equal(got, w)
    back = vd.Cache.empty(3, 2, 2, cap + 3, d)
    back.k.fill_(7.0)
    back.v.fill_(7.0)
    vd.vd_q4_unpack(c, back)
    assert back.len.tolist() == lens
    for t, codes, scales in ((back.k, c.k, c.k_scale), (back.v, c.v, c.v_scale)):
        for s, n in enumerate(lens):
            v = ref.values(codes[s, :, :, :n].cpu(), scales[s, :, :, :n].cpu())
            assert torch.equal(t[s, :, :, :n].cpu().double(), v)
            assert bool((t[s, :, :, n:] == 7.0).all())
    if kind == "gauss":  # what a code stands for is stored as the same code
        again = q4_filled(3, 2, 2, cap4, d, seed=6)
        vd.vd_q4_pack(again, back)
        for s, n in enumerate(lens):
            for a, b in ((again.k, c.k), (again.v, c.v), (again.k_scale, c.k_scale),
                         (again.v_scale, c.v_scale)):
                assert torch.equal(a[s, :, :, :n], b[s, :, :, :n])


def test_buffers_at_16_byte_boundaries():
    """bf16 buffers that are 16-byte but not 32-byte aligned."""
    def shifted(t):
        flat = torch.zeros(t.numel() + 8, dtype=t.dtype, device="cuda")
        assert flat.data_ptr() % 32 == 0
        flat[8:].copy_(t.reshape(-1))
        return flat[8:].view(t.shape)

    kn, vn = (shifted(rows((2, 2, 3, 5, 96), s)) for s in (1, 2))
    c = q4_filled(2, 2, 3, 16, 96)
    vd.vd_q4_append(c, kn, vn, 5)
    for x, codes, scales in ((kn, c.k, c.k_scale), (vn, c.v, c.v_scale)):
        wc, ws = ref.quantise(x.cpu())
        assert torch.equal(codes[:, :, :, :5].cpu(), wc)
        assert torch.equal(scales[:, :, :, :5].cpu(), ws)
    cache = vd.Cache(shifted(torch.zeros(2, 2, 3, 16, 96, dtype=torch.bfloat16)),
                     shifted(torch.zeros(2, 2, 3, 16, 96, dtype=torch.bfloat16)), c.len.clone())
    vd.vd_q4_unpack(c, cache)
    for t, codes, scales in ((cache.k, c.k, c.k_scale), (cache.v, c.v, c.v_scale)):
        want = ref.values(codes[:, :, :, :5].cpu(), scales[:, :, :, :5].cpu())
        assert torch.equal(t[:, :, :, :5].cpu().double(), want)
    again = q4_filled(2, 2, 3, 16, 96, seed=9)
    cache.k.fill_(1.25)
    cache.v.fill_(-3.0)
    vd.vd_q4_pack(again, cache)
    wc, ws = ref.quantise(cache.v[:, :, :, :5].cpu())
    assert torch.equal(again.v[:, :, :, :5].cpu(), wc)
    assert torch.equal(again.v_scale[:, :, :, :5].cpu(), ws)


def test_layers_one_by_one():
    """A bf16 cache of one layer serves as the staging buffer of every layer in turn; the
    lengths follow the last layer."""
    L, lens = 3, [20, 9]
    c = q4_filled(2, L, 2, 24, 64)
    c.len.copy_(torch.tensor([1, 2], dtype=torch.int32))
    stage = vd.Cache.empty(2, 1, 2, 24, 64)
    data = [(rows((2, 1, 2, 24, 64), 10 + i), rows((2, 1, 2, 24, 64), 20 + i)) for i in range(L)]
    for i, (k, v) in enumerate(data):
        stage.k.copy_(k)
        stage.v.copy_(v)
        stage.len.copy_(torch.tensor(lens, dtype=torch.int32))
        vd.vd_q4_pack(c, stage, layer0=i)
        assert c.len.tolist() == (lens if i == L - 1 else [1, 2])
    for i, (k, _) in enumerate(data):
        stage.len.zero_()
        vd.vd_q4_unpack(c, stage, layer0=i)
        assert stage.len.tolist() == lens
        for s, n in enumerate(lens):
            want = ref.values(*ref.quantise(k[s, :, :, :n]))
            assert torch.equal(stage.k[s, :, :, :n].cpu().double(), want)


def test_groups_that_are_not_finite():
    kn = rows((1, 1, 1, 4, 64), 1)
    kn[0, 0, 0, 1, 17] = float("inf")
    kn[0, 0, 0, 2, 3] = float("nan")
    kn[0, 0, 0, 3, 63] = -float("inf")
    c = q4_filled(1, 1, 1, 8, 64)
    c.len.zero_()
    vd.vd_q4_append(c, kn.cuda(), rows((1, 1, 1, 4, 64), 2).cuda(), 4)
    assert vd.vd_get_device_status() == 4
    codes, scales = ref.quantise(kn[0, 0, 0])
    assert torch.equal(c.k_scale[0, 0, 0, :4].cpu(), scales)
    assert torch.equal(c.k[0, 0, 0, :4].cpu(), codes)
    back = vd.Cache.empty(1, 1, 1, 8, 64)
    vd.vd_q4_unpack(c, back)
    nan = torch.isnan(back.k[0, 0, 0, :4].cpu()).unflatten(-1, (-1, 16))
    assert torch.equal(nan.all(-1), scales == 255) and torch.equal(nan.any(-1), scales == 255)
    assert vd.vd_get_device_status() == 0


def test_lengths_out_of_range_leave_the_sequence_alone():
    for bad in (-1, 17, 24, 2 ** 30):
        c = q4_filled(3, 2, 2, 24, 32)
        c.len.copy_(torch.tensor([0, bad, 16], dtype=torch.int32))
        before = snapshot(c)
        kn = rows((3, 2, 2, 8, 32), 1).cuda()
        vd.vd_q4_append(c, kn, kn, 8)
        assert vd.vd_get_device_status() == 7
        after = snapshot(c)
        for a, b in zip(after[:4], before[:4]):
            assert torch.equal(a[1], b[1]) and not torch.equal(a[0], b[0])
        assert after[4].tolist() == [8, bad, 24]
    for pack in (True, False):
        for bad in (-5, 25):
            c = q4_filled(2, 1, 2, 24, 32)
            cache = vd.Cache.empty(2, 1, 2, 30, 32)
            cache.len.fill_(3)
            c.len.fill_(3)
            (cache if pack else c).len[0] = bad
            before = snapshot(c) + [cache.k.cpu(), cache.len.cpu()]
            (vd.vd_q4_pack if pack else vd.vd_q4_unpack)(*((c, cache)))
            assert vd.vd_get_device_status() == 7
            after = snapshot(c) + [cache.k.cpu(), cache.len.cpu()]
            for a, b in zip(after, before):
                assert torch.equal(a[0], b[0])
            # a longer bf16 cache's length that the 4-bit one cannot hold
    c, cache = q4_filled(1, 1, 1, 8, 32), vd.Cache.empty(1, 1, 1, 30, 32)
    cache.len.fill_(9)
    vd.vd_q4_pack(c, cache)
    assert vd.vd_get_device_status() == 7


def test_rows_beyond_32_bit_offsets():
    """Units whose rows start past 4 GB of codes."""
    n_layer, cap, d = 36, 524288, 256
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB of free device memory")
    c = vd.Q4Cache.empty(1, n_layer, 1, cap, d)  # 2 x 4.8 GB codes
    c.len.fill_(cap - 3)
    kn, vn = rows((1, n_layer, 1, 3, d), 1), rows((1, n_layer, 1, 3, d), 2)
    vd.vd_q4_append(c, kn.cuda(), vn.cuda(), 3)
    for x, codes, scales in ((kn, c.k, c.k_scale), (vn, c.v, c.v_scale)):
        wc, ws = ref.quantise(x)
        assert torch.equal(codes[..., cap - 3:, :].cpu(), wc)
        assert torch.equal(scales[..., cap - 3:, :].cpu(), ws)
        assert not bool(codes[..., :cap - 3, :].any())
