"""Rows into and out of a paged cache (vd_paged_append, _pack, _unpack, _advance) against the
formulas in 64 bits.  Needs a GB300."""
from __future__ import annotations

import pytest
import torch

import paged_ref as ref
import paper_2609_23314_gb300 as vd
import q4_ref
from paged_ref import FILL, FP8, raw
from paper_2609_23314_gb300 import build

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    vd.load_library()
    torch.cuda.set_device(0)
    vd.vd_get_device_status()
    yield
    assert vd.vd_get_device_status() == 0


def projections(n, B, heads, d, rd, seed=0):
    g = torch.Generator().manual_seed(100 + seed)
    qkv = torch.randn((n, B, heads, d), generator=g).to(BF)
    qw, kw = (1 + 0.3 * torch.randn((2, d), generator=g)).to(BF)
    freq = (1e4 ** (-torch.arange(0, rd, 2).double() / rd)).float() if rd else None
    return qkv.cuda(), qw.cuda(), kw.cuda(), None if freq is None else freq.cuda()


def untouched(c, before, written):
    """All slots but the written ones ([(layer, page, slot)]) hold what they held."""
    for pool, old in zip((c.k, c.v), before):
        now = raw(pool).clone()
        for layer, page, slot in written:
            now[layer, page, :, slot] = old[layer, page, :, slot]
        assert torch.equal(now, old)


APPENDS = {
    # lens, B, n_kv, group, d, rd, page, options
    "one": ([5], 1, 2, 4, 128, 128, 16, dict()),
    "pages_end_inside": ([5, 0, 31], 40, 2, 3, 64, 64, 24, dict(news=[40, 17, 33])),
    "padded": ([9, 0, 100, 3], 7, 3, 1, 96, 48, 16, dict(news=[0, 7, 1, 3])),
    "interleaved_by_token": ([30, 2], 5, 2, 2, 80, 32, 8, dict(interleaved=True, by_token=True)),
    "one_buffer": ([3, 8], 9, 2, 2, 64, 64, 4, dict(one_buffer=True, layers=3, layer=1)),
    "pages_of_one": ([2, 1], 3, 1, 1, 256, 256, 1, dict()),
    "no_norm_no_rotation": ([7], 33, 1, 8, 16, 0, 5, dict(norm=False)),
    "many_tokens": ([0], 2500, 2, 1, 32, 16, 64, dict()),
    "far_positions": ([1, 2], 3, 2, 2, 128, 128, 16, dict(first=[2_000_000_000, 0])),
}


@pytest.mark.parametrize("dtype", [BF, FP8])
@pytest.mark.parametrize("name", APPENDS)
def test_append(name, dtype):
    lens, B, h, G, d, rd, page, o = APPENDS[name]
    n, layers, layer = len(lens), o.get("layers", 1), o.get("layer", 0)
    news = o.get("news", [B] * n)
    c = ref.cache(lens, layers, h, d, page, dtype, o.get("by_token", False), extra=B,
                  one_buffer=o.get("one_buffer", False))
    if name == "pages_of_one":
        c.k_scale = c.v_scale = None
        c = vd.PagedCache(c.k, c.v, c.page_table, c.len)
    qkv, qw, kw, freq = projections(n, B, h * (G + 2), d, rd)
    if not o.get("norm", True):
        qw = kw = None
    q = torch.full((n, B, h * G, d), FILL, dtype=BF, device="cuda")
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32).cuda()
    before = [raw(p).clone() for p in (c.k, c.v)]
    inter = o.get("interleaved", False)
    vd.vd_paged_append(c, qkv, q, layer=layer, q_weight=qw, k_weight=kw, eps=1e-6, inv_freq=freq,
                       pos_first_new=i32(o.get("first")), interleaved=inter,
                       n_new=i32(o.get("news")))
    assert c.len.tolist() == lens
    cpu = lambda t: None if t is None else t.cpu()
    x, written = qkv.cpu().double(), []
    for s in range(n):
        add = news[s]
        pos = (o["first"][s] if "first" in o else lens[s]) + torch.arange(add)
        y, size = q4_ref.norm_rope(x[s, :add, :h * G], cpu(qw), 1e-6, cpu(freq), pos, inter)
        err = (q[s, :add].cpu().double() - y).abs() - q4_ref.norm_rope_tolerance(y, size)
        assert bool((err <= 0).all()), f"queries of {s}: {err.max()} more than allowed"
        assert bool((q[s, add:] == FILL).all())
        c.len[s] = lens[s] + add
        k, v = (ref.rows_of(c, p, f, s, lens[s] + add, layer)[lens[s]:]
                for p, f in ((c.k, c.k_scale), (c.v, c.v_scale)))
        y, size = q4_ref.norm_rope(x[s, :add, h * G:h * (G + 1)], cpu(kw), 1e-6, cpu(freq), pos,
                                   inter)
        tol = q4_ref.norm_rope_tolerance(y, size)
        if dtype == FP8:  # fp32's part of the above, e4m3's half step, and that of its subnormals
            f = 1.0 if c.k_scale is None else c.k_scale[layer].cpu().double()[:, None]
            tol = 2.0 ** -17 * size + 2.0 ** -4 * y.abs() + 2.0 ** -10 * f
            y = torch.where(y.abs() > 448 * f, torch.sign(y) * 448 * f, y)
        err = (k - y).abs() - tol
        assert bool((err <= 0).all()), f"keys of {s}: {err.max()} more than allowed"
        want = qkv[s, :add, h * (G + 1):]
        if dtype == FP8:
            f = 1.0 if c.v_scale is None else c.v_scale[layer][None, :, None]
            want = (want.float() / f).clamp(-448, 448).to(FP8).float() * f
        assert torch.equal(v, want.cpu().float().double() if dtype == BF else v_exact(want, f))
        written += [(layer, int(c.page_table[s, t // page]), t % page)
                    for t in range(lens[s], lens[s] + add)]
    untouched(c, before, written)


def v_exact(rows, f):
    """Stored values times the scale in 64 bits, from their products in fp32."""
    if not torch.is_tensor(f):
        return rows.cpu().double()
    return ((rows / f).to(FP8).float().double() * f.double()).cpu()


@pytest.mark.parametrize("value,stored", [(float("nan"), 0x7f), (float("inf"), 0x7e),
                                          (-1e30, 0xfe), (-0.0, 0x80)])
def test_values_that_8_bits_do_not_hold(value, stored):
    c = ref.cache([0], 1, 1, 16, 4, FP8, extra=1, scales=False)
    qkv = torch.full((1, 1, 3, 16), value, dtype=BF, device="cuda")
    vd.vd_paged_append(c, qkv, torch.empty((1, 1, 1, 16), dtype=BF, device="cuda"))
    for pool in (c.k, c.v):
        assert raw(pool)[0, int(c.page_table[0, 0]), 0, 0].tolist() == [stored] * 16


def test_every_bf16_value_by_many_scales():
    """What is stored is the fp32 quotient rounded to e4m3, for every value and odd divisors."""
    g = torch.Generator().manual_seed(3)
    scales = torch.cat((2.0 ** (torch.rand(52, generator=g) * 40 - 20),
                        torch.tensor([1.0, 0.3, 3.0, 2.0 - 2.0 ** -23, 1.0 + 2.0 ** -23, 1e-30, 1e30,
                                      2.0 ** -126, 7.0 / 8, 2.0 ** -61, 2.0 ** 61, 1.0 / 448])))
    h = scales.numel()
    c = vd.PagedCache.empty(1, 1, h, 256, n_page=16, page_size=16, max_pages=16, dtype=FP8)
    c.page_table.copy_(torch.arange(16))
    c = vd.PagedCache(c.k, c.v, c.page_table, c.len, scales[None].cuda(), scales[None].cuda())
    rows = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF).view(256, 1, 256).cuda()
    qkv = rows.expand(256, 1 + 2 * h, 256).contiguous()[None]
    flat = vd.Cache.empty(1, 1, h, 256, 256)
    for pack in (False, True):
        if pack:  # the same by way of the contiguous layout
            flat.k.copy_(rows.transpose(0, 1).expand(h, 256, 256)[None, None])
            flat.v.copy_(flat.k)
            flat.len.fill_(256)
            raw(c.k).zero_(), raw(c.v).zero_()
            vd.vd_paged_pack(c, flat)
        else:
            vd.vd_paged_append(c, qkv, torch.empty((1, 256, 1, 256), dtype=BF, device="cuda"))
        want = rows[:, 0].float()[None] / scales.cuda()[:, None, None]
        want = raw(want.clamp(-448, 448).to(FP8))
        for pool in (c.k, c.v):
            got = raw(pool)[0].transpose(0, 1).reshape(h, 256, 256)
            nan = torch.isnan(rows[:, 0].float())[None].expand_as(got)
            assert torch.equal(got[~nan], want[~nan])
            assert bool(((got[nan] & 0x7f) == 0x7f).all())


@pytest.mark.parametrize("dtype", [BF, FP8])
@pytest.mark.parametrize("by_token,d,page", [(False, 128, 16), (True, 96, 24), (False, 16, 1),
                                             (True, 256, 7), (False, 64, 128)])
def test_out_of_pages_and_back(dtype, by_token, d, page):
    lens, L, h = [0, 1, 300, 23], 3, 2
    c = ref.cache(lens, L, h, d, page, dtype, by_token)
    flat = vd.Cache(*(torch.full((4, 2, h, 301, d), FILL, dtype=BF, device="cuda")
                      for _ in range(2)), torch.full((4,), 77, dtype=torch.int32, device="cuda"))
    vd.vd_paged_unpack(c, flat, layer0=1)
    assert flat.len.tolist() == lens
    for s, m in enumerate(lens):
        for pool, f, rows in ((c.k, c.k_scale, flat.k), (c.v, c.v_scale, flat.v)):
            for i in range(2):
                want = ref.rows_of(c, pool, f, s, m, 1 + i).transpose(0, 1)
                # the product with the scale in fp32, then bf16
                assert torch.equal(rows[s, i, :, :m].cpu(), want.float().to(BF))
            assert bool((rows[s, :, :, m:] == FILL).all())
    # into other pages, in another layout of slots; and the same bytes come back
    other = ref.cache([0] * 4, L, h, d, page, dtype, not by_token, extra=301, spare=3)
    other = vd.PagedCache(other.k, other.v, other.page_table, other.len, c.k_scale, c.v_scale)
    before = [raw(p).clone() for p in (other.k, other.v)]
    vd.vd_paged_pack(other, flat, layer0=1)
    assert other.len.tolist() == lens  # layers 1, 2 are the last ones
    for s, m in enumerate(lens):
        for layer in (1, 2):
            for a, b in ((other.k, c.k), (other.v, c.v)):
                assert torch.equal(ref.rows_of(other, a, None, s, m, layer),
                                   ref.rows_of(c, b, None, s, m, layer))
    other.len.zero_()
    vd.vd_paged_pack(other, flat, layer0=0)  # layers 0, 1: not the last one
    assert other.len.tolist() == [0] * 4
    written = []
    for s, m in enumerate(lens):
        for layer in (0, 1):  # under the scales of these layers
            for a, f, rows in ((other.k, c.k_scale, flat.k), (other.v, c.v_scale, flat.v)):
                want = rows[s, layer, :, :m].float()
                if f is not None:
                    want = (want / f[layer][:, None, None]).clamp(-448, 448)
                want = want.to(dtype).float().double().transpose(0, 1).cpu()
                assert torch.equal(ref.rows_of(other, a, None, s, m, layer), want)
        written += [(layer, int(other.page_table[s, t // page]), t % page)
                    for t in range(m) for layer in range(L)]
    untouched(other, before, written)


def test_advance():
    c = ref.cache([5, 0, 62], 1, 1, 16, 16, extra=2)  # 5 places of 16 a sequence
    new = torch.tensor([2, 0, 1], dtype=torch.int32).cuda()
    vd.vd_paged_advance(c, 2, new)
    assert c.len.tolist() == [7, 0, 63]
    vd.vd_paged_advance(c)
    vd.vd_paged_advance(c, 0)
    assert c.len.tolist() == [8, 1, 64]
    assert vd.vd_get_device_status() == 0
    vd.vd_paged_advance(c, 17)  # the third has room for 16
    assert c.len.tolist() == [25, 18, 64]
    assert vd.vd_get_device_status() == 7
    vd.vd_paged_advance(c, 1, new)  # 2 of 1
    assert c.len.tolist() == [25, 18, 65]
    assert vd.vd_get_device_status() == 7


def test_lengths_and_pages_out_of_range():
    lens = [3, 3, -1, 40]
    for bad, code in (("len", 7), ("page", 11)):
        c = ref.cache([3, 3, 3, 3], 1, 2, 32, 8, extra=6)
        c.len.copy_(torch.tensor(lens if bad == "len" else [3] * 4, dtype=torch.int32))
        news = torch.tensor([6, 7, 6, 6] if bad == "len" else [6] * 4, dtype=torch.int32).cuda()
        if bad == "page":
            c.page_table[1, 1], c.page_table[2, 0] = c.n_page, -5
        before = [raw(p).clone() for p in (c.k, c.v)]
        qkv, qw, kw, freq = projections(4, 6, 6, 32, 32)
        q = torch.full((4, 6, 2, 32), FILL, dtype=BF, device="cuda")
        vd.vd_paged_append(c, qkv, q, q_weight=qw, k_weight=kw, inv_freq=freq, n_new=news)
        assert vd.vd_get_device_status() == code
        ok = [s for s in range(4) if bad == "page" or s == 0]
        assert all(bool((q[s] != FILL).any()) == (s in ok) for s in range(4))
        at = [(s, t) for s in ok for t in range(3, 9)
              if 0 <= int(c.page_table[s, t // 8]) < c.n_page]
        untouched(c, before, [(0, int(c.page_table[s, t // 8]), t % 8) for s, t in at])
        flat = vd.Cache.empty(4, 1, 2, 39, 32)
        if bad == "len":
            c.len.copy_(torch.tensor([3, 40, -1, 25], dtype=torch.int32))  # 24 slots a sequence
        vd.vd_paged_unpack(c, flat)
        assert vd.vd_get_device_status() == code
        if bad == "len":
            assert flat.len.tolist() == [3, 0, 0, 0] and bool((flat.k[1:] == 0).all())
            flat.len.copy_(torch.tensor([3, 40, -1, 25], dtype=torch.int32))
            c.len.zero_()
            vd.vd_paged_pack(c, flat)
            assert vd.vd_get_device_status() == 7 and c.len.tolist() == [3, 0, 0, 0]


def test_on_a_stream_and_in_a_graph():
    c = ref.cache([4, 9], 1, 2, 64, 16, extra=8)
    qkv, qw, kw, freq = projections(2, 2, 8, 64, 64)
    q = torch.empty((2, 2, 4, 64), dtype=BF, device="cuda")
    flat = vd.Cache.empty(2, 1, 2, 32, 64)

    def step(stream=None):
        vd.vd_paged_append(c, qkv, q, q_weight=qw, k_weight=kw, inv_freq=freq, stream=stream)
        vd.vd_paged_advance(c, 2, stream=stream)
        vd.vd_paged_unpack(c, flat, stream=stream)
        vd.vd_paged_pack(c, flat, stream=stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    step(side)
    side.synchronize()
    assert c.len.tolist() == [6, 11]
    first = ref.rows_of(c, c.k, None, 0, 6, 0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert c.len.tolist() == [12, 17] == flat.len.tolist()
    assert torch.equal(first, ref.rows_of(c, c.k, None, 0, 6, 0))
    assert torch.equal(flat.v[1, 0, :, 15:17].transpose(0, 1), qkv[1, :, 6:])
