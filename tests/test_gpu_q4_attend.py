"""Attention over a 4-bit cache and the new rows (vd_q4_attend) against its formula in
64 bits.  Needs a GB300."""
from __future__ import annotations

import math

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


@pytest.fixture(params=["automatic", "streaming", "block"])
def route(request, monkeypatch):
    """Runs a test with the kernel that the library picks, and with each of the two."""
    if request.param != "automatic":
        monkeypatch.setenv("VD_Q4_KERNEL", "0" if request.param == "streaming" else "2")


def state(lens, n_layer, n_kv, group, d, B, cap, seed=0, spread=1.0):
    """A cache whose slots behind the lengths hold random codes with NaN scales, and
    new rows and queries."""
    g = torch.Generator().manual_seed(1000 + seed)
    n = len(lens)
    c = vd.Q4Cache.empty(n, n_layer, n_kv, cap, d)
    for codes, scales in ((c.k, c.k_scale), (c.v, c.v_scale)):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8))
        scales.fill_(255)
        for s, m in enumerate(lens):
            x = torch.randn((n_layer, n_kv, m, d), generator=g) * spread
            x = (x + torch.randn(d, generator=g)).to(torch.bfloat16)
            a, b = ref.quantise(x)
            codes[s, :, :, :m].copy_(a)
            scales[s, :, :, :m].copy_(b)
    c.len.copy_(torch.tensor(lens, dtype=torch.int32))
    k_new, v_new = (torch.randn((n, n_layer, n_kv, B, d), generator=g).to(torch.bfloat16).cuda()
                    for _ in range(2))
    q = (torch.randn((n, B, n_kv * group, d), generator=g) * spread).to(torch.bfloat16).cuda()
    return c, q, k_new, v_new


def expected(c, q, k_new, v_new, layer, scale):
    n, B, heads, d = q.shape
    group = heads // c.n_kv_head
    lens = c.len.tolist()
    parts = {f: torch.zeros((n, B, heads) + t, dtype=torch.float64)
             for f, t in (("out", (d,)), ("lse", ()), ("t_out", (d,)), ("t_lse", ()))}
    for s in range(n):
        for h in range(c.n_kv_head):
            m = lens[s]
            ks, vs = (ref.values(x[s, layer, h, :m].cpu(), y[s, layer, h, :m].cpu())
                      for x, y in ((c.k, c.k_scale), (c.v, c.v_scale)))
            new = [None, None] if k_new is None else \
                [x[s, layer, h].cpu().double() for x in (k_new, v_new)]
            hs = slice(h * group, (h + 1) * group)
            got = ref.attend(q[s, :, hs].cpu().double(), ks, vs, new[0], new[1], scale)
            t = ref.attend_tolerance(*got, m + B, d)
            for f, x in zip(("out", "lse", "t_out", "t_lse"), got[:2] + t):
                parts[f][s, :, hs] = x
    return parts


def check(c, q, k_new, v_new, layer=0, scale=None):
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    out = torch.full_like(q, 9.0)
    lse = torch.full(q.shape[:-1], 9.0, device="cuda")
    vd.vd_q4_attend(c, q, out, k_new, v_new, layer, scale, lse)
    want = expected(c, q, k_new, v_new, layer, scale)
    o, e = out.cpu().double(), lse.cpu().double()
    none = torch.isneginf(want["lse"])
    assert torch.equal(torch.isneginf(e), none)
    assert bool((o[none] == 0).all())
    err = (o - want["out"]).abs() - want["t_out"]
    assert bool((err <= 0).all()), f"out off by {(o - want['out']).abs().max()}, {err.max()} more " \
                                   f"than allowed"
    err = ((e - want["lse"]).abs() - want["t_lse"])[~none]
    assert bool((err <= 0).all()), f"lse {err.max()} more than allowed"
    return out, lse


LENS = [0, 1, 7, 8, 15, 16, 17, 31, 32, 33, 64, 100]


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("group,B", [(1, 1), (4, 1), (8, 1), (3, 2), (5, 3), (16, 1)])
def test_head_dims_and_groups(d, group, B):
    check(*state(LENS, 2, 2, group, d, B, 104), layer=1)


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("group,B", [(1, 17), (4, 16), (4, 40), (2, 128), (7, 31), (1, 200)])
def test_many_new_tokens(d, group, B):
    check(*state([0, 1, 90, 300], 1, 2, group, d, B, 304))


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("d,group,B", [(128, 4, 1), (96, 3, 1), (64, 8, 2), (256, 2, 1),
                                       (128, 4, 32), (192, 1, 1)])
def test_long_caches(d, group, B):
    """Few units, so that a cluster shares one; a length that fills no stage."""
    check(*state([5003, 2048], 1, 1, group, d, B, 8192))


@pytest.mark.parametrize("B", [1, 24])
@pytest.mark.parametrize("n_seq,n_kv", [(40, 3), (3, 40), (2, 5)])
def test_many_units(n_seq, n_kv, B):
    check(*state([(37 * s) % 257 for s in range(n_seq)], 1, n_kv, 4, 64, B, 264))


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("B", [1, 5, 33])
def test_without_new_rows(d, B):
    """Every token sees the cached rows alone; where there are none, zeros."""
    c, q, _, _ = state([0, 1, 50, 33], 1, 2, 4, d, B, 56)
    check(c, q, None, None)


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("spread,scale", [(30.0, 1.0), (1e-3, 1.0), (1.0, 5.0), (200.0, 0.5)])
@pytest.mark.parametrize("B", [1, 40])
def test_large_and_small_scores(spread, scale, B):
    check(*state([70, 130], 1, 2, 4, 128, B, 136, spread=spread), scale=scale)


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("factor", [1e-30, 1e-36, 1e30])
@pytest.mark.parametrize("B", [1, 40])
def test_queries_of_any_size(factor, B):
    """Queries far outside fp16's range, with the scale that makes up for them."""
    c, q, k_new, v_new = state([70, 33], 1, 2, 4, 128, B, 72)
    check(c, (q.double() * factor).to(torch.bfloat16), k_new, v_new, scale=0.08 / factor)


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("B", [2, 40])
def test_new_keys_near_the_largest_number(B):
    """Scores whose products with small queries are ordinary numbers."""
    c, q, k_new, v_new = state([0, 33], 1, 2, 4, 128, B, 40)
    check(c, (q.double() * 1e-37).to(torch.bfloat16),
          (k_new.double() * 5e37).to(torch.bfloat16), v_new, scale=0.02)


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("B", [2, 40])
def test_queries_near_the_largest_number(B):
    c, q, k_new, v_new = state([70, 33], 1, 2, 4, 128, B, 72)
    check(c, (q.double() * 1e36).to(torch.bfloat16), k_new, v_new, scale=8e-38)


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("B", [3, 40])
@pytest.mark.parametrize("d", [96, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_later_tokens_do_not_reach_earlier_ones(B, d, value):
    """Non-finite new rows of token 2 leave tokens 0 and 1 as they are; the tokens that
    see them become non-finite."""
    c, q, k_new, v_new = state([40, 5], 1, 2, 4, d, B, 40)
    clean, _ = check(c, q, k_new, v_new)
    # both results are within the tolerance of the same tokens' exact ones
    tol = 2 * expected(c, q, k_new, v_new, 0, d ** -0.5)["t_out"][:, :2]
    for tensors in ((k_new, None), (None, v_new)):
        kn, vn = k_new.clone(), v_new.clone()
        for t, x in zip(tensors, (kn, vn)):
            if t is not None:
                x[:, :, :, 2] = value
        out = torch.full_like(q, 9.0)
        vd.vd_q4_attend(c, q, out, kn, vn)
        assert bool(((out[:, :2].double() - clean[:, :2].double()).abs().cpu() <= tol).all())
        if tensors[1] is not None:
            assert not bool(torch.isfinite(out[:, 2:]).any())
        elif math.isnan(value):
            assert bool(torch.isnan(out[:, 2:]).all())


def test_a_group_that_is_not_finite_reads_as_nan():
    c, q, k_new, v_new = state([40, 40], 1, 2, 4, 64, 2, 40)
    out = torch.empty_like(q)
    vd.vd_q4_attend(c, q, out, k_new, v_new)
    c.v_scale[1, 0, 1, 17, 2] = 255  # values 32 .. 47 of one token of one head
    got = torch.empty_like(q)
    vd.vd_q4_attend(c, q, got, k_new, v_new)
    nan = torch.isnan(got)
    want = torch.zeros_like(nan)
    want[1, :, 4:8, 32:48] = True
    assert torch.equal(nan, want)
    assert torch.equal(got[~want], out[~want])


def test_lengths_out_of_range_give_no_output():
    for bad in (-1, 41, 2 ** 31 - 1):
        for B in (1, 40):
            c, q, k_new, v_new = state([40, 40, 40], 1, 2, 4, 64, B, 40)
            whole = torch.empty_like(q)
            vd.vd_q4_attend(c, q, whole, k_new, v_new)
            c.len[1] = bad
            out = torch.full_like(q, 9.0)
            vd.vd_q4_attend(c, q, out, k_new, v_new)
            assert vd.vd_get_device_status() == 7
            assert torch.equal(out[0], whole[0]) and torch.equal(out[2], whole[2])
            assert bool((out[1] == 9.0).all())


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("B,group", [(1, 4), (40, 4)])
def test_same_call_same_bytes(B, group):
    """On the current stream, on another one, from two streams at once, captured and
    replayed: the same bytes."""
    c, q, k_new, v_new = state([700, 90], 1, 2, group, 128, B, 704)
    first = torch.empty_like(q)
    vd.vd_q4_attend(c, q, first, k_new, v_new)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [torch.empty_like(q) for _ in range(8)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        vd.vd_q4_attend(c, q, o, k_new, v_new, stream=streams[i % 2])
    torch.cuda.synchronize()
    graph, captured = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(graph):
        vd.vd_q4_attend(c, q, captured, k_new, v_new)
        vd.vd_q4_attend(c, q, captured, k_new, v_new)
    graph.replay()
    torch.cuda.synchronize()
    for o in outs + [captured]:
        assert torch.equal(o, first)


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("d", [64, 128, 192, 256])
@pytest.mark.parametrize("B,new", [(2, True), (40, True), (40, False)])
def test_cold_and_warm_reads_give_the_same_bytes(d, B, new):
    """The parts of a CTA run at different speeds when their rows come from memory and
    when they come from the L2 cache; the results have to be the same."""
    c, q, k_new, v_new = state([300, 90], 1, 2, 4, d, B, 304)
    if not new:
        k_new = v_new = None
    flush = torch.empty(80 << 20, dtype=torch.int32, device="cuda")
    first, _ = check(c, q, k_new, v_new)
    for i in range(12):
        if i % 2:
            flush.fill_(i)
        out = torch.full_like(q, 9.0)
        vd.vd_q4_attend(c, q, out, k_new, v_new)
        assert torch.equal(out, first), f"call {i}"


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("B", [1, 40])
def test_a_wait_that_gives_up(B, monkeypatch):
    """With no polls left every copy counts as late: the call returns, the status says
    so, and the next call is whole."""
    c, q, k_new, v_new = state([300, 290], 1, 2, 4, 128, B, 304)
    out = torch.empty_like(q)
    monkeypatch.setenv("VD_WAIT_LIMIT", "0")
    vd.vd_q4_attend(c, q, out, k_new, v_new)
    torch.cuda.synchronize()
    assert vd.vd_get_device_status() == 5
    monkeypatch.delenv("VD_WAIT_LIMIT")
    check(c, q, k_new, v_new)


def test_offsets_beyond_32_bits():
    """The last layer of a cache with more than 4 GB of codes in each tensor."""
    n_layer, cap, d = 36, 524288, 256
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB of free device memory")
    c = vd.Q4Cache.empty(1, n_layer, 1, cap, d)
    small, q, k_new, v_new = state([1500], 1, 1, 4, d, 1, 1504)
    for big, few in ((c.k, small.k), (c.v, small.v), (c.k_scale, small.k_scale),
                     (c.v_scale, small.v_scale)):
        big[0, n_layer - 1, 0, :1504].copy_(few[0, 0, 0])
    c.len.fill_(1500)
    new = [torch.zeros((1, n_layer) + tuple(x.shape[2:]), dtype=x.dtype, device="cuda")
           for x in (k_new, v_new)]
    for x, y in zip(new, (k_new, v_new)):
        x[:, n_layer - 1] = y[:, 0]
    check(c, q, new[0], new[1], layer=n_layer - 1)
