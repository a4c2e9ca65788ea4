"""Every kernel that vd_q4_attend chooses from, and every cluster size, on the forms of a call
that its own choice brings to one or two of them: streaming with tiles of 8 and of 16 query
rows, and block.  Needs a GB300."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2609_23314_gb300 as vd
import q4_ref as ref
from paper_2609_23314_gb300 import build
from test_gpu_q4_attend import LENS, check, state

pytestmark = pytest.mark.gpu

KINDS = {"streaming8": "0", "streaming16": "1", "block": "2"}
# tiles of 16 rows exist where their sums fit the registers
HEAD_DIMS_16 = [32, 64, 96, 128]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    vd.load_library()
    torch.cuda.set_device(0)
    vd.vd_get_device_status()
    yield
    assert vd.vd_get_device_status() == 0


@pytest.fixture(params=list(KINDS))
def kind(request, monkeypatch):
    monkeypatch.setenv("VD_Q4_KERNEL", KINDS[request.param])
    return request.param


@pytest.fixture
def streaming16(monkeypatch):
    monkeypatch.setenv("VD_Q4_KERNEL", KINDS["streaming16"])


def attend(c, q, k_new, v_new, **kw):
    out = torch.full_like(q, 9.0)
    vd.vd_q4_attend(c, q, out, k_new, v_new, **kw)
    return out


@pytest.mark.usefixtures("streaming16")
@pytest.mark.parametrize("d", HEAD_DIMS_16)
@pytest.mark.parametrize("group,B", [(1, 1), (4, 1), (8, 2), (3, 5), (16, 1), (5, 3), (2, 40), (1, 200)])
def test_16_row_tiles(d, group, B):
    check(*state(LENS, 2, 2, group, d, B, 104), layer=1)


@pytest.mark.usefixtures("streaming16")
@pytest.mark.parametrize("d", HEAD_DIMS_16)
@pytest.mark.parametrize("B", [1, 4, 33])
def test_16_row_tiles_without_new_rows(d, B):
    c, q, _, _ = state([0, 1, 50, 33], 1, 2, 4, d, B, 56)
    check(c, q, None, None)


@pytest.mark.parametrize("d,group,B", [(128, 4, 4), (96, 3, 5), (64, 8, 2)])
@pytest.mark.usefixtures("streaming16")
def test_16_row_tiles_over_long_caches(d, group, B):
    check(*state([5003, 2048], 1, 1, group, d, B, 8192))


@pytest.mark.parametrize("cluster", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("d,B", [(64, 1), (96, 12), (128, 40), (256, 3)])
def test_cluster_sizes(kind, cluster, d, B, monkeypatch):
    """From a CTA for everything to 16 that share a unit, most of them without a token in the
    short sequences; new rows and none."""
    monkeypatch.setenv("VD_Q4_CLUSTER", str(cluster))
    c, q, k_new, v_new = state([0, 1, 33, 700, 130], 1, 2, 4, d, B, 704)
    check(c, q, k_new, v_new)
    check(c, q, None, None)


@pytest.mark.parametrize("cluster", [1, 4])
@pytest.mark.parametrize("bad", [-1, 41, 2 ** 31 - 1, -2 ** 31])
@pytest.mark.parametrize("B", [1, 40])
def test_lengths_out_of_range(kind, bad, B, cluster, monkeypatch):
    """No output for the sequence, the others' as without it, and the next call is whole."""
    monkeypatch.setenv("VD_Q4_CLUSTER", str(cluster))
    c, q, k_new, v_new = state([40, 40, 40], 1, 2, 4, 64, B, 40)
    whole = attend(c, q, k_new, v_new)
    for new in ((k_new, v_new), (None, None)):
        want = attend(c, q, *new)
        c.len[1] = bad
        lse = torch.full(q.shape[:-1], 9.0, device="cuda")
        out = attend(c, q, *new, lse_out=lse)
        assert vd.vd_get_device_status() == 7
        assert torch.equal(out[0], want[0]) and torch.equal(out[2], want[2])
        assert bool((out[1] == 9.0).all()) and bool((lse[1] == 9.0).all())
        c.len[1] = 40
    assert torch.equal(attend(c, q, k_new, v_new), whole)


@pytest.mark.parametrize("B", [1, 40])
@pytest.mark.parametrize("d", [64, 96, 256])
def test_groups_that_are_not_finite(kind, B, d):
    """A value group reads as NaN in its 16 dims of every query that sees it, a key group in
    the whole output and in lse; nothing else changes."""
    c, q, k_new, v_new = state([40, 40], 1, 2, 4, d, B, 40)
    clean = attend(c, q, k_new, v_new)
    c.v_scale[1, 0, 1, 17, 2 % (d // 16)] = 255
    got = attend(c, q, k_new, v_new)
    want = torch.zeros_like(got, dtype=torch.bool)
    want[1, :, 4:8, 32:48] = True
    assert torch.equal(torch.isnan(got), want) and torch.equal(got[~want], clean[~want])
    c.k_scale[0, 0, 0, 39, 0] = 255
    lse = torch.zeros(q.shape[:-1], device="cuda")
    got = attend(c, q, k_new, v_new, lse_out=lse)
    want[0, :, 0:4] = True
    assert torch.equal(torch.isnan(got), want) and torch.equal(got[~want], clean[~want])
    assert torch.equal(torch.isnan(lse), want.all(-1))


@pytest.mark.usefixtures("streaming16")
@pytest.mark.parametrize("B", [3, 40])
@pytest.mark.parametrize("d", [32, 96, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_16_row_tiles_later_tokens_do_not_reach_earlier_ones(B, d, value):
    c, q, k_new, v_new = state([40, 5], 1, 2, 4, d, B, 40)
    clean = attend(c, q, k_new, v_new)
    for which in (0, 1):
        new = [k_new.clone(), v_new.clone()]
        new[which][:, :, :, 2] = value
        out = attend(c, q, *new)
        # the same call on other rows: the weights of a tile may be rounded elsewhere, 2^-8 each
        assert bool((out[:, :2] - clean[:, :2]).abs().max() <= 2.0 ** -6 * clean.abs().max())
        if which:
            assert not bool(torch.isfinite(out[:, 2:]).any())
        elif math.isnan(value):
            assert bool(torch.isnan(out[:, 2:]).all())


@pytest.mark.parametrize("d", HEAD_DIMS_16)
@pytest.mark.parametrize("B", [3, 40])
@pytest.mark.usefixtures("streaming16")
def test_16_row_tiles_cold_warm_streams_and_graph(d, B):
    c, q, k_new, v_new = state([700, 90], 1, 2, 4, d, B, 704)
    flush = torch.empty(80 << 20, dtype=torch.int32, device="cuda")
    first, _ = check(c, q, k_new, v_new)
    for i in range(6):
        if i % 2:
            flush.fill_(i)
        assert torch.equal(attend(c, q, k_new, v_new), first), f"call {i}"
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [torch.empty_like(q) for _ in range(6)]
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
    assert all(torch.equal(o, first) for o in outs + [captured])


@pytest.mark.usefixtures("streaming16")
@pytest.mark.parametrize("B", [1, 40])
def test_16_row_tiles_a_wait_that_gives_up(B, monkeypatch):
    c, q, k_new, v_new = state([300, 290], 1, 2, 4, 128, B, 304)
    monkeypatch.setenv("VD_WAIT_LIMIT", "0")
    attend(c, q, k_new, v_new)
    torch.cuda.synchronize()
    assert vd.vd_get_device_status() == 5
    monkeypatch.delenv("VD_WAIT_LIMIT")
    check(c, q, k_new, v_new)


@pytest.mark.parametrize("d,B", [(128, 4), (128, 40)])
def test_offsets_beyond_32_bits(kind, d, B):
    """The last layer of a cache with more than 4 GB of codes in each tensor."""
    n_layer, cap = 68, 524288
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB of free device memory")
    c = vd.Q4Cache.empty(1, n_layer, 2, cap, d)
    assert c.k.numel() > 1 << 32
    small, q, k_new, v_new = state([1500], 1, 2, 4, d, B, 1504)
    for big, few in ((c.k, small.k), (c.v, small.v), (c.k_scale, small.k_scale),
                     (c.v_scale, small.v_scale)):
        big[0, n_layer - 1, :, :1504].copy_(few[0, 0])
    c.len.fill_(1500)
    new = [torch.zeros((1, n_layer) + tuple(x.shape[2:]), dtype=x.dtype, device="cuda")
           for x in (k_new, v_new)]
    for x, y in zip(new, (k_new, v_new)):
        x[:, n_layer - 1] = y[:, 0]
    check(c, q, new[0], new[1], layer=n_layer - 1)
