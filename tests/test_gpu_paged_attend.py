"""Attention over a paged cache (vd_paged_attend) against the definition in 64 bits.  Needs a
GB300."""
from __future__ import annotations

import threading

import pytest
import torch

import paged_ref as ref
import paper_2609_23314_gb300 as vd
from paged_ref import FILL, FP8, check_attend, raw
from paper_2609_23314_gb300 import build

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("route")]
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    vd.load_library()
    torch.cuda.set_device(0)
    vd.vd_get_device_status()
    yield
    assert vd.vd_get_device_status() == 0


ROUTES = {"automatic": {}, "pieces": dict(VD_PAGED_CLUSTER="1"),
          "tiles_of_16": dict(VD_PAGED_KERNEL="1", VD_PAGED_CLUSTER="1"),
          "block": dict(VD_PAGED_KERNEL="2"),
          "clusters_of_3": dict(VD_PAGED_KERNEL="0", VD_PAGED_CLUSTER="3"),
          "block_clusters_of_7": dict(VD_PAGED_KERNEL="2", VD_PAGED_CLUSTER="7"),
          "block_alone": dict(VD_PAGED_KERNEL="2", VD_PAGED_CLUSTER="1")}


@pytest.fixture(params=ROUTES)
def route(request, monkeypatch):
    """The kernel and plan that the library takes by the sizes, which for few units is a cluster for
    each; pieces of the line and the join; the other kernels for all sizes."""
    for name, value in ROUTES[request.param].items():
        monkeypatch.setenv(name, value)


def queries(n, B, n_q, d, seed=0, size=1.0):
    g = torch.Generator().manual_seed(1000 + seed)
    return (size * torch.randn((n, B, n_q, d), generator=g)).to(BF).cuda()


CASES = {
    # lens (with the new tokens' rows behind them), B, n_kv, group, d, page, options
    "one_token": ([100], 1, 2, 4, 128, 16, dict()),
    "first_token": ([0], 1, 2, 4, 128, 16, dict()),
    "stage_ends": ([15, 16, 17, 31, 32, 33], 1, 1, 2, 64, 16, dict()),
    "many_short": ([(7 * i) % 50 for i in range(300)], 1, 1, 1, 64, 16, dict()),
    "skew": ([3000, 0, 1, 900, 2], 1, 1, 8, 128, 16, dict()),
    "draft": ([500, 0, 17], 4, 3, 5, 96, 24, dict(news=[4, 0, 3])),
    "rows_16": ([250, 40], 4, 2, 4, 128, 16, dict()),
    "rows_17_to_33": ([130, 0, 64], 11, 1, 3, 80, 32, dict(news=[11, 6, 8])),
    "block": ([200], 70, 2, 4, 128, 128, dict()),
    "block_ragged": ([65, 0, 300], 50, 1, 3, 64, 8, dict(news=[50, 49, 7], by_token=True)),
    "prompt": ([0], 150, 1, 2, 128, 16, dict()),
    "cached_alone": ([70, 0, 5], 3, 2, 2, 64, 16, dict(causal=False)),
    "cached_alone_padded": ([70, 0, 5], 20, 1, 2, 64, 16, dict(causal=False, news=[0, 20, 3])),
    "pages_of_one": ([37, 5], 2, 2, 1, 32, 1, dict()),
    "pages_of_five": ([37, 5], 2, 2, 1, 32, 5, dict(by_token=True)),
    "head_dim_16": ([40], 1, 1, 1, 16, 16, dict()),
    "head_dim_192": ([340, 20], 2, 2, 3, 192, 16, dict()),
    "head_dim_256": ([340, 20], 3, 1, 8, 256, 64, dict()),
    "head_dim_224": ([100], 9, 1, 4, 224, 16, dict()),
    "head_dim_160_one_buffer": ([333], 1, 2, 7, 160, 16, dict(one_buffer=True)),
    "layer": ([50, 60], 1, 2, 2, 128, 16, dict(layers=3, layer=1)),
    "group_of_13": ([50, 300], 1, 2, 13, 128, 16, dict()),
    "steep": ([700], 1, 2, 4, 128, 16, dict(size=30.0)),
    "steep_block": ([300], 40, 1, 4, 64, 16, dict(size=30.0)),
    "scale": ([60], 2, 1, 4, 64, 16, dict(scale=0.01)),
}


def case(name, dtype):
    lens, B, h, G, d, page, o = CASES[name]
    c = ref.cache(lens, o.get("layers", 1), h, d, page, dtype, o.get("by_token", False), extra=0,
                  one_buffer=o.get("one_buffer", False))
    # with the new tokens' rows: a cache whose lens are taken back
    news = o.get("news", [B] * len(lens))
    if o.get("causal", True):
        c = ref.cache([m + b for m, b in zip(lens, news)], o.get("layers", 1), h, d, page, dtype,
                      o.get("by_token", False), one_buffer=o.get("one_buffer", False))
        c.len.copy_(torch.tensor(lens, dtype=torch.int32))
    q = queries(len(lens), B, h * G, d, size=o.get("size", 1.0))
    kw = {k: o[k] for k in ("layer", "causal", "scale") if k in o}
    return c, q, dict(kw, n_new=o.get("news"))


@pytest.mark.parametrize("dtype", [BF, FP8])
@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(name, dtype):
    c, q, kw = case(name, dtype)
    check_attend(c, q, **kw)


@pytest.mark.parametrize("d", range(8, 257, 8))
def test_every_head_dim(d):
    for dtype in (BF, FP8) if d % 16 == 0 else (BF,):
        for B in (1, 6, 18):
            c = ref.cache([70 + B, 19 + B], 1, 1, d, 16, dtype)
            c.len -= B
            check_attend(c, queries(2, B, 3, d), n_new=[B, B - 1])


@pytest.mark.parametrize("dtype", [BF, FP8])
def test_without_scales_and_without_log_sums(dtype):
    c = ref.cache([90, 33], 1, 2, 64, 16, dtype, scales=False)
    c.len -= 1
    check_attend(c, queries(2, 1, 4, 64, size=0.02 if dtype == FP8 else 1.0), lse=False)


def test_long_sequences():
    """More stages than CTAs take at once, and units that several CTAs share."""
    c = ref.cache([40001, 7, 9000], 1, 2, 64, 64)
    c.len -= 1
    check_attend(c, queries(3, 1, 4, 64))


@pytest.mark.parametrize("G", [3, 8, 16])
def test_one_long_sequence_among_short_ones(G):
    """Units of few parts and one of many in a call; the long one first, in the middle and last."""
    for at, length in ((0, 1500), (50, 3100), (50, 6000), (99, 12000), (50, 40000)):
        lens = [(i * 61) % 300 for i in range(100)]
        lens[at] = length
        c = ref.cache([m + 1 for m in lens], 1, 1, 64, 16)
        c.len -= 1
        check_attend(c, queries(100, 1, G, 64))


def test_more_sequences_than_threads():
    lens = [(i * 37) % 23 for i in range(700)]
    c = ref.cache([m + 2 for m in lens], 1, 2, 32, 8)
    c.len -= 2
    check_attend(c, queries(700, 2, 2, 32), n_new=[i % 3 for i in range(700)])


def test_offsets_beyond_32_bits():
    """A pool of 9 GB: the pages of the sequence lie at its end."""
    P, page, d = 70_000, 256, 128
    pools = [torch.zeros((2, P, 1, page, d), dtype=BF, device="cuda") for _ in range(2)]
    small = ref.cache([600], 1, 1, d, page)
    table = torch.tensor([[P - 1, 0, P - 2]], dtype=torch.int32).cuda()
    for pool, src in zip(pools, (small.k, small.v)):
        pool[1, table[0].long()] = src[0, small.page_table[0, :3].long()]
    c = vd.PagedCache(pools[0], pools[1], table, small.len)
    c.len -= 1
    check_attend(c, queries(1, 1, 4, d), layer=1)


@pytest.mark.parametrize("dtype", [BF, FP8])
@pytest.mark.parametrize("B,G,d", [(1, 4, 128), (6, 3, 64), (40, 4, 128)])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_what_a_token_does_not_see_does_not_reach_it(B, G, d, dtype, what):
    """Rows behind a token hold NaN or infinity, among them those of later new tokens; so do the
    slots behind the last one."""
    n = 45
    c = ref.cache([n + B], 1, 1, d, 16, dtype)
    c.len -= B
    value = {"nan": float("nan"), "inf": float("inf")}[what]
    if dtype == FP8 and what == "inf":
        value = -float("nan")
    bits = torch.full((1,), value).to(dtype)
    last = (n + B - 1) // 16
    for pool, slots in ((c.k, range(n + B, 16 * (last + 1))), (c.v, range(n + B - B // 2, 16 * (last + 1)))):
        for t in slots:
            raw(pool)[0, int(c.page_table[0, t // 16]), :, t % 16] = raw(bits).cuda()[0]
    out, _ = check_attend(c, queries(1, B, G, d))
    assert bool(torch.isfinite(out[0, :B - B // 2]).all())
    if B > 1:
        assert not bool(torch.isfinite(out[0, -1]).any())


@pytest.mark.parametrize("dtype", [BF, FP8])
@pytest.mark.parametrize("B", [1, 5, 40])
def test_nan_keys(B, dtype):
    """A NaN in a key: NaN for the tokens that see it, nothing for the others."""
    n = 33
    c = ref.cache([n + B], 1, 1, 64, 16, dtype)
    c.len -= B
    t = n + B - 1  # the last token's own row
    bits = raw(torch.full((1,), float("nan")).to(dtype)).cuda()[0]
    raw(c.k)[0, int(c.page_table[0, t // 16]), 0, t % 16, 3] = bits
    out, lse = check_attend(c, queries(1, B, 2, 64))
    assert bool(torch.isnan(out[0, -1]).all()) and bool(torch.isnan(lse[0, -1]).all())
    raw(c.k)[:] = bits  # every score
    out, lse = check_attend(c, queries(1, B, 2, 64))
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())


@pytest.mark.parametrize("B", [1, 40])
def test_scores_of_minus_infinity(B):
    c = ref.cache([50 + B], 1, 1, 64, 16)
    c.len -= B
    q = queries(1, B, 2, 64).abs() + 0.1
    c.k[..., 0] = -float("inf")
    out, lse = check_attend(c, q)
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())
    # all but one
    t = 20
    c.k[0, int(c.page_table[0, t // 16]), 0, t % 16, 0] = 0.5
    out, lse = check_attend(c, q)
    v = c.v[0, int(c.page_table[0, t // 16]), 0, t % 16]
    assert torch.equal(out, v.expand_as(out))


@pytest.mark.parametrize("name", ["skew", "block", "draft"])
def test_the_same_bits(name):
    c, q, kw = case(name, BF)
    first = check_attend(c, q, **kw)
    again = check_attend(c, q, **kw)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_shared_pages():
    """Two sequences over the same first pages."""
    c = ref.cache([64, 80], 1, 2, 64, 16)
    c.page_table[1, :3] = c.page_table[0, :3]
    c.len -= 1
    check_attend(c, queries(2, 1, 4, 64))


def test_lengths_and_pages_out_of_range():
    for B, causal in ((1, True), (40, True), (3, False)):
        c = ref.cache([100] * 5, 1, 2, 64, 16)
        cap = c.page_size * c.max_pages
        c.len.copy_(torch.tensor([50, -1, cap + 1, 50, cap - B + 1 if causal else 50]))
        news = torch.tensor([B, B, B, B + 1, B], dtype=torch.int32).cuda()
        q, out = queries(5, B, 4, 64), torch.full((5, B, 4, 64), FILL, dtype=BF, device="cuda")
        work = torch.empty(vd.vd_paged_attend_workspace(c, 4, B), dtype=torch.uint8, device="cuda")
        vd.vd_paged_attend(c, q, out, work, causal=causal, n_new=news)
        assert vd.vd_get_device_status() == 7
        wrote = [bool((out[s] != FILL).any()) for s in range(5)]
        assert wrote == [True, False, False, False, not causal]
        # a page that is not one: the others' outputs are right
        c = ref.cache([100] * 3, 1, 2, 64, 16)
        c.len -= B
        c.page_table[1, 2] = c.n_page
        got = torch.empty((3, B, 4, 64), dtype=BF, device="cuda")
        vd.vd_paged_attend(c, q[:3].contiguous(), got, work, causal=causal)
        assert vd.vd_get_device_status() == 11
        c.page_table[1, 2] = 0
        fine, _ = check_attend(c, q[:3].contiguous(), causal=causal)
        assert torch.equal(got[0], fine[0]) and torch.equal(got[2], fine[2])


def test_a_workspace_that_is_too_small_is_refused():
    c = ref.cache([20], 1, 1, 64, 16)
    q = queries(1, 1, 2, 64)
    size = vd.vd_paged_attend_workspace(c, 2, 1)
    with pytest.raises(vd.VdError, match="invalid argument"):
        vd.vd_paged_attend(c, q, torch.empty_like(q),
                           torch.empty(size - 1, dtype=torch.uint8, device="cuda"), causal=False)


@pytest.mark.parametrize("B", [1, 40])
def test_graphs_replay_over_new_lengths(B):
    """A captured call reads the lengths, the table and the rows of the moment."""
    lens = [[30, 900], [0, 0], [1500, 3], [17, 1600]]
    c = ref.cache([1600 + B] * 2, 1, 2, 64, 16)
    q = queries(2, B, 4, 64)
    out = torch.empty_like(q)
    work = torch.empty(vd.vd_paged_attend_workspace(c, 4, B), dtype=torch.uint8, device="cuda")
    c.len.copy_(torch.tensor(lens[0]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vd.vd_paged_attend(c, q, out, work)
    for i, ln in enumerate(lens):
        c.len.copy_(torch.tensor(ln))
        q.copy_(queries(2, B, 4, 64, seed=i))
        work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        want, _ = check_attend(c, q)
        assert torch.equal(out, want)


def test_two_streams_with_a_workspace_each():
    c, q, kw = case("skew", BF)
    want, _ = check_attend(c, q, **kw)
    outs = [torch.empty_like(q) for _ in range(2)]
    size = vd.vd_paged_attend_workspace(c, q.shape[2], 1)
    works = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()

    def run(i):
        torch.cuda.set_device(0)
        for _ in range(20):
            vd.vd_paged_attend(c, q, outs[i], works[i], stream=streams[i])

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


@pytest.mark.parametrize("dtype", [BF, FP8])
def test_decode_steps_with_eviction(dtype):
    """The calls as a server makes them: a prompt in blocks, evicted to a budget after each one by
    way of the contiguous layout, then single tokens; the attention of every step is held to the
    definition over what the pages hold."""
    n, L, h, G, d, page, N = 2, 2, 2, 2, 64, 16, 48
    c = vd.PagedCache.empty(n, L, h, d, n_page=30, page_size=page, max_pages=8, dtype=dtype)
    order = torch.randperm(30, generator=torch.Generator().manual_seed(5)).int()
    c.page_table[:, :7] = order[:14].view(2, 7).cuda()
    flat = vd.Cache.empty(n, L, h, 8 * page, d)
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    freq = (1e4 ** (-torch.arange(0, d, 2).double() / d)).float().cuda()
    g = torch.Generator().manual_seed(6)
    for B, news in ((40, [40, 33]), (40, [12, 40]), (1, None), (1, None), (3, [0, 3])):
        count = None if news is None else torch.tensor(news, dtype=torch.int32).cuda()
        for layer in range(L):
            qkv = torch.randn((n, B, h * (G + 2), d), generator=g).to(BF).cuda()
            q = torch.zeros((n, B, h * G, d), dtype=BF, device="cuda")
            vd.vd_paged_append(c, qkv, q, layer=layer, inv_freq=freq, pos_first_new=pos,
                               n_new=count)
            check_attend(c, q, layer=layer, n_new=news)
        vd.vd_paged_advance(c, B, count)
        pos += B if count is None else count
        before = c.len.tolist()
        vd.vd_paged_unpack(c, flat)
        vd.vd_evict_block(flat, N, B=B)
        kept = flat.k.clone(), flat.v.clone()
        vd.vd_paged_pack(c, flat)
        assert c.len.tolist() == [min(m, N) for m in before]
        for s, m in enumerate(c.len.tolist()):
            for layer in range(L):
                for t, (pool, f) in enumerate(((c.k, c.k_scale), (c.v, c.v_scale))):
                    rows = ref.rows_of(c, pool, f, s, m, layer).transpose(0, 1)
                    assert torch.equal(rows, kept[t][s, layer, :, :m].cpu().double())
    assert vd.vd_get_device_status() == 0
