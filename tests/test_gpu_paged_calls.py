"""Calls on a paged cache that users make in other orders and places than one by one: the first call
of a process inside a capture, graphs replayed on two streams at once, a wait that gives up, many
sequences, tables that repeat a page.  Needs a GB300."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest
import torch

import paged_ref as ref
import paper_2609_23314_gb300 as vd
from paged_ref import FP8, check_attend
from paper_2609_23314_gb300 import build
from test_gpu_paged_attend import queries, route  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    vd.load_library()
    torch.cuda.set_device(0)
    vd.vd_get_device_status()
    yield
    assert vd.vd_get_device_status() == 0


FIRST = """
import sys
import torch
import paper_2609_23314_gb300 as vd
torch.cuda.set_device(0)
dtype = getattr(torch, sys.argv[1])
n, L, H, G, d, B, page = 2, 2, 2, 4, 128, int(sys.argv[2]), 16
g = torch.Generator(device="cuda"); g.manual_seed(1)
rows = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
old, qkv = [rows(n, L, H, 50, d) for _ in range(2)], rows(n, B, (G + 2) * H, d)
freq = torch.ones(d // 2, device="cuda")
stages = [vd.Cache(old[0].clone(), old[1].clone(), torch.full((n,), 40, dtype=torch.int32, device="cuda"))
          for _ in range(2)]
caches = [vd.PagedCache.empty(n, L, H, d, 2 * 20, page, 20, dtype) for _ in range(2)]
for c in caches:
    c.page_table.copy_(torch.randperm(40, generator=torch.Generator().manual_seed(2)).view(2, 20))
q = rows(n, B, G * H, d)
outs = [torch.zeros_like(q) for _ in range(2)]
work = [torch.empty(vd.vd_paged_attend_workspace(c, G * H, B), dtype=torch.uint8, device="cuda") for c in caches]
back = [vd.Cache.empty(n, L, H, 50 + B, d) for _ in range(2)]
def step(i):
    vd.vd_paged_pack(caches[i], stages[i])
    for layer in range(L):
        vd.vd_paged_append(caches[i], qkv, q, layer=layer, inv_freq=freq)
        vd.vd_paged_attend(caches[i], q, outs[i], work[i], layer=layer)
    vd.vd_paged_advance(caches[i], B)
    vd.vd_paged_unpack(caches[i], back[i])
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step(0)
graph.replay()
step(1)
torch.cuda.synchronize()
assert vd.vd_get_device_status() == 0
assert caches[0].len.tolist() == caches[1].len.tolist() == [40 + B] * n == back[0].len.tolist()
for a, b in ((outs[0], outs[1]), (back[0].k, back[1].k), (back[0].v, back[1].v)):
    assert torch.equal(a, b)
assert bool(torch.isfinite(outs[0]).all()) and float(outs[0].abs().max()) > 0
"""


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("dtype,B", [("bfloat16", 1), ("float8_e4m3fn", 40)])
def test_the_first_calls_of_a_process_inside_a_capture(dtype, B):
    r = subprocess.run([sys.executable, "-c", FIRST, dtype, str(B)], cwd=ROOT, capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("B", [1, 40])
def test_graphs_on_two_streams_at_once(B):
    """Two captured calls with a workspace each, replayed together again and again."""
    c = ref.cache([3000 + B, 7 + B, 800 + B], 1, 2, 64, 16)
    c.len -= B
    q = [queries(3, B, 4, 64, seed=i) for i in range(2)]
    want = [check_attend(c, x)[0] for x in q]
    outs = [torch.zeros_like(x) for x in q]
    size = vd.vd_paged_attend_workspace(c, 4, B)
    works = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    graphs, streams = [torch.cuda.CUDAGraph() for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    for i in range(2):
        with torch.cuda.graph(graphs[i]):
            vd.vd_paged_attend(c, q[i], outs[i], works[i])
    torch.cuda.synchronize()
    for _ in range(30):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("dtype", [BF, FP8])
@pytest.mark.parametrize("B", [1, 40])
def test_a_wait_that_gives_up(B, dtype, monkeypatch):
    """With a limit of one poll, which itself may wait long enough: where it does not, the status
    says so; nothing hangs, rows behind the new tokens are left, and the next call is right."""
    c = ref.cache([2100 + B, 900 + B], 1, 2, 64, 16, dtype)
    c.len -= B
    q = queries(2, B, 4, 64)
    out = torch.full_like(q, 9.0)
    work = torch.empty(vd.vd_paged_attend_workspace(c, 4, B), dtype=torch.uint8, device="cuda")
    news = torch.tensor([B, B - 1], dtype=torch.int32).cuda()
    monkeypatch.setenv("VD_WAIT_LIMIT", "0")
    vd.vd_paged_attend(c, q, out, work, n_new=news)
    assert vd.vd_get_device_status() in (0, 5)
    assert bool((out[1, B - 1:] == 9.0).all())
    monkeypatch.delenv("VD_WAIT_LIMIT")
    check_attend(c, q, n_new=[B, B - 1])


@pytest.mark.parametrize("n", [129, 5000])
def test_many_sequences(n):
    """More sequences than one warp takes in, some of them empty."""
    lens = [(i * 53) % 29 for i in range(n)]
    c = ref.cache([m + 1 for m in lens], 1, 1, 32, 8)
    c.len -= 1
    check_attend(c, queries(n, 1, 2, 32), n_new=[int(i % 7 > 0) for i in range(n)])
    flat = vd.Cache.empty(n, 1, 1, 30, 32)
    vd.vd_paged_unpack(c, flat)
    other = ref.cache([0] * n, 1, 1, 32, 16, extra=30)
    vd.vd_paged_pack(other, flat)
    assert flat.len.tolist() == lens == other.len.tolist()
    for s in (0, 1, 128, n - 1):
        assert torch.equal(ref.rows_of(c, c.v, None, s, lens[s], 0),
                           ref.rows_of(other, other.v, None, s, lens[s], 0))


@pytest.mark.usefixtures("route")
def test_a_page_twice_in_a_table():
    """A sequence that reads one page at two places (of slots that no call writes)."""
    c = ref.cache([70], 1, 1, 64, 16)
    c.page_table[0, 1] = c.page_table[0, 3]
    c.len -= 1
    check_attend(c, queries(1, 1, 4, 64))
    check_attend(c, queries(1, 1, 24, 64))


@pytest.mark.usefixtures("route")
def test_calls_that_reuse_one_workspace():
    """Calls of other sizes one after the other on a stream, with the workspace of the largest."""
    cases = [(ref.cache([2000 + B, 90 + B], 1, 2, d, 16, dtype), B, d) for B, d, dtype in
             ((1, 128, BF), (4, 64, FP8), (40, 96, BF), (1, 256, FP8))]
    size = 0
    for c, B, d in cases:
        c.len -= B
        size = max(size, vd.vd_paged_attend_workspace(c, 8, B))
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    qs = [queries(2, B, 8, d) for _, B, d in cases]
    outs = [torch.empty_like(q) for q in qs]
    for _ in range(3):
        for (c, B, d), q, out in zip(cases, qs, outs):
            vd.vd_paged_attend(c, q, out, work)
    torch.cuda.synchronize()
    for (c, B, d), q, out in zip(cases, qs, outs):
        assert torch.equal(out, check_attend(c, q)[0])
