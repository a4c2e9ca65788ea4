"""Calls on a 4-bit cache that users make in other orders and places than one by one: the first
call of a process inside a capture, graphs replayed on two streams at once, calls from several
threads, prompts over themselves.  Needs a GB300."""
from __future__ import annotations

import os
import subprocess
import sys
import threading

import pytest
import torch

import paper_2609_23314_gb300 as vd
from paper_2609_23314_gb300 import build
from test_gpu_q4_attend import check, state

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    vd.load_library()
    torch.cuda.set_device(0)
    vd.vd_get_device_status()
    yield
    assert vd.vd_get_device_status() == 0


@pytest.fixture(params=["automatic", "streaming8", "streaming16", "block"])
def route(request, monkeypatch):
    kinds = {"streaming8": "0", "streaming16": "1", "block": "2"}
    if request.param in kinds:
        monkeypatch.setenv("VD_Q4_KERNEL", kinds[request.param])


FIRST = """
import torch
import paper_2609_23314_gb300 as vd
torch.cuda.set_device(0)
H, G, d, n, B, cap = 2, 4, 128, 40, 3, 64
g = torch.Generator(device="cuda"); g.manual_seed(1)
rows = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
old, qkv = [rows(1, 1, H, n, d) for _ in range(2)], rows(1, B, (G + 2) * H, d)
q, outs = rows(1, B, G * H, d), [rows(1, B, G * H, d) for _ in range(2)]
new = [rows(1, 1, H, B, d) for _ in range(2)]
freq, first = torch.ones(d // 2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
caches = [vd.Q4Cache.empty(1, 1, H, cap, d) for _ in range(2)]
stages = [vd.Cache.empty(1, 1, H, cap, d) for _ in range(2)]
def step(i):
    vd.vd_q4_append(caches[i], old[0], old[1], n)
    vd.vd_qkv_norm_rope(qkv, q, new[0], new[1], inv_freq=freq, pos_first_new=first)
    vd.vd_q4_attend(caches[i], q, outs[i], new[0], new[1])
    vd.vd_q4_append(caches[i], new[0], new[1], B)
    vd.vd_q4_unpack(caches[i], stages[i])
    vd.vd_q4_pack(caches[i], stages[i])
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step(0)
graph.replay()
step(1)
torch.cuda.synchronize()
assert vd.vd_get_device_status() == 0
assert caches[0].len.tolist() == caches[1].len.tolist() == [n + B]
for a, b in ((outs[0], outs[1]), (stages[0].k, stages[1].k), (caches[0].v, caches[1].v),
             (caches[0].v_scale, caches[1].v_scale)):
    assert torch.equal(a, b)
assert bool(torch.isfinite(outs[0]).all()) and float(outs[0].abs().max()) > 0
"""


@pytest.mark.usefixtures("route")
def test_the_first_calls_of_a_process_inside_a_capture():
    r = subprocess.run([sys.executable, "-c", FIRST], cwd=ROOT, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("B", [1, 40])
def test_graphs_on_two_streams_at_once(B):
    """Two graphs of many calls on caches of their own, replayed side by side: nothing shared."""
    cases = [state([700, 90], 1, 2, 4, 128, B, 704, seed=i) for i in range(2)]
    want = [check(*c)[0] for c in cases]
    outs, graphs = [torch.empty_like(w) for w in want], []
    streams = [torch.cuda.Stream() for _ in cases]
    for (c, q, k, v), o in zip(cases, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            for _ in range(30):
                vd.vd_q4_attend(c, q, o, k, v)
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


@pytest.mark.usefixtures("route")
def test_calls_from_several_threads():
    """Each thread on its own stream, head dim and cache."""
    cases = [state([300, 33], 1, 2, 4, d, B, 304) for d, B in ((64, 1), (96, 5), (128, 40), (256, 2))]
    want = [check(*c)[0] for c in cases]
    outs = [[torch.empty_like(w) for _ in range(20)] for w in want]
    torch.cuda.synchronize()
    errors = []

    def work(case, mine):
        try:
            torch.cuda.set_device(0)
            with torch.cuda.stream(torch.cuda.Stream()):
                for o in mine:
                    vd.vd_q4_attend(case[0], case[1], o, case[2], case[3])
        except Exception as e:  # a thread's exception would be lost
            errors.append(e)

    threads = [threading.Thread(target=work, args=a) for a in zip(cases, outs)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    assert all(torch.equal(o, w) for mine, w in zip(outs, want) for o in mine)


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("d,group,B", [(128, 4, 700), (64, 1, 1100), (160, 2, 300), (192, 3, 200),
                                       (224, 5, 150), (256, 2, 400)])
def test_prompts_over_themselves(d, group, B):
    """An empty cache and a short one, so that most tiles hold new rows."""
    check(*state([0, 70], 1, 1, group, d, B, 72))


@pytest.mark.usefixtures("route")
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d,B", [(64, 1), (128, 40), (256, 3)])
def test_a_query_that_is_not_finite_stays_alone(d, B, value):
    """Its own row becomes NaN; every other row stays as it is, but for roundings."""
    c, q, k_new, v_new = state([300, 33], 1, 2, 4, d, B, 304)
    clean, _ = check(c, q, k_new, v_new)
    bad = q.clone()
    bad[1, B - 1, 5, 3] = value
    out = torch.full_like(q, 9.0)
    vd.vd_q4_attend(c, bad, out, k_new, v_new)
    want = torch.zeros_like(out, dtype=torch.bool)
    want[1, B - 1, 5] = True
    assert torch.equal(torch.isnan(out), want)
    # the weights' references are renewed row by row, their moment for a whole warp: outputs
    # of other rows are within twice their rounding
    diff = (out.double() - clean.double()).abs()[~want]
    assert bool((diff <= 2.0 ** -7 * clean.double().abs()[~want] + 2.0 ** -12).all())
