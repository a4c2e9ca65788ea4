"""Norms per head, rotation and the split into queries and new rows (vd_qkv_norm_rope)
against the formula in 64 bits, and the operators of the 4-bit cache run together.
Needs a GB300."""
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


def inputs(n_seq, B, n_q, n_kv, d, rd, seed=0, size=1.0):
    g = torch.Generator().manual_seed(seed)
    qkv = (torch.randn((n_seq, B, n_q + 2 * n_kv, d), generator=g) * size).to(torch.bfloat16)
    qw, kw = (1 + 0.3 * torch.randn((2, d), generator=g)).to(torch.bfloat16)
    freq = (1e4 ** (-torch.arange(0, rd, 2).double() / max(rd, 1))).float() if rd else None
    return qkv.cuda(), qw.cuda(), kw.cuda(), None if freq is None else freq.cuda()


def call(qkv, n_q, n_kv, layer=0, n_layer=1, **kw):
    n_seq, B, _, d = qkv.shape
    q = torch.full((n_seq, B, n_q, d), 9.0, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.full((n_seq, n_layer, n_kv, B, d), 9.0, dtype=torch.bfloat16, device="cuda")
            for _ in range(2))
    vd.vd_qkv_norm_rope(qkv, q, k, v, layer=layer, **kw)
    return q, k, v


def check(qkv, n_q, n_kv, qw, kw, freq, pos0, interleaved, eps=1e-6, layer=0, n_layer=1):
    n_seq, B, _, d = qkv.shape
    pos = torch.tensor(pos0, dtype=torch.int32)
    q, k, v = call(qkv, n_q, n_kv, layer, n_layer, q_weight=qw, k_weight=kw, eps=eps,
                   inv_freq=freq, pos_first_new=None if freq is None else pos.cuda(),
                   interleaved=interleaved)
    x = qkv.cpu().double()
    cpu = lambda t: None if t is None else t.cpu()
    for s in range(n_seq):
        at = int(pos0[s]) + torch.arange(B, dtype=torch.int64)
        for got, lo, hi, w in ((q[s], 0, n_q, qw), (k[s, layer].transpose(0, 1), n_q, n_q + n_kv,
                                                    kw)):
            y, size = ref.norm_rope(x[s, :, lo:hi], cpu(w), eps, cpu(freq), at, interleaved)
            err = (got.cpu().double() - y).abs() - ref.norm_rope_tolerance(y, size)
            assert bool((err <= 0).all()), f"{err.max()} more than allowed"
        assert torch.equal(v[s, layer].transpose(0, 1), qkv[s, :, n_q + n_kv:])
    others = [i for i in range(n_layer) if i != layer]
    assert bool((k[:, others] == 9.0).all()) and bool((v[:, others] == 9.0).all())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rd", [(8, 0), (16, 16), (24, 16), (64, 64), (72, 48), (80, 80),
                                  (96, 32), (128, 128), (128, 64), (200, 160), (248, 16),
                                  (256, 256)])
def test_head_dims(d, rd, interleaved):
    for n_seq, B, n_q, n_kv in ((1, 1, 4, 1), (2, 5, 6, 3), (3, 2, 1, 1)):
        qkv, qw, kw, freq = inputs(n_seq, B, n_q, n_kv, d, rd)
        check(qkv, n_q, n_kv, qw, kw, freq, [7 * s for s in range(n_seq)], interleaved)


@pytest.mark.parametrize("which", ["none", "queries", "keys"])
def test_norms_are_optional(which):
    qkv, qw, kw, freq = inputs(2, 3, 4, 2, 64, 64)
    check(qkv, 4, 2, qw if which == "queries" else None, kw if which == "keys" else None, freq,
          [3, 90], False)


@pytest.mark.parametrize("first", [0, 1000003, 2 ** 31 - 5000, -40])
def test_positions(first):
    """Far positions: the angle is reduced before it is rounded to fp32.  Enough tokens
    that a CTA takes several of them, across the border between two sequences."""
    qkv, qw, kw, freq = inputs(3, 1001, 2, 1, 64, 64)
    check(qkv, 2, 1, qw, kw, freq, [first, first + 1500, first + 3], False, layer=1, n_layer=3)


@pytest.mark.parametrize("size", [1e-18, 1e18])
def test_magnitudes(size):
    qkv, qw, kw, freq = inputs(1, 3, 4, 2, 128, 128, size=size)
    check(qkv, 4, 2, qw, kw, freq, [5], False, eps=0.0)


def test_zero_rows():
    qkv, qw, kw, freq = inputs(1, 3, 4, 2, 128, 128)
    qkv[:, 1] = 0
    check(qkv, 4, 2, qw, kw, freq, [5], True, eps=1e-6)


def test_graph_and_streams():
    qkv, qw, kw, freq = inputs(4, 300, 8, 2, 128, 128)
    pos = torch.arange(4, dtype=torch.int32, device="cuda") * 1000
    kws = dict(q_weight=qw, k_weight=kw, inv_freq=freq, pos_first_new=pos)
    first = call(qkv, 8, 2, **kws)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = call(qkv, 8, 2, stream=side, **kws)
    torch.cuda.synchronize()
    # the fills ran on the current stream, so the call may have overtaken them: run again
    vd.vd_qkv_norm_rope(qkv, *other, stream=side, **kws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = call(qkv, 8, 2, **kws)
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, other, captured):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_together():
    """Steps of a two-layer model over a 4-bit cache: rows from projections, attention over
    the cache and the step's own rows, the rows appended; then the cache read back, evicted
    with the library's own call and packed again.  Every step against the 64-bit forms on
    the step's own inputs."""
    n_seq, L, H, G, d, cap = 2, 2, 2, 4, 64, 64
    c = vd.Q4Cache.empty(n_seq, L, H, cap, d)
    qw, kw = torch.ones((2, d), dtype=torch.bfloat16, device="cuda")
    freq = (1e4 ** (-torch.arange(0, d, 2).double() / d)).float().cuda()
    pos, length = 0, 0
    for step, B in enumerate((24, 1, 7, 1, 1)):
        k_new, v_new = (torch.empty((n_seq, L, H, B, d), dtype=torch.bfloat16, device="cuda")
                        for _ in range(2))
        for layer in range(L):
            qkv, _, _, _ = inputs(n_seq, B, H * G, H, d, 0, seed=10 * step + layer)
            q, out = (torch.empty((n_seq, B, H * G, d), dtype=torch.bfloat16, device="cuda")
                      for _ in range(2))
            vd.vd_qkv_norm_rope(qkv, q, k_new, v_new, layer=layer, q_weight=qw, k_weight=kw,
                                inv_freq=freq, pos_first_new=torch.full((n_seq,), pos,
                                                                        dtype=torch.int32,
                                                                        device="cuda"))
            vd.vd_q4_attend(c, q, out, k_new, v_new, layer=layer)
            for s in range(n_seq):
                for h in range(H):
                    m = length
                    ks, vs = (ref.values(x[s, layer, h, :m].cpu(), y[s, layer, h, :m].cpu())
                              for x, y in ((c.k, c.k_scale), (c.v, c.v_scale)))
                    hs = slice(h * G, (h + 1) * G)
                    got = ref.attend(q[s, :, hs].cpu().double(), ks, vs,
                                     k_new[s, layer, h].cpu().double(),
                                     v_new[s, layer, h].cpu().double(), d ** -0.5)
                    tol, _ = ref.attend_tolerance(*got, m + B, d)
                    assert bool(((out[s, :, hs].cpu().double() - got[0]).abs() <= tol).all())
        vd.vd_q4_append(c, k_new, v_new, B)
        pos, length = pos + B, length + B
        assert c.len.tolist() == [length] * n_seq
        want_k, want_s = ref.quantise(k_new.cpu())
        assert torch.equal(c.k[:, :, :, length - B:length].cpu(), want_k)
        assert torch.equal(c.k_scale[:, :, :, length - B:length].cpu(), want_s)
    stage = vd.Cache.empty(n_seq, L, H, cap, d)
    vd.vd_q4_unpack(c, stage)
    before = [t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale)]
    N = 20
    kept = torch.empty((n_seq, L, H, N), dtype=torch.int32, device="cuda")
    vd.vd_evict_block(stage, N, kept_idx_out=kept)
    vd.vd_q4_pack(c, stage)
    assert c.len.tolist() == [N] * n_seq
    for t, old in zip((c.k, c.v, c.k_scale, c.v_scale), before):
        idx = kept.long()[..., None].expand(-1, -1, -1, -1, t.shape[-1])
        assert torch.equal(t[:, :, :, :N], torch.gather(old, 3, idx))


def test_readme_example_of_the_4_bit_cache():
    """The README's examples run as written, one after the other."""
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), flags=re.S)
    names = {}
    exec(compile("\n".join(blocks[:2]), "README.md", "exec"), names)
    assert names["q4"].len.tolist() == [names["N"]] * names["n_seq"]
    assert bool(torch.isfinite(names["out"]).all())
