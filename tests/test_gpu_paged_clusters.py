"""Attention over a paged cache by clusters of more CTAs than eight, which single long sequences take:
the joins over 9, 12 and 16 parts, forced on every kernel, and as the library chooses them.  Needs a
GB300."""
from __future__ import annotations

import pytest
import torch

import paged_ref as ref
import paper_2609_23314_gb300 as vd
from paged_ref import FP8, check_attend
from paper_2609_23314_gb300 import build
from test_gpu_paged_attend import queries

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


@pytest.mark.parametrize("dtype", [BF, FP8])
@pytest.mark.parametrize("kernel", ["0", "1", "2"])
@pytest.mark.parametrize("cluster", ["9", "12", "16"])
@pytest.mark.parametrize("d,G", [(128, 4), (256, 8), (96, 5)])
def test_forced(d, G, cluster, kernel, dtype, monkeypatch):
    """A long sequence, one of fewer stages than CTAs, a single slot, and none."""
    monkeypatch.setenv("VD_PAGED_KERNEL", kernel)
    monkeypatch.setenv("VD_PAGED_CLUSTER", cluster)
    for B in (1, 5):
        c = ref.cache([3000 + B, 100 + B, 1 + B, B], 1, 1, d, 24, dtype)
        c.len -= B
        check_attend(c, queries(4, B, G, d), n_new=[B, B, B, B - 1])
    c = ref.cache([3000, 0], 1, 1, d, 24, dtype)  # no slot at all: zeros
    check_attend(c, queries(2, 2, G, d), causal=False)


@pytest.mark.parametrize("dtype", [BF, FP8])
@pytest.mark.parametrize("n,h,length,B", [(1, 8, 16000, 1), (1, 4, 9000, 2), (2, 4, 16000, 1),
                                          (1, 1, 9000, 40)])
def test_as_chosen(n, h, length, B, dtype):
    """Sizes for which the rule takes 9 to 16 CTAs."""
    c = ref.cache([length + B - 7 * s for s in range(n)], 1, h, 128, 64, dtype)
    c.len -= B
    q = queries(n, B, 2 * h, 128)
    first = check_attend(c, q)
    again = check_attend(c, q)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("kernel", ["0", "2"])
def test_nan_in_one_part(kernel, monkeypatch):
    """A NaN that one CTA's slots hold, and slots of -infinity in another one's."""
    monkeypatch.setenv("VD_PAGED_KERNEL", kernel)
    monkeypatch.setenv("VD_PAGED_CLUSTER", "12")
    n = 2400
    c = ref.cache([n + 3], 1, 1, 64, 16)
    c.len -= 3
    q = queries(1, 3, 4, 64).abs() + 0.1
    for t in range(0, 200):  # the first CTA's: nothing but -infinity
        c.k[0, int(c.page_table[0, t // 16]), 0, t % 16, 0] = -float("inf")
    out, lse = check_attend(c, q)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    t = n + 2  # the last token's own row
    c.k[0, int(c.page_table[0, t // 16]), 0, t % 16, 5] = float("nan")
    out, _ = check_attend(c, q)
    assert bool(torch.isfinite(out[0, :2]).all()) and bool(torch.isnan(out[0, 2]).all())
