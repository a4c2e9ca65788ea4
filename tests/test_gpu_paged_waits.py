"""Attention over a paged cache with waits that give up after a few polls, again and again, so that some
of a warp's lanes may see a phase end that others do not wait for: every call ends, records
VD_ERR_TIMEOUT or is right, leaves what lies behind the new tokens, and the calls after it are right.
Needs a GB300."""
from __future__ import annotations

import pytest
import torch

import paged_ref as ref
import paper_2609_23314_gb300 as vd
from paged_ref import FILL, FP8, check_attend
from paper_2609_23314_gb300 import build
from test_gpu_paged_attend import queries, route  # noqa: F401 (a fixture)

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


@pytest.mark.parametrize("dtype", [BF, FP8])
@pytest.mark.parametrize("B", [1, 12])
def test_few_polls(B, dtype, monkeypatch):
    c = ref.cache([5000 + B, 40 + B, 1700 + B], 1, 2, 128, 16, dtype)
    c.len -= B
    news = [B, 0, max(0, B - 1)]
    q = queries(3, B, 8, 128)
    want, _ = check_attend(c, q, n_new=news)
    out = torch.empty_like(q)
    work = torch.empty(vd.vd_paged_attend_workspace(c, 8, B), dtype=torch.uint8, device="cuda")
    new = torch.tensor(news, dtype=torch.int32).cuda()
    for limit in (0, 1, 2, 3, 5, 8, 13, 40) * 4:
        out.fill_(FILL)
        monkeypatch.setenv("VD_WAIT_LIMIT", str(limit))
        vd.vd_paged_attend(c, q, out, work, n_new=new)
        status = vd.vd_get_device_status()
        assert status in (0, 5)
        if status == 0:
            assert torch.equal(out, want)
        for s, m in enumerate(news):
            assert bool((out[s, m:] == FILL).all())
        monkeypatch.delenv("VD_WAIT_LIMIT")
        vd.vd_paged_attend(c, q, out, work, n_new=new)
        assert vd.vd_get_device_status() == 0 and torch.equal(out, want)
