"""vd_qkv_norm_rope and vd_paged_append at the token counts where their kernels change: a token's rows
are the same bits, whatever the number of tokens it comes with.  Needs a GB300."""
from __future__ import annotations

import pytest
import torch

import paper_2609_23314_gb300 as vd
from paper_2609_23314_gb300 import build
from test_gpu_qkv import call, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    vd.load_library()
    torch.cuda.set_device(0)
    vd.vd_get_device_status()
    yield
    assert vd.vd_get_device_status() == 0


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rd", [(128, 128), (72, 48)])
def test_the_same_bits_at_any_count(d, rd, interleaved, norm):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    n_q, n_kv, most = 5, 2, 8 * sms + 5
    qkv, qw, kw, freq = inputs(1, most, n_q, n_kv, d, rd)
    kw_all = dict(q_weight=qw if norm else None, k_weight=kw if norm else None, inv_freq=freq,
                  interleaved=interleaved)

    def run(a, b):
        pos = torch.tensor([100 + a], dtype=torch.int32, device="cuda")
        return call(qkv[:, a:b].contiguous(), n_q, n_kv, pos_first_new=pos, **kw_all)

    parts = [run(a, min(most, a + 50)) for a in range(0, most, 50)]
    want = [torch.cat([p[i] for p in parts], 1 if i == 0 else 3) for i in range(3)]
    for count in (2 * sms, 3 * sms, 3 * sms + 1, 8 * sms - 1, 8 * sms, most):
        got = run(0, count)
        assert torch.equal(got[0], want[0][:, :count])
        assert torch.equal(got[1], want[1][:, :, :, :count])
        assert torch.equal(got[2], want[2][:, :, :, :count])
        if d % 16 == 0:  # the same rows into pages
            page = 16
            c = vd.PagedCache.empty(1, 1, n_kv, d, -(-most // page), page, -(-most // page))
            c.page_table.copy_(torch.arange(c.n_page)[None])
            q = torch.zeros_like(got[0])
            vd.vd_paged_append(c, qkv[:, :count].contiguous(), q,
                               pos_first_new=torch.tensor([100], dtype=torch.int32, device="cuda"),
                               **kw_all)
            assert torch.equal(q, got[0])
            for pool, rows in ((c.k, got[1]), (c.v, got[2])):
                flat = pool[0].transpose(0, 1).reshape(n_kv, -1, d)  # pages in order
                assert torch.equal(flat[:, :count], rows[0, 0])
                assert bool((flat[:, count:] == 0).all())
