"""The workspace of the attention over a paged cache: one size for all calls over caches of a type and
head dim, so that what fits one call fits the others.  Needs a GB300."""
from __future__ import annotations

import pytest
import torch

import paged_ref as ref
import paper_2609_23314_gb300 as vd
from paged_ref import FILL, FP8, check_attend
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
@pytest.mark.parametrize("d", [32, 96, 128, 256])
@pytest.mark.parametrize("kernel", [None, "1"])  # the library's choice, tiles of 16 rows in pieces
def test_one_size_for_all_calls(kernel, d, dtype, monkeypatch):
    """Sized once, for a block of tokens of one sequence; then single tokens, drafted ones, more heads
    and more sequences with it, and nothing behind it is written."""
    if kernel is not None:
        monkeypatch.setenv("VD_PAGED_KERNEL", kernel)
        monkeypatch.setenv("VD_PAGED_CLUSTER", "1")
    guard = 4096
    size = vd.vd_paged_attend_workspace(ref.cache([300], 1, 2, d, 16, dtype), 8, 64)
    work = torch.full((size + guard,), 255, dtype=torch.uint8, device="cuda")
    for n, h, n_q, B in ((1, 2, 8, 64), (1, 2, 8, 1), (1, 1, 1, 1), (3, 2, 6, 4), (40, 1, 2, 1),
                         (40, 2, 8, 3), (200, 1, 16, 1)):
        lens = [(97 * s + 1500) % 2000 for s in range(n)] if n < 40 else [(31 * s) % 400 for s in range(n)]
        c = ref.cache([m + B for m in lens], 1, h, d, 16, dtype)
        c.len -= B
        assert vd.vd_paged_attend_workspace(c, n_q, B) == size
        q = queries(n, B, n_q, d)
        out = torch.full_like(q, FILL)
        vd.vd_paged_attend(c, q, out, work[:size])
        assert torch.equal(out, check_attend(c, q)[0])
        assert bool((work[size:] == 255).all())
        with pytest.raises(vd.VdError, match="invalid argument"):
            vd.vd_paged_attend(c, q, out, work[:size - 16])
