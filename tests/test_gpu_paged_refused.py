"""vd_paged_pack and vd_paged_unpack where sequences that they refuse stand between valid ones: the
refused ones are left untouched on both sides, the others arrive whole.  Needs a GB300."""
from __future__ import annotations

import pytest
import torch

import paged_ref as ref
import paper_2609_23314_gb300 as vd
from paged_ref import FILL, FP8, raw
from paper_2609_23314_gb300 import build

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
PAGE, PLACES, CAP = 8, 3, 39  # 24 slots a sequence in pages, 39 in the contiguous cache
SLOTS = PAGE * PLACES

LENS = {
    "one_between": [3, 25, 3],
    "many_between": [3, 25, 3, 39, 5],
    "first": [39, 24, 0, 1],
    "of_each_kind": [25, 7, -1, 24, 40, 2, 39, -2147483648, 9, 2147483647],
    "more_than_a_block_of_threads": [(25 + i % 15 if i % 3 == 1 else (i * 7) % 25) for i in range(300)],
    # the last sequences that one look of the threads takes in and the first of the next
    "at_the_seam": [(30 if 250 <= i < 260 else (i * 5) % 25) for i in range(520)],
}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    vd.load_library()
    torch.cuda.set_device(0)
    vd.vd_get_device_status()
    yield
    assert vd.vd_get_device_status() == 0


def paged(n, L, h, d, dtype):
    """A cache of n sequences with all their pages, rows of its own in every slot."""
    c = ref.cache([SLOTS] * n, L, h, d, PAGE, dtype)
    table = c.page_table[:, :PLACES].contiguous()  # no place behind: a row is followed by the next one
    return vd.PagedCache(c.k, c.v, table, c.len, c.k_scale, c.v_scale)


def contiguous(n, L, h, d):
    g = torch.Generator().manual_seed(3)
    rows = [torch.randn((n, L, h, CAP, d), generator=g).to(BF).cuda() for _ in range(2)]
    return vd.Cache(*rows, torch.zeros(n, dtype=torch.int32, device="cuda"))


def valid(lens):
    return [s for s, m in enumerate(lens) if 0 <= m <= SLOTS]


@pytest.mark.parametrize("dtype", [BF, FP8])
@pytest.mark.parametrize("L,h,d", [(1, 2, 32), (3, 1, 96)])
@pytest.mark.parametrize("name", LENS)
def test_unpack(name, L, h, d, dtype):
    lens = LENS[name]
    n = len(lens)
    c, flat = paged(n, L, h, d, dtype), contiguous(n, L, h, d)
    c.len.copy_(torch.tensor(lens, dtype=torch.int64).int())
    flat.len.fill_(77)
    want = [flat.k.clone(), flat.v.clone()]
    for s in valid(lens):
        for t, (pool, f) in enumerate(((c.k, c.k_scale), (c.v, c.v_scale))):
            for layer in range(L):
                rows = ref.rows_of(c, pool, f, s, lens[s], layer).transpose(0, 1)
                want[t][s, layer, :, :lens[s]] = rows.float().to(BF).cuda()
    vd.vd_paged_unpack(c, flat)
    assert vd.vd_get_device_status() == 7
    assert flat.len.tolist() == [m if 0 <= m <= SLOTS else 77 for m in lens]
    assert torch.equal(flat.k, want[0]) and torch.equal(flat.v, want[1])


@pytest.mark.parametrize("dtype", [BF, FP8])
@pytest.mark.parametrize("L,h,d", [(1, 2, 32), (3, 1, 96)])
@pytest.mark.parametrize("name", LENS)
def test_pack(name, L, h, d, dtype):
    lens = LENS[name]
    n = len(lens)
    c, flat = paged(n, L, h, d, dtype), contiguous(n, L, h, d)
    flat.len.copy_(torch.tensor(lens, dtype=torch.int64).int())
    c.len.fill_(77)
    want = [raw(p).clone() for p in (c.k, c.v)]
    for s in valid(lens):
        slot = torch.arange(lens[s], device="cuda")
        page = c.page_table[s, slot // PAGE].long()
        for pool, f, rows in zip(want, (c.k_scale, c.v_scale), (flat.k, flat.v)):
            x = rows[s, :, :, :lens[s]].float()  # [L, h, slots, d]
            if f is not None:
                x = (x / f[:, :, None, None]).clamp(-448, 448)
            pool[:, page, :, slot % PAGE] = raw(x.to(dtype)).permute(2, 0, 1, 3)
    vd.vd_paged_pack(c, flat)
    assert vd.vd_get_device_status() == 7
    assert c.len.tolist() == [m if 0 <= m <= SLOTS else 77 for m in lens]
    assert torch.equal(raw(c.k), want[0]) and torch.equal(raw(c.v), want[1])


def test_nothing_but_refused_sequences():
    c, flat = paged(3, 2, 2, 64, BF), contiguous(3, 2, 2, 64)
    before = [t.clone() for t in (c.k, c.v, flat.k, flat.v)]
    c.len.copy_(torch.tensor([25, -1, 39]))
    flat.len.fill_(77)
    vd.vd_paged_unpack(c, flat)
    assert vd.vd_get_device_status() == 7
    flat.len.copy_(torch.tensor([25, -1, 39]))
    c.len.fill_(77)
    vd.vd_paged_pack(c, flat)
    assert vd.vd_get_device_status() == 7
    assert all(torch.equal(a, b) for a, b in zip(before, (c.k, c.v, flat.k, flat.v)))
    assert c.len.tolist() == [77] * 3


def test_a_whole_cache_with_one_refused_sequence():
    """Many CTAs: the pieces of the line begin and end inside sequences."""
    lens = [1000, 1025, 77, 1024, 2000, 513]
    page, L, h, d, cap = 64, 12, 4, 128, 2048
    c = ref.cache([1024] * 6, L, h, d, page, extra=0)
    c = vd.PagedCache(c.k, c.v, c.page_table[:, :16].contiguous(), c.len)
    flat = vd.Cache(*(torch.full((6, L, h, cap, d), FILL, dtype=BF, device="cuda") for _ in range(2)),
                    torch.full((6,), 77, dtype=torch.int32, device="cuda"))
    c.len.copy_(torch.tensor(lens))
    vd.vd_paged_unpack(c, flat)
    assert vd.vd_get_device_status() == 7
    assert flat.len.tolist() == [1000, 77, 77, 1024, 77, 513]
    for s, m in enumerate(lens):
        good = m <= 1024
        slot = torch.arange(m if good else 0, device="cuda")
        for pool, rows in ((c.k, flat.k), (c.v, flat.v)):
            if good:
                got = pool[:, c.page_table[s, slot // page].long(), :, slot % page]  # [m, L, h, d]
                assert torch.equal(rows[s, :, :, :m], got.permute(1, 2, 0, 3))
            assert bool((rows[s, :, :, m if good else 0:] == FILL).all())
