"""Tensors that are not on a GPU do not reach the library: a kernel would take their
addresses for device memory.  CPU only: every call here is refused in the binding."""
import pytest
import torch

import paper_2609_23314_gb300 as vd


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2609_23314_gb300 import build
    build.build()
    vd.load_library()


N_SEQ, L, H, CAP, D = 2, 2, 3, 16, 64


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


@pytest.fixture
def cache():
    return vd.Cache.empty(N_SEQ, L, H, CAP, D, device="cpu")


@pytest.fixture
def cache4():
    return vd.Q4Cache.empty(N_SEQ, L, H, CAP, D, device="cpu")


def refused():
    return pytest.raises(ValueError, match="must live on a CUDA device, got cpu")


def test_calls_on_a_4_bit_cache(cache, cache4):
    new, q = bf(N_SEQ, L, H, 1, D), bf(N_SEQ, 1, 2 * H, D)
    with refused():
        vd.vd_q4_append(cache4, new, new, 1)
    with refused():
        vd.vd_q4_pack(cache4, cache)
    with refused():
        vd.vd_q4_unpack(cache4, cache)
    for rows in (new, None):
        with refused():
            vd.vd_q4_attend(cache4, q, torch.empty_like(q), rows, rows)


def test_projections():
    new, q = bf(N_SEQ, L, H, 1, D), bf(N_SEQ, 1, 2 * H, D)
    with refused():
        vd.vd_qkv_norm_rope(bf(N_SEQ, 1, 4 * H, D), q, new, new.clone())


def test_calls_on_a_bf16_cache(cache):
    us, N = (N_SEQ, L, H), 4
    new = bf(*us, 1, D)
    scores, kept = torch.empty(us + (CAP,)), torch.empty(us + (N,), dtype=torch.int32)
    pos = torch.zeros(us + (CAP,), dtype=torch.int32)
    first = torch.zeros(N_SEQ, dtype=torch.int32)
    calls = [
        lambda: vd.vd_score(cache, vd.VD_SCORE_L2, scores),
        lambda: vd.vd_score_ex(cache, vd.VD_SCORE_L2, scores_out=scores),
        lambda: vd.vd_evict_block(cache, N, kept_idx_out=kept),
        lambda: vd.vd_evict_block_ex(cache, N),
        lambda: vd.vd_evict_decode(cache, N),
        lambda: vd.vd_append_evict_block(cache, new, new, 1, N),
        lambda: vd.vd_append_evict_block_ex(cache, new, new, 1, N),
        lambda: vd.vd_append_evict_decode(cache, new, new, N),
        lambda: vd.vd_evict_block_holefill(cache, N, pos=pos, pos_first_new=first),
        lambda: vd.vd_evict_decode_holefill(cache, N, pos=pos, pos_first_new=first),
        lambda: vd.vd_append(cache, new, new, 1),
        lambda: vd.vd_running_sum_init(cache, torch.zeros(us + (D,), dtype=torch.float64)),
        lambda: vd.vd_running_sum_init_ex(cache, True, torch.zeros(us + (D,),
                                                                   dtype=torch.float64)),
    ]
    for call in calls:
        with refused():
            call()
    assert vd.vd_workspace_size(cache) == 0  # asks no kernel
