"""Caches whose summaries would fill 4 GiB or more: the paged-cache calls that touch no summaries
take them, the calls that address the store refuse them."""
import ctypes

import pytest
import torch

from paper_2607_24555_amd import cache as C
from paper_2607_24555_amd import locks as B
from tests.test_cache_binding import FAKE, cfg, lib, q8, rope, rows  # noqa: F401

BIG = dict(num_blocks=2_600_000)      # x 2 KV heads x 832 bytes


def test_only_calls_with_summaries_refuse_a_large_store(lib):  # noqa: F811
    c, s = cfg(**BIG).c(), q8()
    ref = ctypes.byref(c)
    need = lib.locks_workspace_bytes(ref)
    assert need == lib.locks_workspace_bytes(ctypes.byref(cfg().c())) > 0
    assert lib.locks_table_error_offset(ref) == lib.locks_table_error_offset(ctypes.byref(cfg().c()))
    empty = ctypes.byref(rows(n_tokens=0))            # (no rows: no launch)
    assert lib.locks_rope_append_kv(ref, empty, ctypes.byref(rope()), FAKE, FAKE, FAKE, FAKE, None) == 0
    assert lib.locks_q8_append_kv(ref, empty, ctypes.byref(rope()), ctypes.byref(s), FAKE, FAKE, None) == 0
    # (past the configuration: what is refused is the small workspace)
    assert lib.locks_q8_dense_attend(ref, FAKE, ctypes.byref(s), FAKE, FAKE, FAKE, None, FAKE, need - 1, None) == -3
    assert lib.locks_q8_sparse_attend(ref, FAKE, ctypes.byref(s), FAKE, FAKE, FAKE, FAKE, None, FAKE, need - 1,
                                      None) == -3
    assert lib.locks_q8_build_summaries(ref, ctypes.byref(s), FAKE, FAKE, None, 0, FAKE, None) == -2
    assert lib.locks_build_summaries(ref, FAKE, FAKE, FAKE, None, 0, FAKE, None) == -2
    assert lib.locks_select(ref, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, need, None) == -2
    # other bad configurations are refused everywhere
    bad = cfg(rank=0, **BIG).c()
    assert lib.locks_workspace_bytes(ctypes.byref(bad)) == 0
    assert lib.locks_rope_append_kv(ctypes.byref(bad), empty, None, FAKE, FAKE, FAKE, FAKE, None) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("checks", [False, True])
def test_append_and_attend_with_a_large_store(checks):
    """One KV head, 5.2 million blocks of 16 tokens (10.6 GB of codes a tensor, a summary store of
    4.3 GB): tokens go to the last blocks and are attended."""
    nb, P, T, D = 5_200_000, 16, 70, 128
    c = B.Config(1, 4, 1, 8, 2 * P, 5, nb, B.LOCKS_FP32, B.LOCKS_FP32, page_size=P)
    assert nb * B.summary_stride(8) >= 1 << 32
    store = C.alloc_q8_cache(c)
    g = torch.Generator().manual_seed(3)
    pt = torch.tensor([[nb - 1, 7, nb - 2, 0, nb - 3]], dtype=torch.int32)
    sl = torch.tensor([T], dtype=torch.int32).cuda()
    k, v, q = torch.randn(T, 1, D, generator=g), torch.randn(T, 1, D, generator=g), torch.randn(1, 4, D, generator=g)
    ws = B.alloc_workspace(c)
    was = B.set_table_checks(checks)
    try:
        C.q8_append_kv(c, k.cuda(), v.cuda(), store, pt.cuda(), sl, cu_tokens=torch.tensor([0, T], dtype=torch.int32).cuda())
        out, lse = C.q8_dense_attend(c, q.cuda(), store, pt.cuda(), sl, ws)
        if checks:
            assert B.table_errors(c, ws) == (0, [0])
    finally:
        B.set_table_checks(was)
    at = pt[0].long().cuda()
    K, V = ((x[at, 0].double() * s[at, 0].double()[:, None, None]).reshape(-1, D)[:T].cpu()
            for x, s in ((store.k, store.k_scale), (store.v, store.v_scale)))
    # a code is within half a step of its row (and 2^-23 of 127 steps): the rows are there
    step = torch.stack([s[at, 0] for s in (store.k_scale, store.v_scale)]).cpu().repeat_interleave(P, 1)[:, :T, None]
    assert bool(((K - k[:, 0]).abs() <= step[0] * (0.5 + 2.0 ** -16)).all())
    assert bool(((V - v[:, 0]).abs() <= step[1] * (0.5 + 2.0 ** -16)).all())
    z = q[0].double() @ K.t() / D ** 0.5
    # 264 roundings of 2^-24 of a logit's products; 2^-19 for the weights and sums
    dz = 264 * 2.0 ** -24 * float((q[0].double().abs() @ K.abs().t()).max()) / D ** 0.5
    want = torch.softmax(z, -1) @ V
    assert bool(((out[0].cpu().double() - want).abs() <= (2 * dz + 2.0 ** -19) * V.abs().amax(0)).all())
    assert bool(((lse[0].cpu().double() - torch.logsumexp(z, -1)).abs() <= dz + 2.0 ** -19).all())
