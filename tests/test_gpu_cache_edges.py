"""GPU checks of the paged-cache calls at the edges of their definition (include/locks_cache.h):
rows that are not finite, scales of extreme size or sign, one token a sequence."""
import numpy as np
import pytest
import torch

from paper_2607_24555_amd import cache as C
from paper_2607_24555_amd import locks as B

pytestmark = pytest.mark.gpu
D = 128
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
LK = {"bf16": B.LOCKS_BF16, "fp32": B.LOCKS_FP32}
CODES = [torch.int8, torch.float8_e4m3fn]
INF, NAN = float("inf"), float("nan")


def _most(code):
    return 127.0 if code == torch.int8 else 448.0


def _nan_code(code):
    return 0.0 if code == torch.int8 else NAN


def _same(got, want):
    """Equal values, NaN where there is NaN (the sign of a zero does not count)."""
    got, want = got.cpu().float(), want.float()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got[~nan], want[~nan])


# First elements of a page's rows; the others are zero.  The largest finite magnitude is under
# 2^-100, so the page's scale is 0.
NOT_FINITE = [[[INF, -INF]], [[INF, 2.0 ** -110, NAN]], [[-INF], [0.0, INF], [NAN]], [[NAN, -NAN]],
              [[2.0 ** -101, -2.0 ** -120], [0.0, -INF]], [[INF] * D] * 3]


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("kv", ["bf16", "fp32"])
@pytest.mark.parametrize("P", [16, 32, 64])
def test_q8_append_infinities_beside_nothing_finite(code, kv, P):
    """An infinity takes the largest code also where the page's scale is 0, a NaN 0 (int8) or NaN
    (e4m3); the page attends as zeros; a row that makes the scale grow turns the earlier codes
    into code * 0, and one beside finite rows leaves their scale."""
    S, H = len(NOT_FINITE), 2
    print(f"[q8 append, infinities] {code} {kv} P={P}", flush=True)
    cfg = B.Config(S, H, H, 8, 2 * P, 2, 2 * S, LK[kv], B.LOCKS_FP32, page_size=P)
    n = [len(rows) for rows in NOT_FINITE]
    cu = torch.tensor(np.cumsum([0] + n), dtype=torch.int32).cuda()
    x = torch.zeros(sum(n), H, D, dtype=DT[kv])
    for t, row in enumerate(r for rows in NOT_FINITE for r in rows):
        x[t, :, :len(row)] = torch.tensor(row, dtype=DT[kv])
    most = _most(code)
    want = torch.zeros(x.shape)
    want[torch.isnan(x)] = _nan_code(code)
    want[torch.isposinf(x)], want[torch.isneginf(x)] = most, -most
    tab = torch.randperm(2 * S, generator=torch.Generator().manual_seed(P)).int().reshape(S, 2)
    at = [(int(tab[s, 0]), i) for s in range(S) for i in range(n[s])]
    cache = C.alloc_q8_cache(cfg, code)
    pt, sl = tab.cuda(), torch.tensor(n, dtype=torch.int32).cuda()
    for _ in range(2):                        # (again: nothing changes)
        C.q8_append_kv(cfg, x.cuda(), x.cuda(), cache, pt, sl, cu_tokens=cu)
        for t, (b, i) in enumerate(at):
            _same(cache.k[b, :, i], want[t])
            _same(cache.v[b, :, i], want[t])
        assert not bool(cache.k_scale.any()) and not bool(cache.v_scale.any())
    q = torch.ones(S, H, D).cuda()
    out, lse = C.q8_dense_attend(cfg, q, cache, pt, sl, B.alloc_workspace(cfg))
    for s in range(S):
        if code == torch.int8 or not any(np.isnan(r).any() for r in NOT_FINITE[s]):
            assert not bool(out[s].any())
            assert bool(((lse[s] - float(np.log(n[s]))).abs() <= 2.0 ** -20).all())
    # a finite row of magnitude 3 to every sequence
    y = torch.full((S, H, D), -3.0, dtype=DT[kv])
    scale = torch.tensor(3.0) / 127 if code == torch.int8 else torch.tensor(2.0 ** -7)   # 3 <= 448 / 128
    C.q8_append_kv(cfg, y.cuda(), y.cuda(), cache, pt, sl + 1)
    for t, (b, i) in enumerate(at):
        _same(cache.k[b, :, i], want[t] * 0)
    for s in range(S):
        b = int(tab[s, 0])
        assert bool((cache.k_scale[b].cpu() == scale).all())
        _same(cache.v[b, :, n[s]], torch.full((H, D), -127.0 if code == torch.int8 else -384.0))
    # one of infinities after it: the largest codes, the scale stays
    z = torch.full((S, H, D), -INF, dtype=DT[kv])
    C.q8_append_kv(cfg, z.cuda(), z.cuda(), cache, pt, sl + 2)
    for s in range(S):
        b = int(tab[s, 0])
        assert bool((cache.k_scale[b].cpu() == scale).all())
        _same(cache.k[b, :, n[s] + 1], torch.full((H, D), -most))
        _same(cache.v[b, :, n[s]], torch.full((H, D), -127.0 if code == torch.int8 else -384.0))
