"""GPU checks of the calls on single cached tokens (include/locks_tokens.h) where only a part of an
answer can go wrong: the roundings of bf16 outputs."""
import numpy as np
import pytest
import torch

from paper_2607_24555_amd import tokens as T
from tests import _tokens_reference as R
from tests.test_gpu_tokens import D, Batch

pytestmark = pytest.mark.gpu

# new tokens of 4 heads a group: 20, 40, 100 and 280 rows, so tiles of 32, 64, 128 and 256
TILES = [5, 10, 25, 70]
WIDE = [1, 80]          # pages of 16 tokens more than needed: an item a block, or cut into shares


def _attend(b, out="fp32", v=None):
    d = b.d
    o = torch.empty(b.n, b.G * b.H, D, dtype=torch.bfloat16 if out == "bf16" else torch.float32).cuda()
    got, lse = T.tree_attend(b.cfg, d["q"], d["k"], d["v"] if v is None else v, d["pt"], d["sl"], d["ws"],
                             cu_tokens=d["cu"], mask=d["mask"], out=o)
    torch.cuda.synchronize()
    return got.cpu(), lse.cpu()


@pytest.mark.parametrize("extra", WIDE)
@pytest.mark.parametrize("past", [0, 11, 300])
@pytest.mark.parametrize("new", TILES)
def test_bf16_outputs_are_the_fp32_ones_rounded(new, past, extra):
    """Whatever the tile.  Two terms of a weight are within 2^-16 of it (a bf16 rounding is within
    2^-8, that of its rest within 2^-8 of 2^-8), three within 2^-24; the sums over N tokens of the
    two calls have N / 8 + 64 roundings to 2^-23 between them; the output's own is within 2^-8.  What
    the first three are relative to is the attention over |v|."""
    print(f"[round] past={past} new={new} extra={extra}", flush=True)
    b = Batch([past, past // 3], [new, new], P=16, seed=new + past, extra=extra)
    b.dev()
    want, l32 = _attend(b)
    got, l16 = _attend(b, "bf16")
    size, _ = _attend(b, v=b.d["v"].abs())
    assert torch.equal(l32, l16)
    off = (got.double() - want.double()).abs()
    bound = 2.0 ** -8 * 1.01 * want.double().abs() + (2.0 ** -16 * 1.01 + (max(b.lens) / 8 + 64) * 2.0 ** -23) * size.double()
    assert bool((off <= bound).all()), float((off / bound).max())


@pytest.mark.parametrize("rows", [(1, 200), (1, 40), (6, 300)])
def test_bf16_rows_beside_others_are_as_exact_as_alone(rows):
    """One new token beside a prompt's piece: two calls, the second of its sequence alone, whose
    logits, sums and orders differ, within the bounds of both."""
    few, many = rows
    print(f"[round] {few} beside {many}", flush=True)
    b = Batch([400, 90], [few, many], mask=None, seed=few + many)
    b.dev()
    both, lse = _attend(b, "bf16")
    size, _ = _attend(b, v=b.d["v"].abs())
    for s, h, at, q, K, V, ok in b.units():
        want, wl, big = R.attend(q, K, V, ok)
        heads = slice(h * b.G, (h + 1) * b.G)
        zmax = np.abs(q @ K.T).max() / np.sqrt(D)
        e = 2 * (130 * 2.0 ** -24 * big + 2.0 ** -22 * (1 + zmax)) + (b.lens[s] + 64) * 2.0 ** -23
        bound = 2.0 ** -8 * 1.01 * np.abs(want) + (e + 2.0 ** -16) * 1.01 * size[at, heads].double().numpy()
        assert (np.abs(both[at, heads].double().numpy() - want) <= bound).all()
