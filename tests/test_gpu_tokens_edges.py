"""GPU checks of the calls on single cached tokens (include/locks_tokens.h) where only a part of an
answer can go wrong: the roundings of bf16 outputs, and the LSE of rows that a NaN reaches; of workspaces that
serve smaller batches, of row ranges that do not ascend over very long tables, of masses whose
last sequences are empty or whose LSE holds a NaN, and of kept tokens in front of a sequence's start, and
of lists of nearly 2^31 entries."""
import numpy as np
import pytest
import torch

from paper_2607_24555_amd import locks as B
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


@pytest.mark.parametrize("extra", WIDE)
@pytest.mark.parametrize("new", TILES)
@pytest.mark.parametrize("q", ["bf16", "fp32"])
def test_lse_of_rows_that_a_nan_reaches(q, new, extra):
    """A NaN query head and a NaN key that is alone in its 32 tokens (the last one; a run, so that
    only the last row sees it): their rows' outputs and LSEs are NaN, all others keep their bits."""
    print(f"[nan] {q} new={new} extra={extra}", flush=True)
    L = 97 if new == 70 else 33
    b = Batch([L - new, 5], [new, new], P=16, q=q, kv=q, mask=None, seed=new, extra=extra)
    d = b.dev()
    o0, l0 = _attend(b)
    assert bool(torch.isfinite(o0).all()) and bool(torch.isfinite(l0).all())

    hit = torch.zeros(b.n, b.G * b.H, dtype=torch.bool)
    hit[0, 3] = hit[new // 2, 5] = hit[b.n - 1, 0] = True
    clean = d["q"].clone()
    d["q"][hit.cuda()] = float("nan")
    o1, l1 = _attend(b)
    d["q"].copy_(clean)
    assert bool(o1[hit].isnan().all()) and bool(l1[hit].isnan().all())
    assert torch.equal(o1[~hit], o0[~hit]) and torch.equal(l1[~hit], l0[~hit])

    d["k"][int(b.table[0, (L - 1) // 16]), :, (L - 1) % 16] = float("nan")
    o1, l1 = _attend(b)
    hit[:] = False
    hit[new - 1] = True
    assert bool(o1[hit].isnan().all()) and bool(l1[hit].isnan().all())
    assert torch.equal(o1[~hit], o0[~hit]) and torch.equal(l1[~hit], l0[~hit])


@pytest.mark.parametrize("extra", WIDE)
@pytest.mark.parametrize("new", TILES)
@pytest.mark.parametrize("q", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_lse_of_trees_with_bad_tokens(bad, q, new, extra):
    """A drafted token with a bad key: the LSE of the rows that see it is NaN (NaN) or not finite
    (infinity, whose products with a query are of both signs), of the others as before; a bad value
    changes no LSE."""
    b = Batch([40], [new], P=16, q=q, kv=q, seed=new, extra=extra)
    d = b.dev()
    o0, l0 = _attend(b)
    j = new // 2
    at = (int(b.table[0, (40 + j) // 16]), slice(None), (40 + j) % 16)
    sees = torch.tensor([bool(int(b.mask[i, j // 32]) >> (j % 32) & 1) for i in range(new)])
    assert bool(sees.any()) and not bool(sees.all())
    old = d["v"][at].clone()
    d["v"][at] = bad
    o1, l1 = _attend(b)
    d["v"][at] = old
    assert torch.equal(l1, l0) and torch.equal(o1[~sees], o0[~sees]) and not bool(torch.isfinite(o1[sees]).any())
    d["k"][at] = bad
    o1, l1 = _attend(b)
    assert torch.equal(o1[~sees], o0[~sees]) and torch.equal(l1[~sees], l0[~sees])
    assert not bool(torch.isfinite(o1[sees]).any())
    assert bool(l1[sees].isnan().all()) if bad != bad else not bool(torch.isfinite(l1[sees]).any())


@pytest.mark.parametrize("width,seqs", [(131072, [5, 4, 2, 1]), (40000, [7, 6, 3]), (300000, [3, 2, 1])])
def test_a_pick_workspace_serves_fewer_sequences(width, seqs):
    """Whose lists are cut into more chunks."""
    cfg = B.Config(seqs[0], 32, 8, 8, 256, width // 16, 8, page_size=16)
    ws = T.alloc_pick_workspace(cfg)
    ws.fill_(255)
    g = torch.Generator().manual_seed(width)
    x = torch.rand(seqs[0], 8, width, generator=g)
    lens = torch.tensor([width - 977 * s for s in range(seqs[0])], dtype=torch.int32)
    for s in seqs:
        print(f"[pick] {s} of {seqs[0]} x 8 lists of {width}", flush=True)
        cfg.num_seqs = s
        got = T.pick_tokens(cfg, x[:s].cuda(), lens[:s].cuda(), 500, 4, 64, ws).cpu()
        for q in range(s):
            assert got[q, 7].tolist() == R.pick(x[q, 7].numpy(), int(lens[q]), 500, 4, 64)


def test_a_tree_workspace_serves_fewer_sequences():
    """With the same tokens between them, so that their tiles are larger."""
    b = Batch([60] * 16, [4] * 16, seed=3, extra=80)
    ws = T.alloc_tree_workspace(b.cfg, b.n)
    ws.fill_(255)
    for seqs, new in ((16, 4), (8, 8), (4, 16), (1, 64)):
        print(f"[tree] {seqs} x {new}", flush=True)
        one = Batch([60] * seqs, [new] * seqs, seed=seqs, extra=80)
        d = one.dev()
        got = T.tree_attend(one.cfg, d["q"], d["k"], d["v"], d["pt"], d["sl"], ws, cu_tokens=d["cu"], mask=d["mask"])
        one.check(got=(got[0].cpu(), got[1].cpu()))


def test_tree_row_ranges_that_do_not_ascend_over_long_tables():
    """Ten of 19 sequences claim all rows: ten times the 256-row tiles that ascending ranges have, over
    14 M tokens each, whose weighted units in all KV heads pass 2^31.  The first ones are computed.
    Every page is the same block; of zero keys and small whole values every sum is below 2^24
    and exact, so that an output has a reciprocal's and a product's rounding, and an LSE below 32 at
    most two steps of 2^-19 of a logarithm."""
    S, H, P, pages, n = 19, 8, 64, 220000, 2560
    L = pages * P
    assert (S // 2 + 1) * (n // 256) * pages * H * 20 >= 1 << 31 and S * H * L < 1 << 31
    cfg = B.Config(S, H, H, 8, 256, pages, 1, page_size=P)
    g = torch.Generator().manual_seed(1)
    k = torch.zeros(1, H, P, D, dtype=torch.bfloat16).cuda()
    v = torch.randint(0, 2, (1, H, P, D), generator=g).bfloat16()
    q = torch.randn(n, H, D, generator=g).bfloat16().cuda()
    table = torch.zeros(S, pages, dtype=torch.int32).cuda()
    lens = torch.full((S,), L, dtype=torch.int32).cuda()
    cu = torch.tensor([n * (s & 1) for s in range(S + 1)], dtype=torch.int32).cuda()
    print("[tree] row ranges that do not ascend, 14 M tokens", flush=True)
    out, lse = T.tree_attend(cfg, q, k, v.cuda(), table, lens, T.alloc_tree_workspace(cfg, n), cu_tokens=cu)
    torch.cuda.synchronize()
    seen = L - n + 1 + torch.arange(n)                          # of row i, the first ones
    count = (seen[:, None] // P + (torch.arange(P) < seen[:, None] % P)).double()
    want = torch.stack([count @ v[0, h].double() for h in range(H)], 1) / seen[:, None, None]
    assert bool(((out.cpu().double() - want).abs() <= 2.0 ** -22 * want).all())
    assert bool(((lse.cpu().double() - torch.log(seen.double())[:, None]).abs() <= 2.0 ** -18).all())


@pytest.mark.parametrize("H", [1, 3])
@pytest.mark.parametrize("q", ["bf16", "fp32"])
def test_mass_of_many_sequences_whose_last_ones_are_empty(q, H):
    """Beyond 512 sequences a block's lists may end with ones that have no tokens or no rows: what it
    requests behind the last unit is that unit's again, not theirs."""
    print(f"[mass] 1,700 sequences, {H} heads, {q}", flush=True)
    lens = [40 + s % 90 if s < 600 else 0 if s % 2 else 5 for s in range(1700)]
    new = [1 if s < 600 or (s % 2 and s % 3) else 0 for s in range(1700)]
    b = Batch([max(0, L - n) for L, n in zip(lens, new)], [min(L, n) for L, n in zip(lens, new)], H=H, G=2, q=q, kv=q,
              mask=None, seed=H)
    d = b.dev()
    cu = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).int().cuda()  # (some empty sequences have a row)
    n = int(cu[-1])
    qs = torch.zeros(n, 2 * H, D, dtype=d["q"].dtype).cuda()
    rows = torch.tensor([i for i, s in enumerate(s for s, k in enumerate(new) if k) if lens[s]])
    qs[rows.cuda()] = d["q"][:len(rows)]
    _, lse = T.tree_attend(b.cfg, qs, d["k"], d["v"], d["pt"], d["sl"], T.alloc_tree_workspace(b.cfg, n), cu_tokens=cu)
    mass = T.token_mass(b.cfg, qs, lse, d["k"], d["pt"], d["sl"], T.alloc_mass(b.cfg), cu_tokens=cu)
    one = T.alloc_mass(b.cfg)
    for s0 in range(0, 600, 300):             # as few sequences at once as are counted
        c = B.Config(300, 2 * H, H, 8, 256, b.cfg.max_pages_per_seq, b.cfg.num_blocks, b.cfg.kv_dtype, b.cfg.q_dtype)
        T.token_mass(c, d["q"][s0:s0 + 300], lse[rows.cuda()][s0:s0 + 300].contiguous(), d["k"],
                     d["pt"][s0:s0 + 300], d["sl"][s0:s0 + 300], one[s0:s0 + 300])
    torch.cuda.synchronize()
    assert bool((mass[600:] == 0).all()) and bool((mass[:600] != 0).any())
    assert torch.equal(mass, one)


@pytest.mark.parametrize("past,new,extra", [(40, 20, 1), (40, 20, 3000), (30, 70, 1), (30, 70, 3000)])
@pytest.mark.parametrize("q", ["bf16", "fp32"])
@pytest.mark.parametrize("mask", ["tree", None])
def test_mass_of_nan_rows(mask, q, past, new, extra):
    """One NaN in the LSE makes the masses of exactly what its row sees NaN, of its head's KV head
    (rows shared by a block's waves: 70 new tokens in a short table; and not)."""
    print(f"[mass nan] {past}+{new} extra={extra} {q} {mask}", flush=True)
    b = Batch([past], [new], P=16, q=q, kv=q, mask=mask, seed=new, extra=extra)
    d = b.dev()
    _, lse = _attend(b)

    def mass(l):
        m = T.alloc_mass(b.cfg)
        T.token_mass(b.cfg, d["q"], l.cuda(), d["k"], d["pt"], d["sl"], m, cu_tokens=d["cu"], mask=d["mask"])
        return m.cpu()
    want = mass(lse)
    assert bool(torch.isfinite(want).all())
    i, head = new - 3, 6                      # of KV head 1
    lse[i, head] = float("nan")
    got = mass(lse)
    sees = torch.from_numpy(R.sees(new, past + new, None if b.mask is None else b.mask.numpy())[i])
    nan = torch.zeros_like(want, dtype=torch.bool)
    nan[0, 1, :past + new] = sees
    assert torch.equal(got.isnan(), nan) and torch.equal(got[~nan], want[~nan])


@pytest.mark.parametrize("kv", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [6, 900])
def test_keep_in_front_of_the_first_token(kv, n):
    """A negative start: entries whose new place lies in front of the sequence are left out, the
    others move, and the length counts all of them."""
    print(f"[keep] start < 0, {n} entries {kv}", flush=True)
    g = torch.Generator().manual_seed(n)
    H, P, L, start = 2, 16, 2000, [-4, -1000]
    table, nb = R.table_of([L, L], P, g)
    dt, kind = (torch.bfloat16, B.LOCKS_BF16) if kv == "bf16" else (torch.float32, B.LOCKS_FP32)
    cfg = B.Config(2, 4 * H, H, 8, 256, table.shape[1], nb, kind, kind, page_size=P)
    k, v = (torch.randn(nb, H, P, D, generator=g).to(dt) for _ in range(2))
    mass = torch.rand(2, H, table.shape[1] * P, generator=g)
    kept = torch.stack([torch.stack([torch.randperm(L, generator=g)[:n].sort()[0] for _ in range(H)])
                        for _ in range(2)]).int()
    dk, dv, dm = k.cuda(), v.cuda(), mass.cuda()
    got = T.keep_tokens(cfg, kept.cuda(), dk, dv, table.cuda(), start=torch.tensor(start, dtype=torch.int32).cuda(),
                        mass=dm)
    wk, wv, wm = k.clone(), v.clone(), mass.clone()
    for s in range(2):
        for h in range(H):
            for i in range(max(0, -start[s]), n):
                src, dst = int(kept[s, h, i]), start[s] + i
                a, b = int(table[s, src // P]), int(table[s, dst // P])
                wk[b, h, dst % P], wv[b, h, dst % P] = k[a, h, src % P], v[a, h, src % P]
                wm[s, h, dst] = mass[s, h, src]
    assert got.tolist() == [x + n for x in start]
    assert torch.equal(dk.cpu(), wk) and torch.equal(dv.cpu(), wv) and torch.equal(dm.cpu(), wm)


def test_pick_of_the_longest_list():
    """n_keep at its limit: the fill's last step passes 2^31."""
    n = (1 << 31) - 1
    cfg = B.Config(1, 1, 1, 8, 256, 3, 8, page_size=16)
    print("[pick] 2^31 - 1 kept", flush=True)
    got = T.pick_tokens(cfg, torch.rand(1, 1, 48).cuda(), torch.tensor([37], dtype=torch.int32).cuda(), n, 0, 0,
                        T.alloc_pick_workspace(cfg))[0, 0]
    assert got[:37].tolist() == list(range(37))
    for a in range(37, n, 1 << 28):
        assert bool((got[a:a + (1 << 28)] == -1).all())


@pytest.mark.parametrize("with_mass", [False, True])
def test_keep_of_the_longest_list(with_mass):
    """2^31 - 1 entries, none of which moves but one at the front: the rounds' ends pass 2^31."""
    n = (1 << 31) - 1
    cfg = B.Config(1, 1, 1, 8, 256, 4, 5, page_size=16)
    k, v = (torch.randn(5, 1, 16, D).bfloat16() for _ in range(2))
    mass = torch.rand(1, 1, 64) if with_mass else None
    kept = torch.zeros(1, 1, n, dtype=torch.int32, device="cuda")
    kept[0, 0, 3] = 50
    table = torch.tensor([[2, 0, 4, 1]], dtype=torch.int32).cuda()
    dk, dv, dm = k.cuda(), v.cuda(), mass.cuda() if with_mass else None
    print("[keep] 2^31 - 1 entries", flush=True)
    got = T.keep_tokens(cfg, kept, dk, dv, table, mass=dm)
    assert got.tolist() == [n]
    k[2, 0, 3], v[2, 0, 3] = k[1, 0, 2], v[1, 0, 2]
    assert torch.equal(dk.cpu(), k) and torch.equal(dv.cpu(), v)
    if with_mass:
        mass[0, 0, 3] = mass[0, 0, 50]
        assert torch.equal(dm.cpu(), mass)


@pytest.mark.parametrize("mask", ["tree", None])
def test_steps_without_new_tokens(mask):
    """Of some sequences, and of all: nothing is written."""
    b = Batch([30, 0, 700], [0, 0, 3], mask=mask, seed=1)
    b.check()
    d = b.d
    none = torch.zeros(4, dtype=torch.int32).cuda()
    out, lse = T.tree_attend(b.cfg, d["q"][:0], d["k"], d["v"], d["pt"], d["sl"], d["ws"], cu_tokens=none,
                             mask=None if mask is None else d["mask"][:0])
    assert out.shape == (0, 8, D) and lse.shape == (0, 8)
    mass = torch.full((3, 2, b.cfg.max_pages_per_seq * 16), 2.0).cuda()
    T.token_mass(b.cfg, d["q"][:0], lse, d["k"], d["pt"], d["sl"], mass, cu_tokens=none, decay=0.5)
    assert bool((mass == 2.0).all())
    kept = torch.full((3, 1, 5), -1, dtype=torch.int32).cuda()
    k, v = d["k"].clone(), d["v"].clone()
    lens = T.keep_tokens(b.cfg, kept, d["k"], d["v"], d["pt"], start=d["sl"], mass=mass)
    assert torch.equal(lens, d["sl"]) and torch.equal(d["k"], k) and torch.equal(d["v"], v) and bool((mass == 2.0).all())


def test_calls_on_a_stream_that_is_not_the_current_one():
    """The four calls in order on one side stream, their inputs made on it, equal the current
    stream's."""
    def step(b, d, stream):
        mass, pws = T.alloc_mass(b.cfg), T.alloc_pick_workspace(b.cfg)
        torch.cuda.synchronize()
        out, lse = T.tree_attend(b.cfg, d["q"], d["k"], d["v"], d["pt"], d["sl"], d["ws"], cu_tokens=d["cu"],
                                 mask=d["mask"], stream=stream)
        T.token_mass(b.cfg, d["q"], lse, d["k"], d["pt"], d["sl"], mass, cu_tokens=d["cu"], mask=d["mask"],
                     decay=0.5, stream=stream)
        ids = T.pick_tokens(b.cfg, mass, d["sl"], 64, 4, 16, pws, stream=stream)
        lens = T.keep_tokens(b.cfg, ids, d["k"], d["v"], d["pt"], mass=mass, stream=stream)
        torch.cuda.synchronize()
        return out, lse, mass, ids, lens, d["k"], d["v"]
    got = []
    for stream in (None, torch.cuda.Stream()):
        b = Batch([9000, 300], [20, 9], seed=5)
        got.append(step(b, b.dev(), stream))
    assert all(torch.equal(x, y) for x, y in zip(*got))
