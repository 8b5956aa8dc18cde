"""GPU checks of the calls on single cached tokens (include/locks_tokens.h) against the plain
64-bit definitions of tests/_tokens_reference.py.

Bounds.  A logit is a sum of 128 products in float32, in any order, off by at most
dz = 130 2^-24 sum |q k| / sqrt d, its scaling and the hardware's power of two by 2^-22 (1 + |z|)
more; N weights are added with N + 64 roundings.  So with e = 2 (dz + 2^-22 (1 + |z|max)) +
(N + 64) 2^-23 an output is within (e + w) max |v| of the 64-bit one, w the weights' own
rounding in the product with the values (their sum is of unrounded ones): half a bf16 step, 2^-8
of each, for bf16 outputs, three terms (2^-24; 2^-22 is allowed) for fp32 ones; and a bf16 output
is half a step (2^-8 of itself) further off; the LSE within e + 2^-22 (|lse| + 1).  A token's
mass is a sum of R weights exp(z - lse), each within dz + 2^-21 (1 + |z| + |lse|) of itself,
added with R + 64 roundings, and its old part one product and one sum."""
import itertools

import numpy as np
import pytest
import torch

from paper_2607_24555_amd import cache as C
from paper_2607_24555_amd import locks as B
from paper_2607_24555_amd import tokens as T
from tests import _tokens_reference as R

pytestmark = pytest.mark.gpu
D = 128
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
LK = {"bf16": B.LOCKS_BF16, "fp32": B.LOCKS_FP32}


class Batch:
    """Sequences of `past` cached and `new` tokens, whose rows are all in the cache."""

    def __init__(self, past, new, H=2, G=4, P=16, q="bf16", kv="bf16", pad=0, seed=0, mask="tree", ragged=True,
                 extra=1):
        g = self.gen = torch.Generator().manual_seed(seed)
        self.past, self.new, self.H, self.G, self.P, self.qt, self.kt = past, new, H, G, P, q, kv
        self.lens = [a + b for a, b in zip(past, new)]
        self.table, nb = R.table_of(self.lens, P, g, extra=extra)
        S = len(past)
        self.cfg = B.Config(S, G * H, H, 8, max(256, 2 * P), self.table.shape[1], nb, LK[kv], LK[q], page_size=P)
        self.cu = [0]
        for t in new:
            self.cu.append(self.cu[-1] + t)
        self.n = self.cu[-1] + pad
        self.k = torch.randn(nb, H, P, D, generator=g)
        self.k[..., 5] += 6.0
        self.k, self.v = self.k.to(DT[kv]), torch.randn(nb, H, P, D, generator=g).to(DT[kv])
        self.q = (1.5 * torch.randn(self.n, G * H, D, generator=g)).to(DT[q])
        self.mask = None
        if mask is not None:
            parents = []
            for t in new:
                for i in range(t):
                    lo = max(-1, i - 7)
                    parents.append(int(torch.randint(lo, i, (1,), generator=g)) if mask == "tree" else i - 1)
            self.mask = T.tree_mask(parents, self.cu, device="cpu")[0]
            if pad:
                self.mask = torch.cat([self.mask, torch.full((pad, self.mask.shape[1]), -1, dtype=torch.int32)])
        self.ragged = ragged

    def garbage(self):
        """NaN and infinity in every row that is no token's, of live pages too."""
        used = torch.zeros(self.k.shape[0], self.P, dtype=torch.bool)
        for s, L in enumerate(self.lens):
            for t in range(L):
                used[int(self.table[s, t // self.P]), t % self.P] = True
        for c, x in ((self.k, float("nan")), (self.v, float("inf"))):
            c.masked_fill_(~used[:, None, :, None], x)
        return self

    def dev(self):
        wide = torch.full((self.n, self.G * self.H + 3, D), float("nan"), dtype=self.q.dtype).cuda()
        wide[:, 1:1 + self.G * self.H] = self.q.cuda()
        self.d = dict(q=wide[:, 1:1 + self.G * self.H], k=self.k.cuda(), v=self.v.cuda(), pt=self.table.cuda(),
                      sl=torch.tensor(self.lens, dtype=torch.int32).cuda(),
                      cu=torch.tensor(self.cu, dtype=torch.int32).cuda() if self.ragged else None,
                      mask=None if self.mask is None else self.mask.cuda(),
                      ws=T.alloc_tree_workspace(self.cfg, self.n))
        return self.d

    def units(self):
        """(sequence, head, rows, q [n][G][128], K, V, sees) in 64 bits."""
        for s, h in itertools.product(range(len(self.past)), range(self.H)):
            a, b = self.cu[s], self.cu[s + 1]
            K, V = (R.rows_of(c, self.table[s], h, self.lens[s], self.P) for c in (self.k, self.v))
            q = self.q[a:b, h * self.G:(h + 1) * self.G].double().numpy()
            m = None if self.mask is None else self.mask[a:b].numpy()
            yield s, h, slice(a, b), q, K, V, R.sees(b - a, self.lens[s], m)

    def run(self, out="fp32", **kw):
        d = self.dev()
        o = torch.full((self.n, self.G * self.H, D), 7.0, dtype=DT[out]).cuda()
        lse = torch.full((self.n, self.G * self.H), 7.0).cuda()
        got = T.tree_attend(self.cfg, d["q"], d["k"], d["v"], d["pt"], d["sl"], d["ws"], cu_tokens=d["cu"],
                            mask=d["mask"], out=o, out_lse=lse, **kw)
        torch.cuda.synchronize()
        assert got[0] is o and got[1] is lse
        return o.cpu(), lse.cpu()

    def check(self, out="fp32", got=None):
        o, lse = self.run(out) if got is None else got
        for s, h, rows, q, K, V, ok in self.units():
            want, wl, big = R.attend(q, K, V, ok)
            heads = slice(h * self.G, (h + 1) * self.G)
            go, gl = o[rows, heads].double().numpy(), lse[rows, heads].double().numpy()
            none = np.isneginf(wl)
            assert (np.isneginf(gl) == none).all() and (go[none] == 0).all()
            if none.all():
                continue
            N = self.lens[s]
            zmax = np.abs(q @ K.T).max() / np.sqrt(D)
            e = 2 * (130 * 2.0 ** -24 * big + 2.0 ** -22 * (1 + zmax)) + (N + 64) * 2.0 ** -23
            w = 2.0 ** -8 if out == "bf16" else 2.0 ** -22
            bound = (e + w) * np.abs(V[np.isfinite(V).all(1)]).max()
            if out == "bf16":
                bound = bound + 2.0 ** -8 * np.abs(want) * 1.01
            assert (np.abs(go - want) <= bound)[~none].all(), (s, h, np.abs(go - want).max(), np.max(bound))
            assert (np.abs(gl - wl)[~none] <= (e + 2.0 ** -22 * (np.abs(wl) + 1))[~none]).all()
        pad = slice(self.cu[-1], None)
        assert bool((o[pad] == 7).all()) and bool((lse[pad] == 7).all())
        return o, lse


SHAPES = [
    # past, new: one token of nothing, page and tile borders, ragged trees, empty sequences
    ([0], [1]), ([15], [1]), ([63], [1]), ([64], [2]), ([127, 128, 129], [5, 1, 31]),
    ([0, 7, 300, 40], [33, 0, 16, 70]), ([61, 0], [67, 130]), ([500], [8]), ([1000, 3], [3, 40]),
    ([0] * 40, [1, 0, 2, 5, 17] * 8),
]


@pytest.mark.parametrize("mask", ["tree", "run-mask", None])
@pytest.mark.parametrize("q,kv,out", [("bf16", "bf16", "fp32"), ("bf16", "bf16", "bf16"), ("fp32", "fp32", "fp32"),
                                      ("bf16", "fp32", "fp32"), ("fp32", "bf16", "bf16")])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_tree_attend(shape, q, kv, out, mask):
    past, new = SHAPES[shape]
    G, P = (4, 7, 1, 16, 3)[shape % 5], (16, 32, 64)[shape % 3]
    print(f"[tree] {past} {new} G={G} P={P} {q}/{kv}->{out} mask={mask}", flush=True)
    Batch(past, new, G=G, P=P, q=q, kv=kv, pad=3, seed=shape, mask=mask).garbage().check(out)


@pytest.mark.parametrize("G", range(1, 17))
def test_tree_groups(G):
    print(f"[tree] G={G}", flush=True)
    Batch([70, 201], [9, 23], G=G, H=1, P=32, seed=G, pad=2).check("bf16" if G % 2 else "fp32")


@pytest.mark.parametrize("rows", [(40, 1), (150, 3), (700, 2)])
@pytest.mark.parametrize("q", ["bf16", "fp32"])
def test_tree_many_sequences(rows, q):
    """More sequences than threads of a block; one token each, without cu_tokens too."""
    S, n = rows
    print(f"[tree] S={S} n={n} {q}", flush=True)
    past = [(37 * s) % 90 for s in range(S)]
    b = Batch(past, [n] * S, H=1, G=2, q=q, kv=q, seed=S, mask=None)
    got = b.check()
    if n == 1:
        b.ragged = False
        again = b.run()
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("new,G,q", [(6, 8, "bf16"), (10, 8, "bf16"), (17, 8, "bf16"), (10, 8, "fp32"), (1, 16, "fp32")])
def test_tree_more_tiles_than_are_cut_into_shares(new, G, q):
    """520 sequences: every tile size with a block for each item."""
    print(f"[tree] 520 x {new} tokens, G={G} {q}", flush=True)
    b = Batch([(29 * s) % 50 for s in range(520)], [new - s % 2 if new > 1 else 1 for s in range(520)], H=1, G=G, P=16,
              q=q, kv=q, seed=new, pad=1)
    b.check("bf16" if new == 17 else "fp32")


def test_tree_row_ranges_that_do_not_ascend():
    # every second sequence claims all rows, over the same pages: 750 tiles where ascending ranges
    # would have 305 at most
    S, n = 300, 40
    b = Batch([20], [n], seed=37, extra=40)   # (tables of more than 512 tokens)
    want, lse = b.run()
    d = dict(b.d)
    b.cfg.num_seqs = S
    pt, sl = d["pt"].expand(S, -1).contiguous(), d["sl"].expand(S).contiguous()
    cu = torch.tensor([n * (s & 1) for s in range(S + 1)], dtype=torch.int32).cuda()
    ws, out = T.alloc_tree_workspace(b.cfg, n), torch.full_like(want, 7.0).cuda()
    _, l = T.tree_attend(b.cfg, d["q"], d["k"], d["v"], pt, sl, ws, cu_tokens=cu, mask=d["mask"], out=out)
    m = T.token_mass(b.cfg, d["q"], l, d["k"], pt, sl, T.alloc_mass(b.cfg), cu_tokens=cu, mask=d["mask"])
    torch.cuda.synchronize()
    assert (m[1::2] == 0).all() and (m[::2] == m[0]).all()
    b.cfg.num_seqs = 1
    b.check(got=(out.cpu(), l.cpu()))


@pytest.mark.parametrize("new,G", [(300, 1), (300, 7), (520, 2)])
@pytest.mark.parametrize("bad", [None, float("nan")])
def test_tree_masks_wider_than_the_block_holds(new, G, bad):
    """Trees of more than 192 tokens, whose masks are read from memory, over several tiles."""
    b = Batch([77], [new], H=1, G=G, P=64, seed=G)
    o0, l0 = b.check("bf16")
    if bad is not None:
        j = new - 40
        b.v[int(b.table[0, (77 + j) // 64]), :, (77 + j) % 64, 5] = bad
        o1, l1 = b.run("bf16")
        sees = np.array([bool(int(b.mask[i, j // 32]) >> (j % 32) & 1) for i in range(new)])
        assert sees.any() and torch.equal(o0[~sees], o1[~sees]) and bool(o1[sees][..., 5].isnan().all())


def test_tree_rows_do_not_depend_on_others():
    """A row's bits are the same whatever the other rows of its tile are."""
    b = Batch([600, 90], [40, 9], seed=8)
    o0, l0 = b.run()
    b.q[::2] *= 30
    o1, l1 = b.run()
    assert torch.equal(o0[1::2], o1[1::2]) and torch.equal(l0[1::2], l1[1::2])
    assert not torch.equal(o0[::2], o1[::2])


def test_tree_equals_dense_attention_for_single_tokens():
    b = Batch([900, 64, 4000], [1, 1, 1], G=8, mask=None, ragged=False)
    o, lse = b.check()
    ws = B.alloc_workspace(b.cfg)
    want, wl = B.dense_attend(b.cfg, b.d["q"].contiguous(), b.d["k"], b.d["v"], b.d["pt"], b.d["sl"], ws)
    # (the other kernel's weights are two bf16 terms)
    assert (want.cpu() - o).abs().max() < 2.0 ** -12 and (wl.cpu() - lse).abs().max() < 2.0 ** -14


@pytest.mark.parametrize("q", ["bf16", "fp32"])
def test_tree_rows_that_see_nothing(q):
    """Empty masks, sequences of length 0 or shorter than their rows, and masks narrower than
    the tree (tokens from 32 words on are unseen) and wider."""
    b = Batch([0, 0, 9], [40, 3, 35], q=q, kv=q, seed=5)
    b.mask[0] = 0
    b.mask[7] = 0
    b.check("bf16")
    b.mask = b.mask[:, :1].contiguous()
    b.check()
    b.mask = torch.cat([b.mask, torch.full((b.n, 3), -1, dtype=torch.int32)], 1).contiguous()
    b.check()
    d = b.dev()
    d["sl"] = torch.tensor([0, 2, -5], dtype=torch.int32).cuda()
    out, lse = T.tree_attend(b.cfg, d["q"], d["k"], d["v"], d["pt"], d["sl"], d["ws"], cu_tokens=d["cu"])
    out, lse = out.cpu(), lse.cpu()
    assert bool((lse[:41] == -np.inf).all()) and bool((out[:41] == 0).all())   # token 0 of three is before the start
    assert bool(torch.isfinite(lse[41:43]).all()) and bool((lse[43:] == -np.inf).all())


@pytest.mark.parametrize("q", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [7, 40, 200])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_tree_unseen_tokens_do_not_reach_a_row(q, new, bad):
    """A branch whose keys and values are not finite: the rows that do not see it are the same
    as with finite ones, those that do are not finite."""
    b = Batch([50], [new], H=2, G=4, P=16, q=q, kv=q, seed=new)
    o0, l0 = b.check()
    L = b.lens[0]
    hit = [1, new // 2, new - 2]
    for j in hit:
        t = 50 + j
        for c in (b.k, b.v):
            c[int(b.table[0, t // 16]), :, t % 16, 3::5] = bad
    o1, l1 = b.run()
    words = b.mask.numpy()
    sees = np.array([any(int(words[i, j // 32]) >> (j % 32) & 1 for j in hit) for i in range(new)])
    assert sees.any() and not sees.all()
    assert torch.equal(o0[~sees], o1[~sees]) and torch.equal(l0[~sees], l1[~sees])
    if not np.isfinite(bad):
        assert not bool(torch.isfinite(o1[sees]).all(-1).any())


@pytest.fixture
def wide(monkeypatch):
    """Tables of 1,024 tokens more than the sequences have: short ones' items are blocks', these
    are cut into shares."""
    table_of = R.table_of
    monkeypatch.setattr(R, "table_of", lambda lens, P, g, spare=3, extra=1: table_of(lens, P, g, spare, extra + 1024 // P))


@pytest.mark.parametrize("mask", ["tree", None])
@pytest.mark.parametrize("q,kv,out", [("bf16", "bf16", "fp32"), ("bf16", "bf16", "bf16"), ("fp32", "fp32", "fp32"),
                                      ("bf16", "fp32", "fp32"), ("fp32", "bf16", "bf16")])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_tree_wide_tables(wide, shape, q, kv, out, mask):
    test_tree_attend(shape, q, kv, out, mask)


@pytest.mark.parametrize("q", ["bf16", "fp32"])
def test_tree_wide_tables_of_many_sequences(wide, q):
    for rows in ((40, 1), (150, 3), (700, 2)):
        test_tree_many_sequences(rows, q)


@pytest.mark.parametrize("G", [1, 5, 8, 13, 16])
def test_tree_wide_tables_groups(wide, G):
    test_tree_groups(G)


@pytest.mark.parametrize("new,G", [(300, 1), (300, 7), (520, 2)])
@pytest.mark.parametrize("bad", [None, float("nan")])
def test_tree_wide_tables_and_masks(wide, new, G, bad):
    test_tree_masks_wider_than_the_block_holds(new, G, bad)


@pytest.mark.parametrize("q", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [7, 40, 200])
def test_tree_wide_tables_unseen_tokens(wide, q, new):
    for bad in (float("nan"), float("inf"), -float("inf"), 3e38):
        test_tree_unseen_tokens_do_not_reach_a_row(q, new, bad)


@pytest.mark.parametrize("q", ["bf16", "fp32"])
def test_tree_wide_tables_rows_that_see_nothing(wide, q):
    test_tree_rows_that_see_nothing(q)


@pytest.mark.parametrize("q", ["bf16", "fp32"])
@pytest.mark.parametrize("pages", [8, 9, 16, 17, 31, 32, 33])
def test_tree_full_tables_around_the_cut(q, pages):
    """Sequences that fill tables of 128 to 528 tokens."""
    L = 16 * pages
    for new in ([5, 5], [40, 33], [100, 77]):
        Batch([L - new[0], L - 3 - new[1]], new, q=q, kv=q, seed=pages, extra=0).check("bf16" if pages % 2 else "fp32")


@pytest.mark.parametrize("q,out", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("past,new,H,G", [([30000], [6], 2, 4), ([9000, 17, 20011], [50, 64, 31], 2, 4),
                                          ([5000], [700], 1, 4), ([120001], [16], 1, 16), ([2000], [40], 8, 2)])
def test_tree_long(q, out, past, new, H, G):
    """Long lists, cut over many blocks; the reference on the GPU in 64 bits."""
    print(f"[tree long] {past} {new} {H}x{G} {q}->{out}", flush=True)
    b = Batch(past, new, H=H, G=G, P=(16, 64)[H % 2], q=q, kv=q, seed=len(past), extra=40)
    o, lse = b.run(out)
    for s, h in itertools.product(range(len(past)), range(H)):
        L, n = b.lens[s], new[s]
        pages = b.table[s, :-(-L // b.P)].long().cuda()
        K, V = (b.d[x][pages, h].reshape(-1, D)[:L].double() for x in "kv")
        rows = slice(b.cu[s], b.cu[s + 1])
        qd = b.d["q"][rows, h * G:(h + 1) * G].double()
        ok = torch.ones(n, L, dtype=torch.bool)
        ok[:, L - n:] = torch.from_numpy(R.sees(n, n, b.mask[rows].numpy()))
        z = torch.matmul(qd.reshape(n * G, D), K.t().contiguous()).reshape(n, G, L) / np.sqrt(D)
        z = z.masked_fill(~ok.cuda()[:, None], -np.inf)
        wl = torch.logsumexp(z, -1)
        want = torch.matmul(torch.exp(z - wl[..., None]).reshape(n * G, L), V).reshape(n, G, D)
        big = float((qd.abs().reshape(n * G, D) @ K.abs().t().contiguous()).max()) / np.sqrt(D)
        zmax = float(z[torch.isfinite(z)].abs().max())
        # sums of N weights over blocks: no lane adds more than N / 16 in a row
        e = 2 * (130 * 2.0 ** -24 * big + 2.0 ** -22 * (1 + zmax)) + (L / 16 + 256) * 2.0 ** -23
        w = 2.0 ** -8 if out == "bf16" else 2.0 ** -22
        heads = slice(h * G, (h + 1) * G)
        bound = (e + w) * float(V.abs().max()) + (2.0 ** -8 * 1.01 * want.abs() if out == "bf16" else 0)
        assert bool(((o[rows, heads].cuda().double() - want).abs() <= bound).all())
        assert bool(((lse[rows, heads].cuda().double() - wl).abs() <= e + 2.0 ** -22 * (wl.abs() + 1)).all())


def test_tree_table_checks():
    b = Batch([100, 40], [5, 9])
    want = b.run()
    d = b.d
    before = B.set_table_checks(True)
    try:
        got = T.tree_attend(b.cfg, d["q"], d["k"], d["v"], d["pt"], d["sl"], d["ws"], cu_tokens=d["cu"], mask=d["mask"])
        assert torch.equal(got[0].cpu(), want[0]) and B.table_errors(b.cfg, d["ws"]) == (0, [0, 0])
        d["pt"][1, 1] = 1 << 20
        d["sl"][0] = -3
        T.tree_attend(b.cfg, d["q"], d["k"], d["v"], d["pt"], d["sl"], d["ws"], cu_tokens=d["cu"], mask=d["mask"])
        assert B.table_errors(b.cfg, d["ws"])[0] == B.LOCKS_TABLE_E_LENGTH | B.LOCKS_TABLE_E_BLOCK
    finally:
        B.set_table_checks(before)


# ---------------------------------------------------------------- mass

def _mass_case(past, new, q, kv, mask, G, P, H=2, decay=0.75, pad=2, seed=0):
    b = Batch(past, new, H=H, G=G, P=P, q=q, kv=kv, pad=pad, seed=seed, mask=mask).garbage()
    d = b.dev()
    width = b.cfg.max_pages_per_seq * P
    old = torch.rand(len(past), H, width, generator=b.gen)
    old[..., -1] = float("nan")
    for s, L in enumerate(b.lens):
        old[s, :, b.past[s]:L] = float("nan")       # other tokens' that had these slots
    lse = torch.full((b.n, G * H), float("nan"))
    want, bound = old.double().numpy(), np.zeros(old.shape)
    for s, h, rows, qq, K, V, ok in b.units():
        n, L = new[s], b.lens[s]
        if n == 0:
            continue
        _, wl, big = R.attend(qq, K, V, ok)
        wl = wl.astype(np.float32)
        lse[rows, h * G:(h + 1) * G] = torch.from_numpy(wl)
        add, far = R.weights(qq, K, ok, wl.astype(np.float64))
        kept = np.float32(decay) * want[s, h, :L - n]
        want[s, h, :L - n] = kept + add[:L - n]
        want[s, h, L - n:L] = add[L - n:]
        zl = far + 2 * (np.abs(wl[np.isfinite(wl)]).max() if np.isfinite(wl).any() else 0)
        rel = 130 * 2.0 ** -24 * big + 2.0 ** -21 * (1 + zl) + (n * G + 64) * 2.0 ** -23
        bound[s, h, :L] = rel * add * 1.01 + 2.0 ** -22 * np.abs(want[s, h, :L])
    mass = old.cuda()
    got = T.token_mass(b.cfg, d["q"], lse.cuda(), d["k"], d["pt"], d["sl"], mass, cu_tokens=d["cu"], mask=d["mask"],
                       decay=decay)
    assert got is mass
    got = mass.cpu().double().numpy()
    same = np.isnan(want)
    assert (np.isnan(got) == same).all()
    assert (np.abs(got - want)[~same] <= bound[~same]).all(), np.nanmax(np.abs(got - want))
    for s, L in enumerate(b.lens):                   # past the end, and sequences without new tokens
        keep = slice(0 if new[s] == 0 else L, None)
        assert torch.equal(mass[s, :, keep].cpu().nan_to_num(-1), old[s, :, keep].nan_to_num(-1))


@pytest.mark.parametrize("mask", ["tree", None])
@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_token_mass(shape, q, kv, mask):
    past, new = SHAPES[shape]
    G, P = (4, 7, 1, 16, 3)[shape % 5], (16, 32, 64)[shape % 3]
    print(f"[mass] {past} {new} G={G} P={P} {q}/{kv} mask={mask}", flush=True)
    _mass_case(past, new, q, kv, mask, G, P, seed=shape)


@pytest.mark.parametrize("decay", [0.0, 1.0, -0.5])
def test_token_mass_decay_and_many_sequences(decay):
    print(f"[mass] decay={decay}", flush=True)
    _mass_case([(37 * s) % 90 for s in range(300)], [1] * 300, "bf16", "bf16", None, 2, 16, H=1, decay=decay, pad=0)
    _mass_case([0, 3, 1200], [4, 0, 2], "bf16", "bf16", "tree", 4, 32, decay=decay)


@pytest.mark.parametrize("q", ["bf16", "fp32"])
def test_token_mass_of_more_sequences_than_are_counted(q):
    """Beyond 512 sequences a block takes whole lists."""
    print(f"[mass] 600 sequences {q}", flush=True)
    _mass_case([(53 * s) % 300 for s in range(600)], [s % 3 for s in range(600)], q, q, "tree", 2, 16, H=1, pad=1)


@pytest.mark.parametrize("q", ["bf16", "fp32"])
@pytest.mark.parametrize("mask", ["tree", None])
def test_token_mass_of_many_rows(q, mask):
    """More rows than LDS holds at once; trees wider than a word."""
    print(f"[mass] many rows {q} {mask}", flush=True)
    _mass_case([30, 0, 513], [150, 90, 33], q, q, mask, 4, 64, decay=0.25)


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("mask", ["tree", None])
@pytest.mark.parametrize("extra", [0, 40000])
@pytest.mark.parametrize("past,new,G,P", [([0, 31, 100], [64, 33, 40], 8, 16), ([7], [300], 16, 64), ([500, 3], [97, 128], 4, 32)])
def test_token_mass_of_many_rows_and_any_table(monkeypatch, past, new, G, P, extra, mask, q, kv):
    """Rows shared by a block's waves (short tables), and not."""
    table_of = R.table_of
    monkeypatch.setattr(R, "table_of", lambda lens, P, g, spare=3, extra=1, more=extra: table_of(lens, P, g, spare, extra + more // P))
    _mass_case(past, new, q, kv, mask, G, P)


def test_token_mass_of_rows_that_see_nothing_and_of_bad_keys():
    """-inf rows add nothing; a key that is not finite makes only its own token's mass so; a
    NaN row makes what it sees NaN."""
    b = Batch([40], [20], seed=3)
    d = b.dev()
    _, lse = b.run()
    mass = T.alloc_mass(b.cfg)
    T.token_mass(b.cfg, d["q"], lse.cuda(), d["k"], d["pt"], d["sl"], mass, cu_tokens=d["cu"], mask=d["mask"])
    want = mass.cpu()
    none = lse.clone()
    none[:] = -np.inf
    zero = T.alloc_mass(b.cfg)
    T.token_mass(b.cfg, d["q"], none.cuda(), d["k"], d["pt"], d["sl"], zero, cu_tokens=d["cu"], mask=d["mask"])
    assert not bool(zero.any())
    d["k"][int(b.table[0, 1]), :, 4] = float("nan")
    mass = T.alloc_mass(b.cfg)
    T.token_mass(b.cfg, d["q"], lse.cuda(), d["k"], d["pt"], d["sl"], mass, cu_tokens=d["cu"], mask=d["mask"])
    got = mass.cpu()
    assert bool(got[0, :, 20].isnan().all())
    got[0, :, 20] = want[0, :, 20]
    assert torch.equal(got, want)
    # the whole of it: every row's weights sum to 1
    total = want.sum(-1)[0]
    assert bool(((total - b.G * 20).abs() < 1e-3).all())


@pytest.mark.parametrize("q", ["bf16", "fp32"])
def test_token_mass_long(q):
    b = Batch([40000, 900], [33, 2], H=2, G=4, q=q, kv=q, seed=9, extra=50)
    _, lse = b.run()
    d = b.d
    mass = torch.rand(2, 2, b.cfg.max_pages_per_seq * 16, generator=b.gen).cuda()
    old = mass.clone()
    T.token_mass(b.cfg, d["q"], lse.cuda(), d["k"], d["pt"], d["sl"], mass, cu_tokens=d["cu"], mask=d["mask"], decay=0.5)
    for s, h in itertools.product(range(2), range(2)):
        L, n = b.lens[s], b.new[s]
        pages = b.table[s, :-(-L // 16)].long().cuda()
        K = d["k"][pages, h].reshape(-1, D)[:L].double()
        rows = slice(b.cu[s], b.cu[s + 1])
        qd = d["q"][rows, 4 * h:4 * h + 4].double().reshape(4 * n, D)
        ok = torch.ones(n, L, dtype=torch.bool)
        ok[:, L - n:] = torch.from_numpy(R.sees(n, n, b.mask[rows].numpy()))
        e = lse[rows, 4 * h:4 * h + 4].cuda().double()
        z = (qd @ K.t().contiguous()).reshape(n, 4, L) / np.sqrt(D) - e[..., None]
        add = torch.where(ok.cuda()[:, None], z.exp(), 0.0).sum((0, 1))
        want = add.clone()
        want[:L - n] += 0.5 * old[s, h, :L - n].double()
        big = float((qd.abs() @ K.abs().t().contiguous()).max()) / np.sqrt(D)
        rel = 130 * 2.0 ** -24 * big + 2.0 ** -21 * (1 + float(z.abs().max()) + 2 * float(e.abs().max())) + (4 * n + 64) * 2.0 ** -23
        assert bool(((mass[s, h, :L].double() - want).abs() <= 1.01 * rel * add + 2.0 ** -22 * want).all())
        assert torch.equal(mass[s, h, L:], old[s, h, L:])


# ---------------------------------------------------------------- pick

@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "special"])
@pytest.mark.parametrize("lens,n_keep,sink,recent", [
    ([1, 0, 5], 4, 1, 1), ([17, 33, 64], 16, 0, 0), ([100, 1500, 31], 30, 4, 8), ([1030, 1024, 1025], 1024, 0, 1024),
    ([3000], 7, 7, 0), ([3000, 2999], 1000, 3, 100), ([5000, 40], 1, 0, 0), ([9000, 16385, 16384], 4097, 16, 1000),
    ([70001, 33000], 2048, 4, 128), ([200000], 9001, 64, 512),
])
def test_pick_tokens(lens, n_keep, sink, recent, kind):
    P = 16
    H = 2
    g = torch.Generator().manual_seed(len(lens) + n_keep)
    mp = -(-max(lens) // P) + 1
    cfg = B.Config(len(lens), 4 * H, H, 8, 256, mp, 8, page_size=P)
    print(f"[pick] {lens} keep={n_keep} {sink}+{recent} {kind}", flush=True)
    x = torch.exp(2 * torch.randn(len(lens), H, mp * P, generator=g))
    if kind == "ties":
        x = torch.round(x * 2) / 2
    elif kind == "equal":
        x = torch.full_like(x, 0.25)
    elif kind == "special":
        r = torch.rand(x.shape, generator=g)
        x = torch.where(r < 0.2, torch.zeros_like(x), x)
        x = torch.where((r > 0.2) & (r < 0.4), torch.full_like(x, -0.0), x)
        x = torch.where((r > 0.4) & (r < 0.5), torch.full_like(x, float("nan")), x)
        x = torch.where((r > 0.5) & (r < 0.6), -x, x)
        x = torch.where((r > 0.6) & (r < 0.62), torch.full_like(x, float("inf")), x)
        x = torch.where((r > 0.62) & (r < 0.7), torch.full_like(x, -float("inf")), x)
        x = torch.where((r > 0.7) & (r < 0.8), x * 2.0 ** -149, x)
    for s, L in enumerate(lens):
        x[s, :, L:] = float("inf")               # never a token's
    ws = T.alloc_pick_workspace(cfg)
    ws.fill_(255)
    got = T.pick_tokens(cfg, x.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), n_keep, sink, recent, ws).cpu()
    for s, L in enumerate(lens):
        for h in range(H):
            want = R.pick(x[s, h].numpy(), L, n_keep, sink, recent)
            assert got[s, h].tolist() == want + [-1] * (n_keep - len(want)), (s, h)


@pytest.mark.parametrize("kind", ["spread", "ties", "special"])
@pytest.mark.parametrize("lens", [[40000, 32769, 8193, 100], [33000 - 900 * s for s in range(30)],
                                  [33000 - 450 * s for s in range(60)], [600001, 16384]])
def test_pick_chunks_of_every_size(lens, kind):
    test_pick_tokens(lens, 700, 4, 65, kind)


def test_pick_holds_lengths_to_the_table():
    cfg = B.Config(2, 8, 2, 8, 256, 3, 8)
    x = torch.rand(2, 2, 48).cuda()
    got = T.pick_tokens(cfg, x, torch.tensor([4000, -7], dtype=torch.int32).cuda(), 50, 0, 0, T.alloc_pick_workspace(cfg))
    assert got[0].tolist() == [list(range(48)) + [-1, -1]] * 2 and bool((got[1] == -1).all())


# ---------------------------------------------------------------- keep

def _keep_case(lens, lists, start, P, kv, H=2, with_mass=True, in_place=False, seed=0, spare=3):
    """lists [S][heads][n] of token indices (padded here with -1)."""
    g = torch.Generator().manual_seed(seed)
    table, nb = R.table_of(lens, P, g, spare=spare)
    S = len(lens)
    cfg = B.Config(S, 4 * H, H, 8, 256, table.shape[1], nb, LK[kv], LK[kv], page_size=P)
    k, v = (torch.randn(nb, H, P, D, generator=g).to(DT[kv]) for _ in range(2))
    mass = torch.rand(S, H, table.shape[1] * P, generator=g) if with_mass else None
    width = max(len(x) for l in lists for x in l)
    kept = torch.tensor([[list(x) + [-1] * (width - len(x)) for x in l] for l in lists], dtype=torch.int32)
    dk, dv, dm = k.cuda(), v.cuda(), None if mass is None else mass.cuda()
    sl = torch.tensor(lens, dtype=torch.int32).cuda()
    st = None if start is None else torch.tensor(start, dtype=torch.int32).cuda()
    got = T.keep_tokens(cfg, kept.cuda(), dk, dv, table.cuda(), start=st, mass=dm, out_lens=sl if in_place else None)
    want = []
    for s in range(S):
        want.append(R.keep(kept[s].tolist(), start[s] if start else 0, (k, v), None if mass is None else mass[s],
                           table[s], P))
    assert got.tolist() == want and (not in_place or got is sl)
    assert torch.equal(dk.cpu(), k) and torch.equal(dv.cpu(), v)
    assert mass is None or torch.equal(dm.cpu(), mass)


def _ascending(L, n, g, lo=0):
    return sorted((torch.randperm(L - lo, generator=g)[:n] + lo).tolist())


@pytest.mark.parametrize("kv", ["bf16", "fp32"])
@pytest.mark.parametrize("P", [16, 32, 64])
@pytest.mark.parametrize("share", [0.02, 0.5, 0.97])
def test_keep_picked_lists(kv, P, share):
    print(f"[keep] P={P} {kv} {share}", flush=True)
    g = torch.Generator().manual_seed(P)
    lens = [1, 700, 2111, 63, 0]
    lists = [[_ascending(L, max(0, int(L * share)), g) for _ in range(2)] for L in lens]
    _keep_case(lens, lists, None, P, kv, with_mass=P != 32, in_place=P == 16)


@pytest.mark.parametrize("heads", [1, 2])
@pytest.mark.parametrize("kv", ["bf16", "fp32"])
def test_keep_accepted_branches(kv, heads):
    g = torch.Generator().manual_seed(heads)
    past = [0, 15, 16, 300, 45, 9]
    new = [1, 40, 64, 7, 130, 5]
    count = [1, 6, 12, 0, 100, 5]
    lists = [[_ascending(a + b, c, g, lo=a) for _ in range(heads)] for a, b, c in zip(past, new, count)]
    _keep_case([a + b for a, b in zip(past, new)], lists, past, 16, kv)


def test_keep_everything_moves_nothing_and_shifts_by_one():
    L = 3000
    _keep_case([L], [[list(range(L))] * 2], None, 16, "bf16")
    _keep_case([L], [[list(range(1, L))] * 2], None, 16, "bf16")
    _keep_case([L], [[list(range(1500)) + list(range(1501, L))] * 2], None, 64, "fp32")


def test_keep_odd_lists():
    """Lists out of order, the same token twice, entries that would move to the back (left
    out), and ends inside."""
    _keep_case([200], [[[9, 5, 7, 7, 120, 60, 61, 199, 8, 9], [3, 3, 3, 3, 3, 3]]], None, 16, "bf16")
    _keep_case([200, 90], [[[150, 20, 199, 180]], [[50, -1, 60]]], [100, 40], 32, "fp32")


def test_keep_leaves_out_what_lies_outside_the_tables():
    g = torch.Generator().manual_seed(1)
    table, nb = R.table_of([64], 16, g, extra=0)
    cfg = B.Config(1, 8, 2, 8, 256, 4, nb)
    k, v = (torch.randn(nb, 2, 16, D, generator=g).bfloat16() for _ in range(2))
    kept = torch.tensor([[[2, 64, 1 << 30, 40, 63]]], dtype=torch.int32)
    table[0, 2] = nb + 7                             # token 40's page
    want = k.clone()
    for i, t in ((0, 2), (4, 63)):
        want[int(table[0, 0]), :, i] = k[int(table[0, t // 16]), :, t % 16]
    dk, dv = k.cuda(), v.cuda()
    got = T.keep_tokens(cfg, kept.cuda(), dk, dv, table.cuda())
    assert torch.equal(dk.cpu(), want) and got.tolist() == [5]
    got = T.keep_tokens(cfg, kept.cuda(), dk, dv, table.cuda(), start=torch.tensor([-4], dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    got = T.keep_tokens(cfg, torch.empty(1, 1, 0, dtype=torch.int32).cuda(), dk, dv, table.cuda(),
                        start=torch.tensor([9], dtype=torch.int32).cuda())
    assert got.tolist() == [9]


# ---------------------------------------------------------------- together

def test_speculative_step_and_a_bounded_cache():
    """Drafts are appended with their depths as positions, attended as a tree, a branch is
    kept; the cache then holds what appending that branch alone gives, and attention over it
    equals the tree's row.  Then tokens are judged, picked and moved, and attention over the
    smaller cache equals that over the picked rows."""
    H, G, P, past = 2, 4, 16, [70, 33]
    parents, cu = [-1, 0, 0, 1, 2, 4] + [-1, 0, 1, 1], [0, 6, 10]
    branch = [[0, 2, 4, 5], [0, 1, 3]]
    g = torch.Generator().manual_seed(11)
    b = Batch(past, [6, 4], H=H, G=G, P=P, seed=4)
    d = b.dev()
    mask, depth = T.tree_mask(parents, cu)
    seq = torch.tensor([0] * 6 + [1] * 4)
    past_t = torch.tensor(past, dtype=torch.int32)
    pos = past_t[seq].cuda() + depth
    rope = C.Rope(C.rope_table(200, 128))
    kn, vn = (torch.randn(10, H, D, generator=g).bfloat16().cuda() for _ in range(2))
    qn = torch.randn(10, G * H, D, generator=g).bfloat16().cuda()
    base_k, base_v = d["k"].clone(), d["v"].clone()
    q = C.rope_append_kv(b.cfg, kn, vn, d["k"], d["v"], d["pt"], d["sl"], rope=rope, positions=pos, cu_tokens=d["cu"],
                         q=qn)
    out, lse = T.tree_attend(b.cfg, q, d["k"], d["v"], d["pt"], d["sl"], d["ws"], cu_tokens=d["cu"], mask=mask)
    kept = torch.full((2, 1, 4), -1, dtype=torch.int32)
    for s, br in enumerate(branch):
        kept[s, 0, :len(br)] = torch.tensor([past[s] + i for i in br])
    lens = d["sl"].clone()
    T.keep_tokens(b.cfg, kept.cuda(), d["k"], d["v"], d["pt"], start=past_t.cuda(), out_lens=lens)
    assert lens.tolist() == [74, 36]
    rows = torch.tensor(branch[0] + [6 + i for i in branch[1]]).cuda()
    cu2 = torch.tensor([0, 4, 7], dtype=torch.int32).cuda()
    C.rope_append_kv(b.cfg, kn[rows].contiguous(), vn[rows].contiguous(), base_k, base_v, d["pt"], lens, rope=rope,
                     cu_tokens=cu2)
    for s in range(2):
        L = int(lens[s])
        pages = d["pt"][s, :-(-L // P)].long()
        for x, y in ((d["k"], base_k), (d["v"], base_v)):
            assert torch.equal(x[pages].transpose(1, 2).reshape(-1, H, D)[:L], y[pages].transpose(1, 2).reshape(-1, H, D)[:L])
    ws = B.alloc_workspace(b.cfg)
    last = torch.tensor([branch[0][-1], 6 + branch[1][-1]]).cuda()
    q1 = q[last].contiguous()
    o1, l1 = B.dense_attend(b.cfg, q1, d["k"], d["v"], d["pt"], lens, ws)
    assert float((o1 - out[last]).abs().max()) < 2.0 ** -12 and float((l1 - lse[last]).abs().max()) < 2.0 ** -14
    # a bounded cache
    mass = T.alloc_mass(b.cfg)
    T.token_mass(b.cfg, q1, l1, d["k"], d["pt"], lens, mass)
    assert float((mass.sum(-1) - G).abs().max()) < 1e-3
    ids = T.pick_tokens(b.cfg, mass, lens, 24, 2, 6, T.alloc_pick_workspace(b.cfg))
    k0, v0, m0, pt = d["k"].cpu(), d["v"].cpu(), mass.cpu(), b.table
    T.keep_tokens(b.cfg, ids, d["k"], d["v"], d["pt"], mass=mass, out_lens=lens)
    assert lens.tolist() == [24, 24]
    o2, l2 = B.dense_attend(b.cfg, q1, d["k"], d["v"], d["pt"], lens, ws)
    for s, h in itertools.product(range(2), range(H)):
        got = ids[s, h].tolist()
        assert got == R.pick(m0[s, h].numpy(), [74, 36][s], 24, 2, 6)
        K, V = (torch.stack([c[int(pt[s, t // P]), h, t % P] for t in got]).double().numpy() for c in (k0, v0))
        want, wl, _ = R.attend(q1[s:s + 1, h * G:(h + 1) * G].cpu().double().numpy(), K, V, np.ones((1, 24), bool))
        assert np.abs(o2[s, h * G:(h + 1) * G].cpu().numpy() - want[0]).max() < 2.0 ** -12
        assert torch.equal(mass[s, h, :24].cpu(), m0[s, h, got])


def _whole_step(b, d, mass, ids, lens, lse, out, pws):
    T.tree_attend(b.cfg, d["q"], d["k"], d["v"], d["pt"], d["sl"], d["ws"], cu_tokens=d["cu"], mask=d["mask"], out=out,
                  out_lse=lse)
    T.token_mass(b.cfg, d["q"], lse, d["k"], d["pt"], d["sl"], mass, cu_tokens=d["cu"], mask=d["mask"], decay=0.5)
    T.pick_tokens(b.cfg, mass, d["sl"], 64, 4, 16, pws, out=ids)
    T.keep_tokens(b.cfg, ids, d["k"], d["v"], d["pt"], mass=mass, out_lens=lens)


@pytest.mark.parametrize("past", [[300, 900], [40000, 21000]])
def test_captured_step_replays(past):
    """The four calls in one graph, replayed with other inputs between the program's own eager
    work; two graphs that share the workspaces run one after the other."""
    b = Batch(past, [20, 9], seed=2)
    d = b.dev()
    n = b.n

    def bufs():
        return dict(mass=T.alloc_mass(b.cfg), ids=torch.empty(2, 2, 64, dtype=torch.int32).cuda(),
                    lens=torch.empty(2, dtype=torch.int32).cuda(), lse=torch.empty(n, 8).cuda(),
                    out=torch.empty(n, 8, D, dtype=torch.bfloat16).cuda(), pws=T.alloc_pick_workspace(b.cfg))
    x = bufs()
    k0, v0 = d["k"].clone(), d["v"].clone()
    _whole_step(b, d, **x)                       # warm
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for gr in graphs:
        with torch.cuda.graph(gr):
            _whole_step(b, d, **x)
    for turn in range(4):
        qn = torch.randn(n, 8, D, generator=b.gen).bfloat16().cuda()
        d["q"].copy_(qn)
        got = []
        for how in (0, 1, None):
            d["k"].copy_(k0)
            d["v"].copy_(v0)
            x["mass"].zero_()
            if how is None:
                _whole_step(b, d, **x)
            else:
                graphs[how].replay()
            got.append([t.clone() for t in (x["out"], x["lse"], x["mass"], x["ids"], x["lens"], d["k"], d["v"])])
            float(got[-1][1].sum())              # eager work and a synchronisation between
        for other in got[1:]:
            assert all(torch.equal(p, q) for p, q in zip(got[0], other)), turn


def test_two_streams_at_once():
    """Calls with workspaces of their own on two streams, one of them not the current one."""
    bs = [Batch([20000, 500], [20, 9], seed=s) for s in (1, 2)]
    ds = [b.dev() for b in bs]
    want = []
    for b, d in zip(bs, ds):
        want.append([t.clone() for t in T.tree_attend(b.cfg, d["q"], d["k"], d["v"], d["pt"], d["sl"], d["ws"],
                                                      cu_tokens=d["cu"], mask=d["mask"])])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [T.tree_attend(b.cfg, d["q"], d["k"], d["v"], d["pt"], d["sl"], d["ws"], cu_tokens=d["cu"],
                             mask=d["mask"], stream=st) for b, d, st in zip(bs, ds, streams)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


def test_a_workspace_serves_fewer_tokens():
    """One workspace for the largest step, used for smaller ones, other contents left in it."""
    big = Batch([100, 300], [64, 64], seed=1)
    ws = T.alloc_tree_workspace(big.cfg, 20000)
    ws.fill_(255)
    for new in ([64, 64], [1, 1], [9, 2], [20, 15]):
        b = Batch([100, 300], new, seed=sum(new))
        d = b.dev()
        assert T.tree_workspace_bytes(b.cfg, b.n) <= ws.numel()
        got = T.tree_attend(b.cfg, d["q"], d["k"], d["v"], d["pt"], d["sl"], ws, cu_tokens=d["cu"], mask=d["mask"])
        b.check(got=(got[0].cpu(), got[1].cpu()))


def test_a_bad_page_is_read_as_block_zero_or_left_out():
    """Without table checks: a block outside the cache is never read."""
    b = Batch([100], [5], seed=3)
    d = b.dev()
    k0 = b.table.clone()
    d["pt"][0, 2] = 1 << 30
    out, lse = T.tree_attend(b.cfg, d["q"], d["k"], d["v"], d["pt"], d["sl"], d["ws"], cu_tokens=d["cu"], mask=d["mask"])
    b.table[0, 2] = 0
    b.check(got=(out.cpu(), lse.cpu()))
    b.table = k0
    mass = T.alloc_mass(b.cfg)
    mass.fill_(2.0)
    T.token_mass(b.cfg, d["q"], lse, d["k"], d["pt"], d["sl"], mass, cu_tokens=d["cu"], mask=d["mask"])
    assert bool((mass[0, :, 32:48] == 2.0).all()) and bool((mass[0, :, :32] != 2.0).all())


def test_the_same_inputs_twice_give_the_same_bits():
    b = Batch([7000, 300], [33, 20], seed=6)
    a, c = b.run("bf16"), b.run("bf16")
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])
