"""GPU checks of the paged-cache calls (include/locks_cache.h) against the plain CPU
definitions of tests/_cache_reference.py: rotated appends into bf16 / fp32 caches and into
8-bit caches, and decode attention over the latter.

Bounds: a rotated float32 value is within 2^-22 (|a c| + |b s|) of the 64-bit one (three
roundings), a bf16 result half a step (2^-8 relative) further, and codes and scales are
the definition's own float32 operations, so they are equal bit for bit.  A logit is a sum
of n exact products in float32 (n = 128, with float32 queries 2 x 128 and 8 more for a
query's two f16 terms, which hold it to 2^-21: 385 is allowed), off by at most dz =
n 2^-24 sum |q k|; a weight times its value scale is held to 2^-16 of itself (two f16
terms hold 2^-21), so an output is within (2 dz + 2^-15) max |v| of the 64-bit one
(numerator and denominator), and the LSE within dz + 2^-18 (|lse| + 1)."""
import numpy as np
import pytest
import torch

from paper_2607_24555_amd import cache as C
from paper_2607_24555_amd import locks as B
from tests import _cache_reference as R

pytestmark = pytest.mark.gpu
D = 128
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
LK = {"bf16": B.LOCKS_BF16, "fp32": B.LOCKS_FP32}
CODES = [torch.int8, torch.float8_e4m3fn]


class Step:
    """A ragged step: per sequence `past` cached and `new` appended tokens."""

    def __init__(self, past, new, H=2, G=4, P=16, q="bf16", kv="bf16", pad=0, seed=0, ragged=True,
                 spare=3):
        self.past, self.new, self.P, self.H, self.G = past, new, P, H, G
        self.lens = [a + b for a, b in zip(past, new)]
        S = len(past)
        g = torch.Generator().manual_seed(seed)
        pages = [max(1, -(-L // P)) for L in self.lens]
        nb = sum(pages) + spare
        mp = max(pages) + 1
        perm = torch.randperm(nb, generator=g).int()
        self.table = torch.full((S, mp), -1, dtype=torch.int32)
        off = 0
        for s in range(S):
            self.table[s, :pages[s]] = perm[off:off + pages[s]]
            off += pages[s]
        self.cfg = B.Config(S, G * H, H, 8, max(256, 2 * P), mp, nb, LK[kv], LK[q], page_size=P)
        cu = [0]
        for t in new:
            cu.append(cu[-1] + t)
        self.cu = cu
        n = cu[-1] + pad
        # one projection's output: q, k, v are slices of it where the types agree
        self.k = (torch.randn(n, H, D, generator=g) * 2).to(DT[kv])
        self.k[:, :, 5] += 9
        self.v = torch.randn(n, H, D, generator=g).to(DT[kv])
        self.q = torch.randn(n, G * H, D, generator=g).to(DT[q])
        self.cu_dev = torch.tensor(cu, dtype=torch.int32).cuda() if ragged else None
        self.pt = self.table.cuda()
        self.sl = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.gen = g

    def strided(self, t):
        """The rows as a slice of a wider buffer (its other columns NaN)."""
        n, h, _ = t.shape
        wide = torch.full((n, h + 3, D), float("nan"), dtype=t.dtype).cuda()
        wide[:, 1:1 + h] = t.cuda()
        return wide[:, 1:1 + h]

    def tokens(self):
        for s in range(len(self.new)):
            for i in range(self.new[s]):
                yield s, self.cu[s] + i, self.past[s] + i


def _rope(rot, inter, axes, n_pos):
    table = R.angles(n_pos, rot)
    half = rot // 2
    split = {1: [half], 2: [half // 2, half - half // 2], 3: [half // 4, 3, half - half // 4 - 3]}[axes]
    return table, split, C.Rope(torch.from_numpy(table).cuda(), inter, None if axes == 1 else split)


SHAPES = [
    # past, new: single tokens, page borders, ragged runs, none at all
    ([0], [1]), ([15], [1]), ([16], [1]), ([5, 0, 31, 16], [1, 1, 1, 1]),
    ([0, 7, 16, 40], [33, 0, 16, 9]), ([3, 0], [80, 130]), ([0] * 70, [1, 0, 2, 5, 17] * 14),
]


ROTATIONS = [(128, False, 1), (64, True, 1), (16, False, 3), (112, True, 2), (48, False, 2), (0, False, 1)]


@pytest.mark.parametrize("rot,inter,axes,q,kv", [
    (*r, q, kv) for r in ROTATIONS
    for q, kv in (("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32"), ("fp32", "bf16"))
    if q == kv or r[0] in (64, 48)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_rope_append(q, kv, rot, inter, axes, shape):
    past, new = SHAPES[shape]
    P = (16, 32, 64)[shape % 3]
    st = Step(past, new, P=P, q=q, kv=kv, pad=3, seed=shape, G=(4, 7, 1)[shape % 3])
    n = st.k.shape[0]
    print(f"[rope append] {past} {new} P={P} {q}/{kv} rot={rot} inter={inter} axes={axes}", flush=True)
    rope = pos = None
    if rot:
        table, split, rope = _rope(rot, inter, axes, 700)
        if axes > 1:
            pos = torch.randint(0, 700, (axes, n), generator=st.gen, dtype=torch.int32)
    kc, vc = (torch.randn(st.cfg.num_blocks, st.H, P, D, generator=st.gen).to(DT[kv]).cuda() for _ in range(2))
    q_out = torch.full((n, st.G * st.H, D), 7.0, dtype=DT[q]).cuda()
    want_k, want_v = kc.cpu().double(), vc.cpu().clone()
    bound = torch.zeros_like(want_k)
    got = C.rope_append_kv(st.cfg, st.strided(st.k), st.strided(st.v), kc, vc, st.pt, st.sl, rope=rope,
                           positions=None if pos is None else pos.cuda(), cu_tokens=st.cu_dev,
                           q=st.strided(st.q), q_out=q_out)
    torch.cuda.synchronize()
    assert got is q_out
    want_q, bound_q = torch.full(q_out.shape, 7.0, dtype=torch.float64), torch.zeros(q_out.shape, dtype=torch.float64)
    half_q, half_k = (torch.finfo(DT[t]).eps / 2 if t == "bf16" else 0.0 for t in (q, kv))
    for s, row, tok in st.tokens():
        b, i = int(st.table[s, tok // P]), tok % P
        kr, qr = st.k[row].float().numpy(), st.q[row].float().numpy()
        if rot:
            p = [tok] * axes if pos is None else pos[:, row].tolist()
            args = (table, inter, split, p)
            want_k[b, :, i] = torch.from_numpy(R.rotate(kr, *args, np.float64))
            want_q[row] = torch.from_numpy(R.rotate(qr, *args, np.float64))
            bound[b, :, i] = torch.from_numpy(R.rotate_bound(kr, *args)) * 2.0 ** -22
            bound_q[row] = torch.from_numpy(R.rotate_bound(qr, *args)) * 2.0 ** -22
            bound[b, :, i, :rot] += want_k[b, :, i, :rot].abs() * half_k
            bound_q[row, :, :rot] += want_q[row, :, :rot].abs() * half_q
        else:
            want_k[b, :, i] = torch.from_numpy(kr).double()
            want_q[row] = torch.from_numpy(qr).double()
        want_v[b, :, i] = st.v[row]
    assert torch.equal(vc.cpu(), want_v)
    # (the half step is of the value before rounding: 2^-22 more covers the difference)
    assert bool(((kc.cpu().double() - want_k).abs() <= bound * (1 + 2.0 ** -7)).all())
    assert bool(((q_out.cpu().double() - want_q).abs() <= bound_q * (1 + 2.0 ** -7)).all())


@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("inter", [False, True])
def test_rope_append_of_a_long_prompt(q, kv, inter):
    """A step that writes more than 48 MiB (its rows bypass the caches): the same rows, bit for
    bit, as in short calls, which the test above checks against the definition."""
    st = Step([5, 0], [1300, 1210], H=8, G=8, q=q, kv=kv, pad=5, seed=9)
    written = st.cu[-1] * D * (64 * st.q.element_size() + 16 * st.k.element_size())
    assert written >= 48 << 20
    _, _, rope = _rope(96, inter, 1, 1400)
    kc, vc, kc2, vc2 = (torch.zeros(st.cfg.num_blocks, st.H, 16, D, dtype=DT[kv]).cuda() for _ in range(4))
    qd, kd, vd = (st.strided(x) for x in (st.q, st.k, st.v))
    out, out2 = (torch.full(st.q.shape, 7.0, dtype=DT[q]).cuda() for _ in range(2))
    C.rope_append_kv(st.cfg, kd, vd, kc, vc, st.pt, st.sl, rope, cu_tokens=st.cu_dev, q=qd, q_out=out)
    for s in range(2):
        for a in range(st.cu[s], st.cu[s + 1], 300):
            b = min(a + 300, st.cu[s + 1])
            lens = torch.tensor([0, 0], dtype=torch.int32)
            lens[s] = st.past[s] + b - st.cu[s]
            cu = torch.tensor([0, b - a, b - a] if s == 0 else [0, 0, b - a], dtype=torch.int32)
            C.rope_append_kv(st.cfg, kd[a:b], vd[a:b], kc2, vc2, st.pt, lens.cuda(), rope, cu_tokens=cu.cuda(),
                             q=qd[a:b], q_out=out2[a:b])
    assert torch.equal(out, out2) and torch.equal(kc, kc2) and torch.equal(vc, vc2)
    C.rope_append_kv(st.cfg, kd, vd, kc, vc, st.pt, st.sl, rope, cu_tokens=st.cu_dev, q=qd, q_out=qd)  # in place
    assert torch.equal(qd[:st.cu[-1]], out[:st.cu[-1]])
    assert bool((out[st.cu[-1]:] == 7.0).all()) and bool((out[:st.cu[-1]] != 7.0).flatten(1).any(1).all())


def test_rope_append_in_place_and_without_queries():
    st = Step([5, 0, 20], [4, 9, 1], seed=3)
    table, split, rope = _rope(128, False, 1, 64)
    kc, vc, kc2, vc2 = (torch.zeros(st.cfg.num_blocks, st.H, 16, D, dtype=torch.bfloat16).cuda() for _ in range(4))
    q = st.strided(st.q)
    out = C.rope_append_kv(st.cfg, st.k.cuda(), st.v.cuda(), kc, vc, st.pt, st.sl, rope, cu_tokens=st.cu_dev, q=q)
    same = C.rope_append_kv(st.cfg, st.k.cuda(), st.v.cuda(), kc2, vc2, st.pt, st.sl, rope, cu_tokens=st.cu_dev,
                            q=q, q_out=q)
    assert same is q and torch.equal(q, out) and torch.equal(kc, kc2) and torch.equal(vc, vc2)
    kc2.zero_()
    assert C.rope_append_kv(st.cfg, st.k.cuda(), st.v.cuda(), kc2, vc2, st.pt, st.sl, rope, cu_tokens=st.cu_dev) is None
    assert torch.equal(kc, kc2)


def test_appends_leave_out_what_lies_outside_its_table():
    """Blocks, pages and positions out of range: those tokens are not written, the others are."""
    st = Step([0, 0, 0, 0], [3, 3, 3, 3], seed=4)
    table, split, rope = _rope(64, False, 1, 40)
    pt = st.table.clone()
    pt[0, 0] = st.cfg.num_blocks           # block outside the cache
    pt[1, 0] = -7
    sl = torch.tensor([3, 3, 16 * st.cfg.max_pages_per_seq + 3, 3], dtype=torch.int32)   # page outside the table
    pos = torch.arange(12, dtype=torch.int32)
    pos[9] = 40                            # sequence 3's first token: position outside
    pos[11] = -1                           # and its last
    for q8 in (False, True):
        q_out = torch.full((12, 8, D), 7.0, dtype=torch.bfloat16).cuda()
        kw = dict(rope=rope, positions=pos.cuda(), cu_tokens=st.cu_dev, q=st.q.cuda(), q_out=q_out)
        if q8:
            c = C.alloc_q8_cache(st.cfg)
            C.q8_append_kv(st.cfg, st.k.cuda(), st.v.cuda(), c, pt.cuda(), sl.cuda(), **kw)
            k, v = c.k.cpu().float(), c.v.cpu().float()
        else:
            kc, vc = (torch.zeros(st.cfg.num_blocks, st.H, 16, D, dtype=torch.bfloat16).cuda() for _ in range(2))
            C.rope_append_kv(st.cfg, st.k.cuda(), st.v.cuda(), kc, vc, pt.cuda(), sl.cuda(), **kw)
            k, v = kc.cpu().float(), vc.cpu().float()
        b = int(st.table[3, 0])
        for t in (k, v):
            assert bool((t[b, :, 1] != 0).any()) and bool((t[b, :, 0] == 0).all()) and bool((t[b, :, 2:] == 0).all())
            t[b] = 0
            assert bool((t == 0).all())
        written = (q_out != 7.0).flatten(1).any(1).cpu().tolist()
        assert written == [False] * 10 + [True, False]


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("rot,inter,axes", [(128, False, 1), (64, True, 1), (32, False, 2)])
@pytest.mark.parametrize("kv,shape", [("bf16", i) for i in range(len(SHAPES))] + [("fp32", i) for i in range(5)])
def test_q8_append(code, rot, inter, axes, kv, shape):
    """Codes and scales bit for bit, over three calls whose rows grow, so that pages with
    earlier rows are rounded again; everything else left as it was."""
    past, new = SHAPES[shape]
    P = (64, 16, 32)[shape % 3]
    table, split, rope = _rope(rot, inter, axes, 1200)
    st = Step(past, new, P=P, kv=kv, seed=shape)
    print(f"[q8 append] {past} {new} P={P} {code} {kv} rot={rot} axes={axes}", flush=True)
    S, H = len(past), st.H
    mp = max(-(-(L + 2 * n) // P) for L, n in zip(st.lens, new)) + 1
    nb = S * mp
    cfg = B.Config(S, 4 * H, H, 8, 2 * P, mp, nb, LK[kv], LK[kv], page_size=P)
    tab = torch.randperm(nb, generator=st.gen).int().reshape(S, mp)
    shape4 = (nb, H, P, D)
    codes = [torch.randint(-100, 100, shape4, generator=st.gen, dtype=torch.int8).view(code) for _ in range(2)]
    if code != torch.int8:
        codes = [torch.nan_to_num(c.float(), nan=1.0).to(code) for c in codes]
    scales = [torch.rand(nb, H, generator=st.gen) * 0.02 + 0.001 for _ in range(2)]
    if code != torch.int8:
        scales = [torch.exp2(torch.round(torch.log2(s))) for s in scales]
    cache = C.Q8Cache(codes[0].cuda(), codes[1].cuda(), scales[0].cuda(), scales[1].cuda())
    lens = list(past)
    for call, gain in enumerate((1.0, 3.0, 0.5)):
        k, v = (st.k * gain).to(DT[kv]), (st.v * gain).to(DT[kv])
        lens = [a + b for a, b in zip(lens, new)]
        n = k.shape[0]
        pos = torch.randint(0, 1200, (axes, n), generator=st.gen, dtype=torch.int32) if axes > 1 else None
        sl = torch.tensor(lens, dtype=torch.int32)
        q = st.strided(st.q.to(DT[kv]))
        qo = C.q8_append_kv(cfg, st.strided(k), st.strided(v), cache, tab.cuda(), sl.cuda(), rope=rope,
                            positions=None if pos is None else pos.cuda(), cu_tokens=st.cu_dev, q=q)
        torch.cuda.synchronize()
        for s in range(S):
            t0 = lens[s] - new[s]
            rows = {}
            for i in range(new[s]):
                row, tok = st.cu[s] + i, t0 + i
                p = [tok] if pos is None else pos[:, row].tolist()
                rows[tok] = (R.rotate(k[row].float().numpy(), table, inter, split, p, np.float32),
                             v[row].float().numpy())
                want = R.rotate(st.q[row].float().numpy(), table, inter, split, p, np.float32)
                assert torch.equal(qo[row].cpu(), torch.from_numpy(want).to(DT[kv]))
            for j in sorted({t // P for t in rows}):
                b = int(tab[s, j])
                here = {t - j * P: r for t, r in rows.items() if t // P == j}
                for x in range(2):
                    for h in range(H):
                        scales[x][b, h] = float(R.q8_append_page(
                            codes[x][b, h], np.float32(scales[x][b, h].item()),
                            {i: r[x][h] for i, r in here.items()}, max(0, t0 - j * P), code))
        for want, got in ((codes[0], cache.k), (codes[1], cache.v)):
            assert torch.equal(want.view(torch.uint8), got.cpu().view(torch.uint8)), call
        assert torch.equal(scales[0], cache.k_scale.cpu()) and torch.equal(scales[1], cache.v_scale.cpu())


@pytest.mark.parametrize("code", CODES)
def test_q8_append_extreme_rows(code):
    """Zeros, tiny rows, the type's largest values, infinities and NaN; and the same rows
    appended again change nothing."""
    P, H = 16, 1
    cfg = B.Config(6, 1, H, 8, 32, 2, 12, B.LOCKS_FP32, B.LOCKS_FP32, page_size=P)
    x = torch.randn(6, H, D, generator=torch.Generator().manual_seed(1))
    x[0] = 0
    x[1] *= 2.0 ** -110
    x[2, 0, 3] = torch.finfo(torch.float32).max
    x[3, 0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 3.0])
    x[4, 0, 0] = -448.0 * 2
    x[5] *= 2.0 ** -99
    tab = torch.arange(12, dtype=torch.int32).reshape(6, 2)
    sl = torch.full((6,), 1, dtype=torch.int32)
    cache = C.alloc_q8_cache(cfg, code)
    for again in range(2):
        C.q8_append_kv(cfg, x.cuda(), x.cuda(), cache, tab.cuda(), sl.cuda())
        torch.cuda.synchronize()
        for s in range(6):
            want = torch.zeros(P, D, dtype=torch.uint8).view(code)
            sc = R.q8_append_page(want, np.float32(0), {0: x[s, 0].numpy()}, 0, code)
            for c, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
                got = c[2 * s, 0].cpu()
                nan = torch.isnan(want.float())
                assert torch.equal(nan, torch.isnan(got.float()))
                assert torch.equal(want.float()[~nan], got.float()[~nan]), s
                assert float(scale[2 * s, 0]) == float(sc), s


@pytest.mark.parametrize("code", CODES)
def test_q8_values_stay_near_the_rows(code):
    """Token by token, as a generation loop appends: every stored value stays within the
    error that its page's scales allow -- half a step of int8 for each scale the page had
    since; half a step of e4m3 once, and half the subnormal step for each scale."""
    P, H, T = 32, 2, 70
    cfg = B.Config(1, 2, H, 8, 64, 4, 4, B.LOCKS_FP32, B.LOCKS_FP32, page_size=P)
    g = torch.Generator().manual_seed(8)
    x = torch.randn(2, T, H, D, generator=g) * torch.linspace(0.3, 3, T)[None, :, None, None]
    cache = C.alloc_q8_cache(cfg, code)
    tab = torch.tensor([[2, 0, 3, 1]], dtype=torch.int32)
    err = torch.zeros(2, T, H, 1, dtype=torch.float64)
    last = torch.zeros(2, 4, H)
    for t in range(T):
        C.q8_append_kv(cfg, x[0, t:t + 1].cuda(), x[1, t:t + 1].cuda(), cache, tab.cuda(),
                       torch.tensor([t + 1], dtype=torch.int32).cuda())
        j = t // P
        b = int(tab[0, j])
        sc = torch.stack([cache.k_scale[b], cache.v_scale[b]]).cpu()
        grew = sc != last[:, j]
        step = sc.double() * (0.5 if code == torch.int8 else 2.0 ** -10) * (1 + 2.0 ** -16)
        if t % P:
            err[:, j * P:t] += (grew * step)[:, None, :, None]
        err[:, t] = step[..., None]
        last[:, j] = sc
    got = torch.empty(2, T, H, D, dtype=torch.float64)
    for t in range(T):
        b = int(tab[0, t // P])
        got[0, t] = cache.k[b, :, t % P].cpu().double() * cache.k_scale[b].cpu().double()[:, None]
        got[1, t] = cache.v[b, :, t % P].cpu().double() * cache.v_scale[b].cpu().double()[:, None]
    # int8: rounding x / s once per scale; the product x (1 / s) is off by 2^-23 of up to 127 steps
    rel = 2.0 ** -16 if code == torch.int8 else 2.0 ** -4
    assert bool(((got - x.double()).abs() <= err + rel * x.abs().double()).all())


def _cache_of(st, code, seed=0, poison=True):
    """A filled 8-bit cache: random codes and scales; rows past the sequences' ends and
    blocks that no table reaches hold NaN codes (e4m3) or the largest ones, and NaN scales."""
    g = torch.Generator().manual_seed(seed)
    nb, H, P = st.cfg.num_blocks, st.H, st.P
    out = []
    for x in range(2):
        if code == torch.int8:
            c = torch.clamp(torch.round(torch.randn(nb, H, P, D, generator=g) * 30), -127, 127).to(torch.int8)
        else:
            c = (torch.randn(nb, H, P, D, generator=g) * 60).clamp(-448, 448).to(code)
        s = torch.exp(torch.randn(nb, H, generator=g) * 0.3) * (0.03 if code == torch.int8 else 2.0 ** -6)
        if poison:
            live = torch.zeros(nb, P, dtype=torch.bool)
            for q, L in enumerate(st.lens):
                for j in range(-(-L // P)):
                    live[int(st.table[q, j]), :max(0, min(P, L - j * P))] = True
            bad = torch.full((D,), 127, dtype=torch.int8)
            c.view(torch.int8).permute(0, 2, 1, 3)[~live] = bad
            s[~live.any(1)] = float("nan")
        out += [c, s]
    return out[0], out[2], out[1], out[3]


def _check_attend(st, code, q, out, lse, kc, vc, ks, vs, ids_of):
    n = 128 if st.cfg.q_dtype == B.LOCKS_BF16 else 3 * 128 + 1
    G, P = st.G, st.P
    for s, L in enumerate(st.lens):
        for h in range(st.H):
            heads = slice(h * G, (h + 1) * G)
            o, l, big, vmax = R.attend(q[s, heads].float().numpy(), kc[:, h], vc[:, h], ks[:, h].numpy(),
                                       vs[:, h].numpy(), st.table[s], ids_of(s, h), L, P)
            dz = n * 2.0 ** -24 * big
            d = np.abs(out[s, heads].cpu().double().numpy() - o)
            assert np.all(d <= (2 * dz + 2.0 ** -15) * vmax + 1e-30), (s, h, d.max())
            e = lse[s, heads].cpu().double().numpy()
            empty = np.isneginf(l)
            assert np.array_equal(np.isneginf(e), empty)
            assert np.all(np.abs(e[~empty] - l[~empty]) <= dz + 2.0 ** -18 * (np.abs(l[~empty]) + 1))


# a block's share within one list, over many short ones, over empty ones; more than 64
# sequences; enough lists for a block each
LENS = [[1], [0, 1, 15, 16, 17, 31, 32, 33], [130, 0, 257, 64], [1000, 3], [5000],
        [0, 0, 40, 0] * 17 + [0, 700, 0, 0, 9], [0, 1, 20, 5] * 70, [0], [0, 0, 0]]


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("q", ["bf16", "fp32"])
@pytest.mark.parametrize("G,P", [(1, 16), (3, 32), (4, 16), (7, 64), (16, 16)])
@pytest.mark.parametrize("lens", range(len(LENS)))
def test_q8_dense_attend(code, q, G, P, lens):
    st = Step([0] * len(LENS[lens]), LENS[lens], G=G, P=P, q=q, seed=lens)
    print(f"[q8 dense] lens={LENS[lens]} G={G} P={P} {q} {code}", flush=True)
    kc, vc, ks, vs = _cache_of(st, code, seed=lens)
    cache = C.Q8Cache(kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda())
    S = len(st.lens)
    qq = (torch.randn(S, G * st.H, D, generator=st.gen) * 1.5).to(DT[q])
    ws = B.alloc_workspace(st.cfg)
    out, lse = C.q8_dense_attend(st.cfg, qq.cuda(), cache, st.pt, st.sl, ws)
    torch.cuda.synchronize()
    _check_attend(st, code, qq, out, lse, kc, vc, ks, vs, lambda s, h: range(-(-st.lens[s] // P)))


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("q", ["bf16", "fp32"])
@pytest.mark.parametrize("G,P,budget", [(1, 16, 33), (4, 16, 256), (7, 32, 300), (16, 64, 128), (5, 16, 2048)])
def test_q8_sparse_attend(code, q, G, P, budget):
    """Tables with gaps, repeats of none, only the last page, nothing at all (-1)."""
    lens = [1, 0, 40, 700, 1500, 16 * 40]
    st = Step([0] * len(lens), lens, G=G, P=P, q=q, seed=G)
    st.cfg.budget_tokens = max(budget, 2 * P)
    print(f"[q8 sparse] G={G} P={P} budget={budget} {q} {code}", flush=True)
    kc, vc, ks, vs = _cache_of(st, code, seed=G + 50)
    cache = C.Q8Cache(kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda())
    k, S = st.cfg.k, len(lens)
    ids = torch.full((S, st.H, k), -1, dtype=torch.int32)
    rng = np.random.RandomState(G)
    for s, L in enumerate(lens):
        n = -(-L // P)
        for h in range(st.H):
            if s == 3 and h == 1:
                continue                                   # a table that lists nothing
            take = sorted(rng.choice(n, min(n, k), replace=False)) if n else []
            if s == 4 and h == 0:
                take = [n - 1]
            at = sorted(rng.choice(k, len(take), replace=False))   # -1 entries anywhere
            ids[s, h, at] = torch.tensor(take, dtype=torch.int32)
    qq = (torch.randn(S, G * st.H, D, generator=st.gen) * 1.5).to(DT[q])
    out, lse = C.q8_sparse_attend(st.cfg, qq.cuda(), cache, st.pt, st.sl, ids.cuda(), B.alloc_workspace(st.cfg))
    torch.cuda.synchronize()
    _check_attend(st, code, qq, out, lse, kc, vc, ks, vs,
                  lambda s, h: [int(j) for j in ids[s, h] if j >= 0])


@pytest.mark.parametrize("code", CODES)
def test_serving_loop(code):
    """Ragged prompts appended, then tokens one at a time, each step attended in full and over
    a table; prepared calls on a side stream, the whole step also captured and replayed."""
    P, H, G = 16, 2, 4
    lens0, T = [37, 1, 200, 16], 6
    S = len(lens0)
    table, split, rope = _rope(64, True, 1, 400)
    mp = 20
    cfg = B.Config(S, G * H, H, 8, 64, mp, S * mp, page_size=P)
    g = torch.Generator().manual_seed(77)
    tab = torch.randperm(S * mp, generator=g).int().reshape(S, mp)
    cu = torch.tensor(np.cumsum([0] + lens0), dtype=torch.int32)
    n = int(cu[-1])
    mk = lambda n: [torch.randn(n, h, D, generator=g).bfloat16().cuda() for h in (G * H, H, H)]
    prompt = mk(n)
    steps = [mk(S) for _ in range(T)]
    pt = tab.cuda()

    def fresh():
        c = C.alloc_q8_cache(cfg, code)
        C.q8_append_kv(cfg, prompt[1], prompt[2], c, pt, torch.tensor(lens0, dtype=torch.int32).cuda(), rope,
                       cu_tokens=cu.cuda())
        return c
    eager = fresh()
    want = []
    for t, (q, k, v) in enumerate(steps):
        sl = torch.tensor([L + t + 1 for L in lens0], dtype=torch.int32).cuda()
        ws = B.alloc_workspace(cfg)
        qr = C.q8_append_kv(cfg, k, v, eager, pt, sl, rope, q=q)
        o, l = C.q8_dense_attend(cfg, qr, eager, pt, sl, ws)
        ids = torch.full((S, H, cfg.k), -1, dtype=torch.int32)
        for s in range(S):
            m = -(-int(sl[s]) // P)
            take = list(range(m)) if m <= cfg.k else [0, 1, m - 2, m - 1]
            ids[s, :, :len(take)] = torch.tensor(take, dtype=torch.int32)
        so, sl2 = C.q8_sparse_attend(cfg, qr, eager, pt, sl, ids.cuda(), ws)
        st = Step([0] * S, [L + t + 1 for L in lens0], H=H, G=G, seed=1)
        st.table, st.cfg = tab, cfg
        host = [x.cpu() for x in (eager.k, eager.v, eager.k_scale, eager.v_scale)]
        _check_attend(st, code, qr.cpu(), o, l, *host, lambda s, h: range(-(-st.lens[s] // P)))
        _check_attend(st, code, qr.cpu(), so, sl2, *host, lambda s, h: [int(j) for j in ids[s, h] if j >= 0])
        want.append((o.clone(), l.clone()))
    # the same loop from fixed buffers: prepared calls captured once, replayed for each token
    c = fresh()
    q, k, v = (torch.zeros_like(x) for x in steps[0])
    sl = torch.tensor(lens0, dtype=torch.int32).cuda()
    q_out = torch.zeros_like(q)
    append = C.prepare_q8_append_kv(cfg, k, v, c, pt, sl, rope, q=q, q_out=q_out)
    attend = C.prepare_q8_dense_attend(cfg, q_out, c, pt, sl, B.alloc_workspace(cfg))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        sl.zero_()                                  # (a warm-up that appends nothing)
        append()
        attend()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            append()
            attend()
    torch.cuda.synchronize()
    for t in range(T):
        for a, b in zip((q, k, v), steps[t]):
            a.copy_(b)
        sl.copy_(torch.tensor([L + t + 1 for L in lens0], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        o, l = attend.outputs
        assert torch.equal(o, want[t][0]) and torch.equal(l, want[t][1]), t
    for a, b in ((eager.k, c.k), (eager.v, c.v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(eager.k_scale, c.k_scale) and torch.equal(eager.v_scale, c.v_scale)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("P,rank", [(16, 8), (16, 2), (16, 15), (32, 8), (32, 12), (64, 8), (64, 9)])
def test_q8_build_equals_the_build_of_the_decoded_keys(code, P, rank):
    """Summaries from codes are those of the fp32 keys code * scale, bit for bit, for every
    page and for a list; what names no complete page is skipped."""
    lens = [P * 5 + 3, P - 1, P * 2, 0]
    st = Step([0] * 4, lens, P=P, kv="fp32", q="fp32", seed=rank)
    st.cfg.rank = rank
    print(f"[q8 build] {code} P={P} r={rank}", flush=True)
    kc, vc, ks, vs = _cache_of(st, code, seed=rank)
    cache = C.Q8Cache(kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda())
    decoded = (kc.float() * ks[..., None, None]).cuda()
    for lst in (None, torch.tensor([[0, 4], [2, 0], [0, 5], [1, 0], [7, 0], [0, -1]], dtype=torch.int32).cuda()):
        want, got = B.alloc_summaries(st.cfg), B.alloc_summaries(st.cfg)
        want.fill_(7)
        got.fill_(7)
        B.build_summaries(st.cfg, decoded, st.pt, st.sl, want, lst)
        C.q8_build_summaries(st.cfg, cache, st.pt, st.sl, got, lst)
        torch.cuda.synchronize()
        assert torch.equal(want, got)
        assert int((got != 7).any(-1).any(-1).sum()) == (7 if lst is None else 2)
    C.q8_build_summaries(st.cfg, cache, st.pt, st.sl, got, torch.zeros(0, 2, dtype=torch.int32).cuda())


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("P", [16, 64])
def test_locks_step_over_an_8_bit_cache(code, P):
    """Prompts appended, their summaries built from the codes, then tokens: append, build of
    the pages that fill, selection, attention over the selected pages -- against the same
    step over an fp32 cache of the decoded values."""
    H, G, lens0, T = 2, 4, [40 * P + 3, 25 * P - 2], 5
    S = 2
    mp = 48
    cfg = B.Config(S, G * H, H, 8, 8 * P, mp, S * mp, page_size=P)
    wide = B.Config(S, G * H, H, 8, 8 * P, mp, S * mp, B.LOCKS_FP32, B.LOCKS_BF16, page_size=P)
    g = torch.Generator().manual_seed(5 + P)
    pt = torch.randperm(S * mp, generator=g).int().reshape(S, mp).cuda()
    rope = C.Rope(C.rope_table(mp * P, 128))
    mk = lambda n: [torch.randn(n, h, D, generator=g).bfloat16().cuda() for h in (G * H, H, H)]
    q, k, v = mk(sum(lens0))
    cache = C.alloc_q8_cache(cfg, code)
    summ = B.alloc_summaries(cfg)
    sl = torch.tensor(lens0, dtype=torch.int32).cuda()
    cu = torch.tensor([0, lens0[0], sum(lens0)], dtype=torch.int32).cuda()
    C.q8_append_kv(cfg, k, v, cache, pt, sl, rope, cu_tokens=cu)
    C.q8_build_summaries(cfg, cache, pt, sl, summ)
    ws, wws = B.alloc_workspace(cfg), B.alloc_workspace(wide)
    for t in range(T):
        q, k, v = mk(S)
        lens = [L + t + 1 for L in lens0]
        sl = torch.tensor(lens, dtype=torch.int32).cuda()
        full = [[s, L // P - 1] for s, L in enumerate(lens) if L % P == 0]
        qr = C.q8_append_kv(cfg, k, v, cache, pt, sl, rope, q=q)
        if full:
            C.q8_build_summaries(cfg, cache, pt, sl, summ, torch.tensor(full, dtype=torch.int32).cuda())
        ids, _ = B.select(cfg, qr, summ, pt, sl, ws)
        out, lse = C.q8_sparse_attend(cfg, qr, cache, pt, sl, ids, ws)
        kd, vd = (c.float() * x[..., None, None] for c, x in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        ws2 = B.alloc_summaries(wide)
        B.build_summaries(wide, kd, pt, sl, ws2)
        ids2, _, out2, lse2 = B.decode_step(wide, qr, kd, vd, pt, sl, ws2, wws)
        torch.cuda.synchronize()
        assert torch.equal(ids, ids2)
        st = Step([0] * S, lens, H=H, G=G, P=P, seed=1)
        st.table, st.cfg = pt.cpu(), cfg
        _check_attend(st, code, qr.cpu(), out, lse, *[x.cpu() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)],
                      lambda s, h: [int(j) for j in ids[s, h] if j >= 0])
        # both within the bound of the 64-bit result, so within twice of each other
        assert float((out - out2).abs().max()) < 1e-3 and float((lse - lse2).abs().max()) < 1e-3
    assert lens[1] // P > lens0[1] // P   # a page filled on the way


def test_q8_attend_with_table_checks():
    """A bad entry and a bad length are clamped and reported, as in the other attentions."""
    st = Step([0, 0], [100, 60], seed=9)
    kc, vc, ks, vs = _cache_of(st, torch.int8, poison=False)
    cache = C.Q8Cache(kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda())
    q = torch.randn(2, st.G * st.H, D, generator=st.gen).bfloat16().cuda()
    ws = B.alloc_workspace(st.cfg)
    good, _ = C.q8_dense_attend(st.cfg, q, cache, st.pt, st.sl, ws)
    pt, sl = st.table.clone(), torch.tensor([16 * st.cfg.max_pages_per_seq + 5, 60], dtype=torch.int32)
    pt[1, 2] = st.cfg.num_blocks
    pt[0] = torch.clamp(pt[0], min=0)
    B.set_table_checks(True)
    try:
        ok, _ = C.q8_dense_attend(st.cfg, q, cache, st.pt, st.sl, ws)
        assert B.table_errors(st.cfg, ws)[0] == 0 and torch.equal(ok, good)
        C.q8_dense_attend(st.cfg, q, cache, pt.cuda(), sl.cuda(), ws)
        word, rows = B.table_errors(st.cfg, ws)
        assert word == 3 and rows == [B.LOCKS_TABLE_E_LENGTH, B.LOCKS_TABLE_E_BLOCK]
    finally:
        B.set_table_checks(False)


def test_q8_dense_attend_in_a_wide_table():
    """The same sequences in a table far wider than they are: the work is cut by their lengths."""
    st = Step([0, 0, 0], [900, 0, 333], G=4, P=16, seed=5)
    kc, vc, ks, vs = _cache_of(st, torch.int8)
    cache = C.Q8Cache(kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda())
    q = torch.randn(3, 8, D, generator=st.gen).bfloat16()
    wide = torch.full((3, 40000), -1, dtype=torch.int32)
    wide[:, :st.table.shape[1]] = st.table
    st.cfg.max_pages_per_seq = 40000
    out, lse = C.q8_dense_attend(st.cfg, q.cuda(), cache, wide.cuda(), st.sl, B.alloc_workspace(st.cfg))
    torch.cuda.synchronize()
    _check_attend(st, torch.int8, q, out, lse, kc, vc, ks, vs, lambda s, h: range(-(-st.lens[s] // 16)))


def test_q8_attend_nan_and_one_output():
    """A NaN query stays NaN and touches no other head or sequence; the LSE is optional."""
    st = Step([0, 0], [300, 40], G=4, seed=6)
    kc, vc, ks, vs = _cache_of(st, torch.int8)
    cache = C.Q8Cache(kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda())
    q = torch.randn(2, 8, D, generator=st.gen).bfloat16().cuda()
    ws = B.alloc_workspace(st.cfg)
    want, lse = C.q8_dense_attend(st.cfg, q, cache, st.pt, st.sl, ws)
    q[0, 2, 17] = float("nan")
    out = torch.zeros(2, 8, D).cuda()
    got, none = C.q8_dense_attend(st.cfg, q, cache, st.pt, st.sl, ws, out=out, out_lse=None)
    nan = torch.zeros(2, 8, dtype=torch.bool).cuda()
    nan[0, 2] = True
    assert none is None and got is out
    assert bool(torch.isnan(got[nan]).all()) and torch.equal(got[~nan], want[~nan])


def test_empty_appends():
    """No new rows at all, and a batch in which no sequence has any: nothing changes."""
    st = Step([5, 20], [0, 0], seed=2)
    cache = C.alloc_q8_cache(st.cfg)
    cache.k_scale += 1
    kc = torch.ones(st.cfg.num_blocks, st.H, 16, D, dtype=torch.bfloat16).cuda()
    rope = C.Rope(C.rope_table(64, 128))
    for n in (0, 3):                                  # (three rows of padding)
        k = torch.ones(n, st.H, D, dtype=torch.bfloat16).cuda()
        q = torch.ones(n, st.G * st.H, D, dtype=torch.bfloat16).cuda()
        q_out = torch.full_like(q, 3)
        C.q8_append_kv(st.cfg, k, k, cache, st.pt, st.sl, rope, cu_tokens=st.cu_dev, q=q, q_out=q_out)
        C.rope_append_kv(st.cfg, k, k, kc, kc, st.pt, st.sl, rope, cu_tokens=st.cu_dev, q=q, q_out=q_out)
        assert bool((q_out == 3).all())
    assert bool((cache.k_scale == 1).all()) and not bool(cache.k.any()) and bool((kc == 1).all())


def test_long_cache_offsets_pass_32_bits():
    """Blocks whose codes lie past 4 GiB, and a cache past 2^31 elements: the last blocks are
    appended to and attended."""
    P, H = 64, 8
    nb = (5 << 30) // (H * P * D)
    cfg = B.Config(1, H, H, 2, 128, 4, nb, page_size=P)
    cache = C.Q8Cache(*(torch.zeros(nb, H, P, D, dtype=torch.int8, device="cuda") for _ in range(2)),
                      *(torch.zeros(nb, H, device="cuda") for _ in range(2)))
    tab = torch.tensor([[nb - 1, 0, nb - 2, 1]], dtype=torch.int32)
    g = torch.Generator().manual_seed(2)
    T = 150
    k, v = (torch.randn(T, H, D, generator=g).bfloat16() for _ in range(2))
    sl = torch.tensor([T], dtype=torch.int32).cuda()
    C.q8_append_kv(cfg, k.cuda(), v.cuda(), cache, tab.cuda(), sl, cu_tokens=torch.tensor([0, T], dtype=torch.int32).cuda())
    q = torch.randn(1, H, D, generator=g).bfloat16()
    out, lse = C.q8_dense_attend(cfg, q.cuda(), cache, tab.cuda(), sl, B.alloc_workspace(cfg))
    torch.cuda.synchronize()
    for b in (nb - 1, 0, nb - 2):
        assert int((cache.k[b] != 0).sum()) > 0
    assert int((cache.k[1:nb - 2] != 0).any())== 0
    kk = torch.stack([cache.k[int(b)].cpu() for b in tab[0, :3]])
    vv = torch.stack([cache.v[int(b)].cpu() for b in tab[0, :3]])
    ks, vs = (x[tab[0, :3].long().cuda()].cpu() for x in (cache.k_scale, cache.v_scale))
    st = Step([0], [T], H=H, G=1, P=P)
    st.table = torch.tensor([[0, 1, 2]])
    _check_attend(st, torch.int8, q, out, lse, kk, vv, ks, vs, lambda s, h: range(3))


@pytest.mark.parametrize("code", CODES)
def test_q8_attend_scales_of_any_sign_and_size(code):
    """Scales of both signs, over six orders of magnitude, and zero."""
    st = Step([0, 0], [1500, 70], G=4, P=16, seed=8)
    kc, vc, ks, vs = _cache_of(st, code, seed=8)
    sign = torch.randint(0, 2, ks.shape, generator=st.gen) * 2.0 - 1.0
    far = 10.0 ** torch.randint(-6, 1, ks.shape, generator=st.gen).float()
    ks, vs = ks * sign, vs * sign.flip(0) * far
    vs[st.table[0, 3]] = 0
    cache = C.Q8Cache(kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda())
    q = torch.randn(2, 8, D, generator=st.gen).bfloat16()
    ws = B.alloc_workspace(st.cfg)
    out, lse = C.q8_dense_attend(st.cfg, q.cuda(), cache, st.pt, st.sl, ws)
    torch.cuda.synchronize()
    _check_attend(st, code, q, out, lse, kc, vc, ks, vs, lambda s, h: range(-(-st.lens[s] // 16)))
    # value scales of one sign only
    cache.v_scale.copy_(-vs.abs())
    out, lse = C.q8_dense_attend(st.cfg, q.cuda(), cache, st.pt, st.sl, ws)
    torch.cuda.synchronize()
    _check_attend(st, code, q, out, lse, kc, vc, ks, -vs.abs(), lambda s, h: range(-(-st.lens[s] // 16)))


@pytest.mark.parametrize("cu", [[0, 9, 3, 12], [0, -5, 40, 12], [4, 2, 0, 12], [12, 12, 12, 12], [0, 1 << 30, 1, 12]])
@pytest.mark.parametrize("P", [16, 32])
def test_appends_with_rows_out_of_order_stay_in_their_blocks(cu, P):
    """cu_tokens that does not ascend: whatever is written lies in the table's blocks and in
    the rows' outputs (many sequences search it in another way)."""
    for S in (3, 90):
        st = Step([5] * S, [4] * S, P=P, seed=1)
        cud = torch.tensor(cu[:3] * (S // 3) + [cu[3]], dtype=torch.int32).cuda()
        k = torch.ones(12, st.H, D, dtype=torch.bfloat16).cuda()
        kc = torch.zeros(st.cfg.num_blocks, st.H, P, D, dtype=torch.bfloat16).cuda()
        cache = C.alloc_q8_cache(st.cfg)
        outside = torch.ones(st.cfg.num_blocks, dtype=torch.bool)
        outside[st.table[st.table >= 0].long()] = False
        C.rope_append_kv(st.cfg, k, k, kc, kc, st.pt, st.sl, cu_tokens=cud)
        C.q8_append_kv(st.cfg, k, k, cache, st.pt, st.sl, cu_tokens=cud)
        assert outside.any() and not kc[outside].any() and not cache.k[outside].any()
        assert not cache.k_scale[outside].any() and not cache.v[outside].any()


def test_two_calls_at_once():
    """Two attentions and two appends on two streams, each with its own buffers."""
    st = Step([0, 0, 0], [3000, 17, 900], G=4, seed=4)
    made = []
    for i, code in enumerate(CODES):
        kc, vc, ks, vs = (x.cuda() for x in _cache_of(st, code, seed=i, poison=False))
        q = torch.randn(3, 8, D, generator=st.gen).bfloat16().cuda()
        store = C.Q8Cache(kc, vc, ks, vs)
        want = C.q8_dense_attend(st.cfg, q, store, st.pt, st.sl, B.alloc_workspace(st.cfg))
        attend = C.prepare_q8_dense_attend(st.cfg, q, store, st.pt, st.sl, B.alloc_workspace(st.cfg))
        wide = Step([0, 0], [700, 900], seed=5 + i)
        rows = [wide.k.cuda(), wide.v.cuda(), wide.q.cuda()]
        twin = [C.alloc_q8_cache(wide.cfg, code) for _ in range(2)]
        C.q8_append_kv(wide.cfg, rows[0], rows[1], twin[0], wide.pt, wide.sl, cu_tokens=wide.cu_dev)
        append = C.prepare_q8_append_kv(wide.cfg, rows[0], rows[1], twin[1], wide.pt, wide.sl,
                                        cu_tokens=wide.cu_dev)
        made.append((want, attend, twin, append))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(4):
        for s, (_, attend, _, append) in zip(streams, made):
            attend(s)
            append(s)
    torch.cuda.synchronize()
    for want, attend, twin, _ in made:
        assert torch.equal(attend.outputs[0], want[0]) and torch.equal(attend.outputs[1], want[1])
        assert torch.equal(twin[0].k.view(torch.uint8), twin[1].k.view(torch.uint8))
        assert torch.equal(twin[0].v_scale, twin[1].v_scale)


@pytest.mark.parametrize("wide", [1, 30])
def test_thousands_of_sequences(wide):
    """More sequences than one search round holds: appended without rotation and attended, in a
    table of their width (a block a list) and in a wide one (shares)."""
    S, P, H = 4500, 16, 1
    g = torch.Generator().manual_seed(12)
    past = torch.randint(0, 14, (S,), generator=g)
    new = torch.randint(0, 3, (S,), generator=g)
    sl = past + new
    cfg = B.Config(S, 2, H, 8, 64, 20 * wide, S + 5, B.LOCKS_FP32, page_size=P)
    pt = torch.full((S, 20 * wide), -1, dtype=torch.int32)
    pt[:, 0] = torch.randperm(S + 5, generator=g)[:S].int()
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]).int()
    n = int(cu[-1])
    # rows whose largest magnitude is 127 in every page: the scale is 1 and codes are the rows
    rows = torch.randint(-127, 128, (2, n, H, D), generator=g).float()
    rows[..., 7] = 127.0
    kc, vc = (torch.zeros(S + 5, H, P, D).cuda() for _ in range(2))
    cache = C.alloc_q8_cache(cfg)
    old = torch.randint(-127, 128, cache.k.shape, generator=g).to(torch.int8)
    cache.k.copy_(old), cache.v.copy_(old.flip(0))
    cache.k_scale.fill_(1.0), cache.v_scale.fill_(1.0)
    want_k, want_v = old.float(), old.flip(0).float()
    dev = [pt.cuda(), sl.int().cuda()]
    for call, store in ((C.rope_append_kv, (kc, vc)), (C.q8_append_kv, (cache,))):
        call(cfg, rows[0].cuda(), rows[1].cuda(), *store, *dev, cu_tokens=cu.cuda())
    seq = torch.repeat_interleave(torch.arange(S), new)
    at = past[seq] + torch.arange(n) - cu[seq].long()
    blk = pt[seq, 0].long()
    plain = torch.zeros(2, S + 5, H, P, D)
    plain[0][blk, :, at], plain[1][blk, :, at] = rows[0], rows[1]
    want_k[blk, :, at], want_v[blk, :, at] = rows[0], rows[1]
    assert torch.equal(kc.cpu(), plain[0]) and torch.equal(vc.cpu(), plain[1])
    assert torch.equal(cache.k.cpu().float(), want_k) and torch.equal(cache.v.cpu().float(), want_v)
    assert bool((cache.k_scale == 1).all()) and bool((cache.v_scale == 1).all())
    cfg.kv_dtype = B.LOCKS_BF16
    q = (torch.randn(S, 2, D, generator=g) / 64).bfloat16()
    out, lse = C.q8_dense_attend(cfg, q.cuda(), cache, *dev, B.alloc_workspace(cfg))
    K, V = want_k[pt[:, 0].long(), 0].double(), want_v[pt[:, 0].long(), 0].double()
    z = torch.matmul(q.double(), K.transpose(1, 2).contiguous()) / D ** 0.5
    z = torch.where(torch.arange(P) < sl[:, None, None], z, -torch.inf)
    big = torch.matmul(q.double().abs(), K.abs().transpose(1, 2).contiguous()).amax() / D ** 0.5
    want = torch.matmul(torch.softmax(z, -1), V)
    want[sl == 0] = 0
    dz = 128 * 2.0 ** -24 * float(big)
    assert bool(((out.cpu().double() - want).abs() <= (2 * dz + 2.0 ** -15) * 127).all())
    lw = torch.logsumexp(z, -1)
    assert torch.equal(torch.isneginf(lse.cpu()), torch.isneginf(lw))
    live = sl > 0
    assert bool(((lse.cpu().double() - lw)[live].abs() <= dz + 2.0 ** -18 * (lw[live].abs() + 1)).all())
