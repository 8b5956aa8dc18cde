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


# ---------------------------------------------------------------- attention's arithmetic

def _one_page_store(S, H, code, codes, k_scale, v_scale):
    """Sequence s's tokens lie in block s."""
    k, v = codes
    tab = torch.arange(S, dtype=torch.int32)[:, None].contiguous()
    return C.Q8Cache(k.to(code).cuda(), v.to(code).cuda(), k_scale.cuda(), v_scale.cuda()), tab.cuda()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("q", ["bf16", "fp32"])
def test_weights_round_without_bias(code, q):
    """Over values that are all the same the output is that value: the roundings of the weights
    must not drift to one side.  Of 32,768 outputs (2,048 sequences of 32 tokens, 16 heads) the mean
    signed error is less than half a float32 step, 2^-25: a weight in two f16 terms rounded to
    nearest is off by at most 2^-23 with a mean of zero, and the few float32 sums stay below 2^-20
    together, so the mean of N = 2^15 errors passes t = 2^-25 with a probability of at most
    2 exp(-2 N t^2 / (2^-19)^2) = 2 exp(-16).  Terms rounded toward zero have a mean of -2^-23.7."""
    S, H, G, P = 2048, 1, 16, 32
    cfg = B.Config(S, G * H, H, 8, 2 * P, 1, S, B.LOCKS_FP32, LK[q], page_size=P)
    g = torch.Generator().manual_seed(21)
    k = torch.randint(-100, 100, (S, H, P, D), generator=g).float()
    v = torch.full((S, H, P, D), 96.0)                                   # (a code of both kinds)
    vs = torch.rand(S, H, generator=g) + 0.5
    store, pt = _one_page_store(S, H, code, (k, v), torch.full((S, H), 1.0 / 128), vs)
    qq = (torch.randn(S, G, D, generator=g) * 2).to(DT[q]).cuda()
    sl = torch.full((S,), P, dtype=torch.int32).cuda()
    out, _ = C.q8_dense_attend(cfg, qq, store, pt, sl, B.alloc_workspace(cfg))
    want = 96.0 * vs.double()[:, :, None]
    off = (out.cpu().double() - want) / want
    print(f"[weights] {code} {q} mean 2^{np.log2(abs(float(off.mean()))):.1f} largest 2^"
          f"{np.log2(float(off.abs().max())):.1f}", flush=True)
    assert float(off.abs().max()) <= 2.0 ** -20
    assert abs(float(off.mean())) <= 2.0 ** -25


@pytest.mark.parametrize("code", CODES)
def test_fp32_queries_with_one_large_channel(code):
    """fp32 queries in two f16 terms: an element is held to 2^-23 of itself or 2^-39 of the head's
    largest (the second term's smallest step is 2^-24 where the largest is 2^14 or more, and half of
    that is lost), whichever is more.  One channel of 2^20 meets keys that are zero there, so a
    logit is off by sum |k| (2^-23 |q| + 2^-39 2^20) / sqrt d and the float32 sum's 256 2^-24
    sum |q k| / sqrt d; outputs by twice that and 2^-19 for the weights and the sums."""
    S, H, G, P = 40, 1, 4, 64
    cfg = B.Config(S, G * H, H, 8, 2 * P, 1, S, B.LOCKS_FP32, B.LOCKS_FP32, page_size=P)
    g = torch.Generator().manual_seed(22)
    k = torch.randint(-100, 100, (S, H, P, D), generator=g).float()
    k = k.to(code).float()
    k[..., 77] = 0
    v = torch.randint(-100, 100, (S, H, P, D), generator=g).to(code).float()
    ks, vs = torch.full((S, H), 1.0 / 256), torch.full((S, H), 1.0 / 64)
    store, pt = _one_page_store(S, H, code, (k, v), ks, vs)
    qq = torch.randn(S, G, D, generator=g) * 2
    qq[..., 77] = 2.0 ** 20
    lens = torch.randint(1, P + 1, (S,), generator=g).int()
    out, lse = C.q8_dense_attend(cfg, qq.cuda(), store, pt, lens.cuda(), B.alloc_workspace(cfg))
    for s in range(S):
        L = int(lens[s])
        K, V, Q = k[s, 0, :L].double() / 256, v[s, 0, :L].double() / 64, qq[s].double()
        z = Q @ K.t() / D ** 0.5
        dz = ((Q.abs() * (2.0 ** -23 + 256 * 2.0 ** -24)) @ K.abs().t()
              + 2.0 ** -19 * K.abs().sum(1)).amax(1) / D ** 0.5
        # (the large channel's products are zero: they add nothing to a sum)
        assert float((Q[:, 77, None] * K[None, :, 77]).abs().max()) == 0
        want = torch.softmax(z, -1) @ V
        bound = (2 * dz + 2.0 ** -19)[:, None] * V.abs().amax(0)
        assert bool(((out[s].cpu().double() - want).abs() <= bound).all()), s
        w = torch.logsumexp(z, -1)
        assert bool(((lse[s].cpu().double() - w).abs() <= dz + 2.0 ** -20 * (w.abs() + 1)).all()), s


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("exps", [(126, 127), (-149, -126), (-149, 127), (-100, 100)])
def test_value_scales_of_any_exponent(code, exps):
    """Value scales from the smallest subnormal to 2^127, codes of one step.  One token a
    sequence and several of one page: weights are held to 2^-20 and the result to one more rounding
    (2^-24, or half a subnormal, 2^-150)."""
    S, H, G, P = 64, 1, 4, 16
    cfg = B.Config(S, G, H, 8, 2 * P, 1, S, B.LOCKS_FP32, B.LOCKS_FP32, page_size=P)
    g = torch.Generator().manual_seed(23)
    k = torch.randint(-100, 100, (S, H, P, D), generator=g).float()
    sign = torch.randint(0, 2, (S, H, 1, D), generator=g) * 2.0 - 1.0
    v = sign.expand(S, H, P, D).contiguous()      # the same in every token: the output is +-scale
    e = torch.tensor(exps)[torch.randint(0, 2, (S, H), generator=g)]
    vs = torch.ldexp(torch.ones(S, H, dtype=torch.float64), e).float()
    assert bool((vs > 0).all()) and bool(torch.isfinite(vs).all())
    store, pt = _one_page_store(S, H, code, (k, v), torch.full((S, H), 1.0 / 64), vs)
    for L in (1, 16):
        if L > 1 and max(exps) > 123:
            continue                # (weights times values, summed before the division, pass float32)
        sl = torch.full((S,), L, dtype=torch.int32).cuda()
        out, _ = C.q8_dense_attend(cfg, torch.randn(S, G, D, generator=g).cuda(), store, pt, sl,
                                   B.alloc_workspace(cfg))
        want = (sign[:, :, 0] * vs[..., None]).double().expand(S, G, D)
        assert bool(((out.cpu().double() - want).abs() <= want.abs() * 2.0 ** -19 + 2.0 ** -149).all()), L


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("P", [16, 64])
def test_q8_append_behind_a_negative_scale(code, P):
    """Attention takes scales of either sign, so appends do too: behind rows whose page has a
    negative scale, a smaller row is coded with it, and a larger one makes its magnitude grow;
    either way the earlier rows keep their values."""
    S, H = 3, 2
    cfg = B.Config(S, H, H, 8, 2 * P, 1, S, B.LOCKS_FP32, B.LOCKS_FP32, page_size=P)
    g = torch.Generator().manual_seed(24)
    cache = C.alloc_q8_cache(cfg, code)
    old = torch.randint(-8, 9, (S, H, P, D), generator=g).float()
    for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        c.copy_(old)
        s.fill_(-1.0)
    x = torch.ones(S, H, D)
    x[0] = 0.0                                   # nothing to scale by
    x[1] *= 5.0                                  # fits the page's scale
    x[2] *= 4.0 * _most(code)                    # needs four times of it
    pt = torch.arange(S, dtype=torch.int32)[:, None].contiguous().cuda()
    C.q8_append_kv(cfg, x.cuda(), x.cuda(), cache, pt, torch.full((S,), 4, dtype=torch.int32).cuda())
    for c, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        c, scale = c.cpu().float(), scale.cpu()
        assert bool((scale[:2] == -1.0).all()) and bool((scale[2] == 4.0).all())
        values = c * scale[..., None, None]
        assert torch.equal(values[:2, :, :3], -old[:2, :, :3])
        assert bool(((values[2, :, :3] + old[2, :, :3]).abs() <= (2.0 if code == torch.int8 else 0.0)).all())
        assert torch.equal(values[:, :, 3], x)
    z = torch.full((S, H, D), -INF)              # an infinity keeps its sign
    C.q8_append_kv(cfg, z.cuda(), z.cuda(), cache, pt, torch.full((S,), 5, dtype=torch.int32).cuda())
    for c, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        c, scale = c.cpu().float(), scale.cpu()
        assert bool((scale[:2] == -1.0).all()) and bool((scale[2] == 4.0).all())
        assert torch.equal((c * scale[..., None, None])[:, :, 4],
                           (-_most(code) * scale.abs())[..., None].expand(S, H, D))


# ---------------------------------------------------------------- one token a sequence

ONE_TOKEN_LENS = [[1], [33], [16, 0, 17, 1, 64], [0, 0], [1 + 7 * i % 50 if i % 9 else 0 for i in range(150)]]


@pytest.mark.parametrize("lens", range(len(ONE_TOKEN_LENS)))
@pytest.mark.parametrize("rot,inter,axes,given", [(0, False, 1, False), (128, False, 1, False), (64, True, 1, True),
                                                  (48, False, 2, True), (112, True, 3, True)])
@pytest.mark.parametrize("q,kv", [("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32"), ("fp32", "bf16")])
def test_rope_append_of_one_token_a_sequence(q, kv, rot, inter, axes, given, lens):
    """Without cu_tokens row s is the newest token of sequence s; a sequence of length 0 has none,
    its output row stays.  Values are within 2^-22 (|a c| + |b s|) of the 64-bit ones, bf16 half a
    step more."""
    lens = ONE_TOKEN_LENS[lens]
    S, H, G = len(lens), 2, (4, 7, 1)[len(lens) % 3]
    P = (16, 32, 64)[S % 3]
    g = torch.Generator().manual_seed(S)
    mp = max(lens) // P + 2
    tab = torch.randperm(S * mp + 3, generator=g).int()[:S * mp].reshape(S, mp)
    cfg = B.Config(S, G * H, H, 8, 2 * P, mp, S * mp + 3, LK[kv], LK[q], page_size=P)
    print(f"[one token] S={S} P={P} {q}/{kv} rot={rot} inter={inter} axes={axes}", flush=True)
    wide = torch.randn(S, G * H + 2 * H + 1, D, generator=g)
    qr, kr, vr = wide[:, :G * H].to(DT[q]), wide[:, G * H:G * H + H].to(DT[kv]), wide[:, G * H + H:-1].to(DT[kv])
    kc, vc = (torch.randn(cfg.num_blocks, H, P, D, generator=g).to(DT[kv]) for _ in range(2))
    q_out = torch.full((S, G * H, D), 7.0, dtype=DT[q])
    rope = pos = None
    half = rot // 2
    split = {1: [half], 2: [5, half - 5], 3: [half // 4, 3, half - half // 4 - 3]}[axes]
    if rot:
        rope = C.Rope(C.rope_table(300, rot), inter, None if axes == 1 else split)
        if given:
            pos = torch.randint(0, 300, (axes, S), generator=g, dtype=torch.int32)
    kd, vd, qo = kc.cuda(), vc.cuda(), q_out.cuda()
    # rows as slices of wider buffers
    src = [torch.nn.functional.pad(t, (0, 0, 1, 2), value=NAN).cuda()[:, 1:-2] for t in (qr, kr, vr)]
    got = C.rope_append_kv(cfg, src[1], src[2], kd, vd, tab.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                           rope, positions=None if pos is None else pos.cuda(), q=src[0], q_out=qo)
    assert got is qo
    want_q, want_k, bound_q, bound_k = q_out.double(), kc.double(), torch.zeros(q_out.shape, dtype=torch.float64), \
        torch.zeros(kc.shape, dtype=torch.float64)
    first, second = (list(range(0, rot, 2)), list(range(1, rot, 2))) if inter else (list(range(half)), list(range(half, rot)))
    axis = [a for a, n in enumerate(split) for _ in range(n)]
    for s, L in enumerate(lens):
        if L == 0:
            continue
        b, i = int(tab[s, (L - 1) // P]), (L - 1) % P
        vc[b, :, i] = vr[s]
        for x, want, bound, at, dt in ((qr[s], want_q, bound_q, (s,), q), (kr[s], want_k, bound_k, (b, slice(None), i), kv)):
            x = x.double()
            y, e = x.clone(), torch.zeros_like(x)
            if rot:
                p = [L - 1] * axes if pos is None else pos[:, s].tolist()
                rows = rope.table.cpu().double()[[p[a] for a in axis]]
                c, sn = (rows[range(half), [o + i for i in range(half)]] for o in (0, half))
                xa, xb = x[:, first], x[:, second]
                y[:, first], y[:, second] = xa * c - xb * sn, xb * c + xa * sn
                e[:, first] = ((xa * c).abs() + (xb * sn).abs()) * 2.0 ** -22
                e[:, second] = ((xb * c).abs() + (xa * sn).abs()) * 2.0 ** -22
                if dt == "bf16":
                    e[:, :rot] = e[:, :rot] * (1 + 2.0 ** -8) + y[:, :rot].abs() * 2.0 ** -8
            want[at], bound[at] = y, e
    assert torch.equal(vd.cpu(), vc)
    assert bool(((kd.cpu().double() - want_k).abs() <= bound_k).all())
    assert bool(((qo.cpu().double() - want_q).abs() <= bound_q).all())


# ---------------------------------------------------------------- streams

def _stream_of(t):
    """The stream that a tensor's memory was allocated on."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]


def test_outputs_belong_to_the_stream_of_their_call():
    """Outputs that a call on another stream allocates are that stream's memory: the current
    stream's may still be in use by the work queued there."""
    S, H, G, P = 64, 2, 8, 16
    cfg = B.Config(S, G * H, H, 8, 2 * P, 4, 4 * S, page_size=P)
    g = torch.Generator().manual_seed(31)
    q, k, v = (torch.randn(S, h, D, generator=g).bfloat16().cuda() for h in (G * H, H, H))
    pt = torch.arange(4 * S, dtype=torch.int32).reshape(S, 4).cuda()
    sl = torch.full((S,), 5, dtype=torch.int32).cuda()
    ids = torch.zeros(S, H, cfg.k, dtype=torch.int32).cuda()
    ids[..., 1:] = -1
    kc, vc = (torch.zeros(4 * S, H, P, D, dtype=torch.bfloat16).cuda() for _ in range(2))
    store, ws, side = C.alloc_q8_cache(cfg), B.alloc_workspace(cfg), torch.cuda.Stream()
    calls = [lambda s: C.rope_append_kv(cfg, k, v, kc, vc, pt, sl, q=q, stream=s),
             lambda s: C.q8_append_kv(cfg, k, v, store, pt, sl, q=q, stream=s),
             lambda s: C.q8_dense_attend(cfg, q, store, pt, sl, ws, stream=s),
             lambda s: C.q8_sparse_attend(cfg, q, store, pt, sl, ids, ws, stream=s)]
    torch.cuda.synchronize()
    for call in calls:
        want = call(None)
        torch.cuda.synchronize()
        got = call(side)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            again = call(None)
        torch.cuda.synchronize()
        want, got, again = (x if isinstance(x, tuple) else (x,) for x in (want, got, again))
        for a, b, c in zip(want, got, again):
            assert torch.equal(a, b) and torch.equal(a, c)
            assert _stream_of(a) == torch.cuda.current_stream().cuda_stream
            assert _stream_of(b) == _stream_of(c) == side.cuda_stream
