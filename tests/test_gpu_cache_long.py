"""GPU checks of the 8-bit attention where lists are long: shares of more than 8 units, waves of
more than one round of 64 units, lists cut into many pieces, and the workspace that holds them.

Against float64 attention of the whole list, formed on the GPU one head at a time.  With p the
softmax weights relative to the largest, l their sum and v the values:
* a logit is off by at most dz = n 2^-24 max sum |q k| / sqrt d: 128 products of bf16 queries, summed
  in float32, and six for its scales and its distance from the largest make n = 134; float32 queries
  enter as two f16 terms that hold an element to 2^-23, so 2 x 128 products and two more, n = 264.
  It moves p by a factor within exp(+-dz);
* weights in two f16 terms are held to 2^-23, sums of weights and products pass at most 1,024
  roundings of 2^-24 on any path (a wave's rounds, four waves, the pieces): together 2^-13 with the
  division, of sum p |v| / l;
* what two f16 terms cannot hold of a weight times its scale is at most 2^-39 of the largest scale
  of its wave: n_tokens 2^-39 max |v| / l.
So |out - want| <= (2 dz + 2^-13) sum p |v| / l + n_tokens 2^-39 max |v| / l, and |lse - want| <=
dz + 2^-13 + 2^-22 |want|."""
import numpy as np
import pytest
import torch

from paper_2607_24555_amd import cache as C
from paper_2607_24555_amd import locks as B

pytestmark = pytest.mark.gpu
D = 128
CODES = [torch.int8, torch.float8_e4m3fn]


def _align(n):
    return (n + 255) // 256 * 256


def _workspace(cfg):
    """A workspace whose bytes from the checked tables on hold a pattern: with checks off no call
    uses them, so a partial written past the ones that were planned for would show there."""
    ws = B.alloc_workspace(cfg)
    err = int(B.lib().locks_table_error_offset(B.ctypes.byref(cfg.c())))
    tail = err - _align(4 * cfg.num_seqs) - _align(4 * cfg.num_seqs * cfg.max_pages_per_seq)
    assert 0 < tail < ws.numel()
    ws[tail:] = 0x5A
    return ws, ws[tail:]


def _store(lens, H, P, code, kind, seed, spare_pages=0):
    """A cache of the sequences in shuffled blocks, and its table.  kind "steps": value scales double
    every 40 units (eight times, then start again) while the codes halve as far as they go, so that
    values of all sizes of scale matter; "flat": scales around one size."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    S = len(lens)
    pages = [-(-L // P) for L in lens]
    nb = sum(pages) + 3
    mp = max(pages) + spare_pages
    perm = torch.randperm(nb, generator=g, device="cuda").int()
    pt = torch.full((S, mp), -1, dtype=torch.int32, device="cuda")
    index = torch.zeros(nb, dtype=torch.int64, device="cuda")           # page within its sequence
    off = 0
    for s in range(S):
        pt[s, :pages[s]] = perm[off:off + pages[s]]
        index[perm[off:off + pages[s]].long()] = torch.arange(pages[s], device="cuda")
        off += pages[s]
    codes = []
    e = (index * (P // 16) // 40 % 8).float() if kind == "steps" else torch.zeros(nb, device="cuda")
    for x in range(2):
        c = torch.empty(nb, H, P, D, dtype=code, device="cuda")
        for b in range(0, nb, 4096):
            y = torch.randn(min(4096, nb - b), H, P, D, generator=g, device="cuda") * 30
            if x == 1:       # (a mean, so that every piece of a list shows in its output)
                y = (y + 40) * torch.exp2(-e[b:b + 4096].clamp(max=4))[:, None, None, None]
            c[b:b + 4096] = y.clamp(-127, 127).round().to(code)
        codes.append(c)
    ks = torch.exp(0.2 * torch.randn(nb, H, generator=g, device="cuda")) * 0.02
    vs = torch.exp(0.2 * torch.randn(nb, H, generator=g, device="cuda")) * 0.02 * torch.exp2(e)[:, None]
    for t in (ks, vs):                                                  # blocks of no sequence
        t[perm[off:].long()] = float("nan")
    return C.Q8Cache(codes[0], codes[1], ks.contiguous(), vs.contiguous()), pt, nb


def _check(cfg, q, cache, pt, lens, out, lse, ids=None):
    H, P, G = cfg.num_kv_heads, cfg.page_size, cfg.num_q_heads // cfg.num_kv_heads
    n = 134 if q.dtype == torch.bfloat16 else 264
    worst = 0.0
    for s, L in enumerate(lens):
        for h in range(H):
            rows = slice(h * G, (h + 1) * G)
            mine = torch.arange(-(-L // P), device="cuda") if ids is None else ids[s, h][ids[s, h] >= 0].long()
            tok = (mine[:, None] * P + torch.arange(P, device="cuda")).reshape(-1)
            keep = tok < L
            if not bool(keep.any()):
                assert not bool(out[s, rows].any()) and bool(torch.isneginf(lse[s, rows]).all())
                continue
            b = pt[s][mine].long()
            K, V = ((c[b, h].double() * sc[b, h].double()[:, None, None]).reshape(-1, D)[keep]
                    for c, sc in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
            Q = q[s, rows].double()
            z = torch.matmul(K, Q.t().contiguous()).t() / D ** 0.5
            big = torch.matmul(K.abs(), Q.abs().t().contiguous()).amax(0) / D ** 0.5
            m = z.amax(1, keepdim=True)
            p = torch.exp(z - m)
            l = p.sum(1, keepdim=True)
            dz = (n * 2.0 ** -24 * big)[:, None]
            want = torch.matmul(p.contiguous(), V) / l
            bound = (2 * dz + 2.0 ** -13) * torch.matmul(p, V.abs()) / l
            bound += K.shape[0] * 2.0 ** -39 * V.abs().amax(0) / l
            d = (out[s, rows].double() - want).abs()
            worst = max(worst, float((d / bound).max()))
            assert bool((d <= bound).all()), (s, h, float((d / bound).max()))
            w = (m + torch.log(l))[:, 0]
            assert bool(((lse[s, rows].double() - w).abs() <= dz[:, 0] + 2.0 ** -13 + 2.0 ** -22 * w.abs()).all()), (s, h)
    print(f"  largest error {worst:.3f} of its bound", flush=True)


# lengths, KV heads, heads a group, page; what of it is long
LONG = {
    # one list in shares of 64 units, its 293 pieces merged by 16 waves a row
    "one list": ([300011], 1, 4, 16),
    # shares of 296 units, 74 a wave: a second round, and pieces of long, short and empty lists
    "second round": ([290001, 0, 12003, 517, 1], 8, 2, 16),
    "second round, large pages": ([150005, 140001, 9000, 33], 8, 3, 64),
    # more than 64 sequences, most lists cut in several shares of 208 units, and empty ones
    "many sequences": ([(977 * i) % 20000 if i % 7 else 0 for i in range(100)], 2, 16, 32),
}


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("kind", ["steps", "flat"])
@pytest.mark.parametrize("q", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", LONG)
def test_long_lists(name, q, kind, code):
    lens, H, G, P = LONG[name]
    S = len(lens)
    print(f"[long] {name} {q} {kind} {code}", flush=True)
    # (a table some wider than the sequences)
    cache, pt, nb = _store(lens, H, P, code, kind, seed=S + H, spare_pages=9)
    cfg = B.Config(S, G * H, H, 2, 2 * P, pt.shape[1], nb, B.LOCKS_BF16,
                   B.LOCKS_BF16 if q == torch.bfloat16 else B.LOCKS_FP32, page_size=P)
    g = torch.Generator(device="cuda").manual_seed(3)
    qq = (torch.randn(S, G * H, D, generator=g, device="cuda") * 1.5).to(q)
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws, tail = _workspace(cfg)
    out, lse = C.q8_dense_attend(cfg, qq, cache, pt, sl, ws)
    torch.cuda.synchronize()
    assert bool((tail == 0x5A).all())
    _check(cfg, qq, cache, pt, lens, out, lse)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("S,H,G,P", [(8, 8, 4, 16), (50, 4, 4, 32), (3, 1, 16, 64)])
def test_long_tables(S, H, G, P, code):
    """Tables of 128 units over 64, 200 and 3 lists: shares of 32 and 64 units that cut a list, and of
    8; some lists are shorter than the table, one is empty."""
    lens = [9000 - 171 * s for s in range(S)]
    lens[-1] = 0
    cache, pt, nb = _store(lens, H, P, code, "steps", seed=S)
    cfg = B.Config(S, G * H, H, 2, 2048, pt.shape[1], nb, page_size=P)
    g = torch.Generator(device="cuda").manual_seed(4)
    ids = torch.full((S, H, cfg.k), -1, dtype=torch.int32, device="cuda")
    for s, L in enumerate(lens):
        n = -(-L // P)
        for h in range(H):
            take = torch.randperm(n, generator=g, device="cuda")[:cfg.k].sort()[0].int()
            ids[s, h, :len(take)] = take
    if S > 3:
        ids[1, 0, 5:] = -1                       # a short list
        ids[2, H - 1] = -1                       # one that lists nothing
        ids[4, 0, ::2] = -1                      # gaps
    qq = torch.randn(S, G * H, D, generator=g, device="cuda").bfloat16()
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    print(f"[long tables] S={S} H={H} G={G} P={P} {code}", flush=True)
    ws, tail = _workspace(cfg)
    out, lse = C.q8_sparse_attend(cfg, qq, cache, pt, sl, ids, ws)
    torch.cuda.synchronize()
    assert bool((tail == 0x5A).all())
    _check(cfg, qq, cache, pt, lens, out, lse, ids)
