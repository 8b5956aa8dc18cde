"""The operators on single tokens of the paged cache as cases to time and to check: their
plain forms, and the calls that a serving loop makes of the library's.

* ``tree``  attention of several new tokens of each sequence, drafted as a tree or a run of
  a prompt, over everything cached before them and over those of each other that they see;
* ``mass``  the attention weight that every cached token got from the new ones, summed over
  a group's heads and added to what earlier steps left;
* ``pick``  the tokens of each KV head to keep: the first ones, the last ones and those of
  largest mass, in order;
* ``keep``  the rows of kept tokens (of an accepted branch, or of a pick) moved together at
  the front of the cache, in place, with their mass.

Activations are seeded draws: keys with a few outlier channels per head, as rotary models
have them, values without; masses span several orders of magnitude and hold ties.
"""
import math
import random

import torch

own = False

D = 128
TORCH_OF = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _attend(name, op, seqs, lo, hi, new_lo, new_hi, q_heads, kv_heads, page=16, dtype="bf16",
            out="bf16", tree=True, empty=False, decay=1.0):
    c = {"op": op, "seqs": seqs, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi,
         "q_heads": q_heads, "kv_heads": kv_heads, "page": page, "dtype": dtype, "tree": tree,
         "empty": empty}
    c.update({"out": out} if op == "tree" else {"decay": decay})
    return dict(c, name=name) if name else c


def _pick(name, seqs, lo, hi, kv_heads, keep, sink, recent, page=16, ties=False):
    c = {"op": "pick", "seqs": seqs, "lo": lo, "hi": hi, "kv_heads": kv_heads, "keep": keep,
         "sink": sink, "recent": recent, "page": page, "ties": ties}
    return dict(c, name=name) if name else c


def _keep(name, seqs, lo, hi, kv_heads, width, new=0, page=16, dtype="bf16"):
    c = {"op": "keep", "seqs": seqs, "lo": lo, "hi": hi, "kv_heads": kv_heads, "width": width,
         "new": new, "page": page, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's short run of guessed tokens: latency
        _attend("tree-run-4k", "tree", 1, 4099, 4099, 5, 5, 32, 8, tree=False),
        # a ragged batch, each sequence with a tree of drafted tokens
        _attend("tree-ragged", "tree", 8, 3000, 65535, 33, 64, 32, 8),
        # the longest context, sixteen heads a group, a small tree, exact outputs
        _attend("tree-1m", "tree", 1, 1048571, 1048571, 16, 16, 32, 2, page=32, out="fp32"),
        # float32 with seven heads a group, one sequence without anything cached
        _attend("tree-fp32", "tree", 3, 900, 5000, 61, 100, 28, 4, page=64, dtype="fp32", out="fp32",
                empty=True),
        # the next piece of several prompts, behind what is cached of them
        _attend("tree-prompts", "tree", 4, 6000, 9000, 700, 1024, 32, 8, tree=False),
        # a decode batch that keeps account of its tokens' weights
        _attend("mass-token", "mass", 64, 1500, 8192, 1, 1, 32, 8, tree=False, decay=0.96875),
        # long prompts judged by their last tokens
        _attend("mass-window", "mass", 8, 20000, 32768, 32, 32, 32, 8, tree=False),
        # one chat's cache cut to a quarter
        _pick("pick-4k", 1, 4099, 4099, 8, 1024, 4, 128),
        # long documents cut to a small cache, masses with ties
        _pick("pick-8x128k", 8, 131072, 131072, 8, 2048, 16, 512, ties=True),
        # the longest context
        _pick("pick-1m", 1, 1048571, 1048571, 2, 8192, 64, 1024, page=32),
        # the accepted branch of each sequence's tree
        _keep("keep-accepted", 64, 40, 400, 8, 8, new=32),
        # a pick's rows moved together, a list for each KV head
        _keep("keep-picked", 4, 12000, 16384, 8, 4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: up to 2^20 cached tokens, up to 1,024 new ones a
    sequence (128 in a tree), every page size, type and group."""
    op = rng.choice(["tree", "tree", "tree", "mass", "mass", "pick", "keep"])
    page = rng.choice([16, 16, 32, 64])
    kv = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 3, 4, 7, 8, 16]) if kv < 8 else rng.choice([1, 4, 5])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    seqs = _log(rng, 1, 24)
    if op in ("tree", "mass"):
        tree = rng.random() < 0.6
        new = _log(rng, 1, 128 if tree else 1024)
        # pairs of query rows and tokens: within the largest listed case's, a fifth of them in float32
        pairs = (1 << 28) // (5 if dtype == "fp32" else 1)
        most = max(2 * new, min((1 << 20) // max(1, kv // 2), pairs // (new * g * kv)) // seqs)
        if most * seqs * new * g * kv > pairs:
            seqs = max(1, pairs // (most * new * g * kv))
        hi = _log(rng, max(2, new), max(2, most))
        return _attend(None, op, seqs, max(1, hi // 6), hi, max(1, new // 3), new, g * kv, kv, page=page,
                       dtype=dtype, out=rng.choice(["bf16", "fp32"]), tree=tree,
                       empty=rng.random() < 0.3, decay=rng.choice([1.0, 0.5, 0.96875]))
    if op == "pick":
        hi = _log(rng, 20, (1 << 21) // (kv * seqs))
        keep = max(1, min(_log(rng, 8, 8192), hi))
        sink = rng.choice([0, min(4, keep // 3)])
        return _pick(None, seqs, max(1, hi // 5), hi, kv, keep, sink, rng.randint(0, keep - sink), page,
                     rng.random() < 0.4)
    if rng.random() < 0.4:
        new = rng.randint(2, 128)
        return _keep(None, seqs, new, new + _log(rng, 1, 600), kv, rng.randint(1, min(new, 12)), new, page,
                     dtype)
    hi = _log(rng, 40, (1 << 18) // (kv * seqs))
    return _keep(None, seqs, max(1, hi // 3), hi, kv, _log(rng, 4, max(4, hi // 2)), 0, page, dtype)


# ---------------------------------------------------------------- inputs

def _lens(case):
    """Tokens of each sequence, new ones included, and how many are new; fixed by the case."""
    r = random.Random(1000003 * case["hi"] + 7919 * case["lo"] + case["seqs"])
    lens = [r.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]
    if case["op"] not in ("tree", "mass"):
        return lens, [case.get("new", 0)] * len(lens)
    new = [min(L, r.randint(case["new_lo"], case["new_hi"])) for L in lens]
    if case["empty"]:                         # a sequence that begins with these tokens
        lens[-1] = new[-1]
    return lens, new


def _seen(case):
    """Of each sequence, for each new token, which of the new tokens it sees, as the bits of
    a whole number.  A tree: its ancestors and itself; with `empty` the last sequence's first
    token sees none at all."""
    _, new = _lens(case)
    r = random.Random(31 * case["new_hi"] + case["seqs"])
    out = []
    for n in new:
        bits = []
        for i in range(n):
            parent = r.randint(max(-1, i - 9), i - 1) if case["tree"] else i - 1
            bits.append((bits[parent] if parent >= 0 else 0) | 1 << i)
        out.append(bits)
    if case["tree"] and case["empty"]:
        out[-1][0] = 0
    return out


def _table(lens, page, gen, dev):
    pages = [max(1, -(-L // page)) for L in lens]
    nb = sum(pages) + 3
    perm = torch.randperm(nb, generator=gen, device=dev).int()
    table = torch.full((len(lens), max(pages)), -1, dtype=torch.int32, device=dev)
    off = 0
    for s, n in enumerate(pages):
        table[s, :n] = perm[off:off + n]
        off += n
    return table, nb


def _cache(shape, mean, dtype, gen, dev):
    """Keys and values, filled in pieces."""
    out = [torch.empty(shape, dtype=dtype, device=dev) for _ in range(2)]
    step = max(1, (1 << 26) // math.prod(shape[1:]))
    for b0 in range(0, shape[0], step):
        b1 = min(shape[0], b0 + step)
        for i in (0, 1):
            x = torch.randn((b1 - b0, *shape[1:]), generator=gen, device=dev)
            out[i][b0:b1] = x + mean[None, :, None] if i == 0 else x
    return out


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + 41)
    lens, new = _lens(case)
    S, H, P = case["seqs"], case["kv_heads"], case["page"]
    table, nb = _table(lens, P, g, dev)
    mp = table.shape[1]
    st = {"case": case, "sl": torch.tensor(lens, dtype=torch.int32, device=dev), "pt": table, "nb": nb}
    mean = torch.zeros(H, D, device=dev)
    mean[:, torch.randperm(D, generator=g, device=dev)[:4]] = 6.0 * torch.sign(
        torch.randn(H, 4, generator=g, device=dev))
    dt = TORCH_OF[case.get("dtype", "bf16")]
    if case["op"] != "tree":
        # what earlier steps left: most tokens got little, some very much
        mass = torch.exp(2.0 * torch.randn(S, H, mp * P, generator=g, device=dev) - 4.0)
        if case.get("ties"):
            mass = torch.round(mass * 64.0) / 64.0
        st["mass"] = mass
    if case["op"] in ("tree", "mass"):
        n = sum(new)
        st["k"], st["v"] = _cache((nb, H, P, D), mean, dt, g, dev)
        cu = [0]
        for t in new:
            cu.append(cu[-1] + t)
        st["cu"] = torch.tensor(cu, dtype=torch.int32, device=dev)
        st["q"] = (1.7 * torch.randn(n, case["q_heads"], D, generator=g, device=dev)).to(dt)
        st["mask"] = None
        if case["tree"]:
            words = -(-max(new) // 32)
            flat = [[b >> 32 * w & 0xffffffff for w in range(words)] for seq in _seen(case) for b in seq]
            st["mask"] = torch.tensor(flat, dtype=torch.int64, device=dev).int()
        if case["op"] == "mass":
            del st["v"]
            lse = []                          # what the attention of the step returned
            for s in range(S):
                one = dict(st, case=dict(case, seqs=1, op="tree"), pt=table[s:s + 1, :-(-lens[s] // P)],
                           sl=st["sl"][s:s + 1], cu=st["cu"][s:s + 2] - st["cu"][s], q=st["q"][cu[s]:cu[s + 1]],
                           mask=None if st["mask"] is None else st["mask"][cu[s]:cu[s + 1]])
                z, rows = _logits(one, new[s])
                lse.append(torch.logsumexp(z, -1).reshape(case["q_heads"], new[s]).t())
            st["lse"] = torch.cat(lse).contiguous()
    elif case["op"] == "keep":
        st["k"], st["v"] = _cache((nb, H, P, D), mean, dt, g, dev)
        w, j = case["width"], torch.arange(mp * P, device=dev)
        first = torch.zeros(S, dtype=torch.int64, device=dev) if not case["new"] else st["sl"].long() - case["new"]
        heads = 1 if case["new"] else H
        # ascending draws from the tokens at hand; an accepted branch has one to `width` of them
        score = torch.rand(S, heads, mp * P, generator=g, device=dev)
        score = torch.where((j >= st["sl"][:, None, None]) | (j < first[:, None, None]),
                            torch.full_like(score, -1.0), score)
        got, ids = torch.topk(score, min(w, mp * P), dim=-1)
        count = torch.full((S,), w, device=dev)
        if case["new"]:
            count = torch.randint(1, w + 1, (S,), generator=g, device=dev)
        none = (got < 0) | (torch.arange(ids.shape[-1], device=dev) >= count[:, None, None])
        ids = torch.where(none, torch.full_like(ids, mp * P), ids).sort(-1)[0]
        kept = torch.full((S, heads, w), -1, dtype=torch.int32, device=dev)
        kept[..., :ids.shape[-1]] = torch.where(ids < mp * P, ids, torch.full_like(ids, -1)).int()
        st["kept"], st["start"] = kept, first.int() if case["new"] else None
        st["lens"] = torch.zeros(S, dtype=torch.int32, device=dev)
    if own:
        from paper_2607_24555_amd import locks as B, tokens as T
        kind = {"bf16": B.LOCKS_BF16, "fp32": B.LOCKS_FP32}[case.get("dtype", "bf16")]
        cfg = B.Config(S, case.get("q_heads", H), H, 8, 2048, mp, nb, kind, kind, page_size=P)
        if case["op"] == "tree":
            ws = T.alloc_tree_workspace(cfg, st["q"].shape[0], dev)
            out = torch.empty(st["q"].shape, dtype=TORCH_OF[case["out"]], device=dev)
            st["call"] = T.prepare_tree_attend(cfg, st["q"], st["k"], st["v"], table, st["sl"], ws,
                                               cu_tokens=st["cu"], mask=st["mask"], out=out)
        elif case["op"] == "mass":
            st["call"] = T.prepare_token_mass(cfg, st["q"], st["lse"], st["k"], table, st["sl"], st["mass"],
                                              cu_tokens=st["cu"], mask=st["mask"], decay=case["decay"])
        elif case["op"] == "pick":
            ws = T.alloc_pick_workspace(cfg, dev)
            st["call"] = T.prepare_pick_tokens(cfg, st["mass"], st["sl"], case["keep"], case["sink"],
                                               case["recent"], ws)
        else:
            st["call"] = T.prepare_keep_tokens(cfg, st["kept"], st["k"], st["v"], table, start=st["start"],
                                               mass=st["mass"], out_lens=st["lens"])
    return st


# ---------------------------------------------------------------- one pass

def _logits(st, most):
    """Logits [S][H][G * most][tokens] in fp32 of the new tokens, padded to `most` a sequence,
    -inf where a token is not seen, and the rows [S][most] of the input that they are."""
    case = st["case"]
    S, H, P = case["seqs"], case["kv_heads"], case["page"]
    G, dev = case["q_heads"] // H, st["sl"].device
    tok = torch.arange(st["pt"].shape[1] * P, device=dev)
    i = torch.arange(most, device=dev)
    cu, sl = st["cu"].long(), st["sl"].long()
    n = cu[1:] - cu[:-1]
    rows = (cu[:-1, None] + i).clamp(max=st["q"].shape[0] - 1)
    at = tok[None] - (sl - n)[:, None]                          # a token's index among the new ones
    if st["mask"] is None:
        seen = at[:, None] <= i[:, None]
    else:
        bits = (st["mask"][:, :, None] >> torch.arange(32, device=dev)) & 1
        bits = bits.reshape(st["mask"].shape[0], -1)[rows]      # [S][most][32 words]
        pick = at.clamp(0, bits.shape[2] - 1)[:, None].expand(S, most, -1)
        seen = (at < 0)[:, None] | ((at < bits.shape[2])[:, None] & (torch.gather(bits, 2, pick) != 0))
    seen = seen & (tok[None] < sl[:, None])[:, None] & (i[None] < n[:, None])[..., None]
    k = _rows_of(st, "k")
    q = st["q"][rows].float().reshape(S, most, H, G, D).permute(0, 2, 3, 1, 4).reshape(S, H, G * most, D)
    z = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D)).view(S, H, G, most, -1)
    z.masked_fill_(~seen[:, None, None], -math.inf)
    return z.view(S, H, G * most, -1), rows


def _rows_of(st, which):
    """The cache's rows in their order, [S][H][tokens][128] in fp32."""
    case = st["case"]
    x = st[which][st["pt"].long().clamp(min=0)]                 # [S][pages][H][P][128]
    return x.transpose(1, 2).reshape(case["seqs"], case["kv_heads"], -1, D).float()


def _live(st, rows):
    n = (st["cu"][1:] - st["cu"][:-1]).long()
    return torch.arange(rows.shape[1], device=rows.device)[None] < n[:, None]


def _plain_tree(st):
    case = st["case"]
    S, H, Hq, most = case["seqs"], case["kv_heads"], case["q_heads"], max(_lens(case)[1])
    G = Hq // H
    z, rows = _logits(st, most)
    m = z.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp_(z.sub_(m))
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, _rows_of(st, "v")) / torch.where(l > 0, l, torch.ones_like(l))
    live = _live(st, rows)
    o = o.reshape(S, Hq, most, D).transpose(1, 2)[live]
    lse = (m + torch.log(l)).reshape(S, Hq, most).transpose(1, 2)[live]
    return {"out": o.to(TORCH_OF[case["out"]]), "lse": lse}


def _plain_mass(st):
    case = st["case"]
    S, H, Hq, most = case["seqs"], case["kv_heads"], case["q_heads"], max(_lens(case)[1])
    z, rows = _logits(st, most)
    lse = st["lse"][rows].transpose(1, 2).reshape(S, H, Hq // H * most, 1)
    none = lse == -math.inf
    got = torch.exp_(z.sub_(torch.where(none, torch.zeros_like(lse), lse))).masked_fill_(none, 0.0).sum(2)
    tok = torch.arange(st["mass"].shape[2], device=lse.device)
    cu, sl = st["cu"].long(), st["sl"].long()
    old = torch.where((tok[None] < (sl - cu[1:] + cu[:-1])[:, None])[:, None], st["mass"] * case["decay"],
                      torch.zeros_like(st["mass"]))
    st["mass"].copy_(torch.where((tok[None] < sl[:, None])[:, None], old + got, st["mass"]))


def _plain_pick(st):
    case = st["case"]
    S, H, W = st["mass"].shape
    tok = torch.arange(W, device=st["sl"].device)
    L = st["sl"].long()[:, None]
    x = torch.where(((tok < case["sink"]) | (tok >= L - case["recent"]))[:, None],
                    torch.full_like(st["mass"], math.inf), st["mass"])
    x = torch.where((tok < L)[:, None], x, torch.full_like(x, -math.inf))
    k = min(case["keep"], W)
    ids = torch.sort(x, dim=-1, descending=True, stable=True)[1][..., :k]
    ids = torch.where(ids < L[:, None], ids, torch.full_like(ids, W)).sort(-1)[0]
    out = torch.full((S, H, case["keep"]), -1, dtype=torch.int32, device=ids.device)
    out[..., :k] = torch.where(ids < W, ids, torch.full_like(ids, -1)).int()
    return {"ids": out}


def _plain_keep(st):
    P, H = st["case"]["page"], st["case"]["kv_heads"]
    kept = st["kept"].long()
    kept = kept.expand(-1, H, -1)
    start = torch.zeros_like(st["sl"]).long() if st["start"] is None else st["start"].long()
    s, h, i = torch.nonzero(kept >= 0, as_tuple=True)
    src, dst = kept[s, h, i], start[s] + i
    frm, to = st["pt"][s, src // P].long(), st["pt"][s, dst // P].long()
    for x in (st["k"], st["v"]):
        x[to, h, dst % P] = x[frm, h, src % P]
    st["mass"][s, h, dst] = st["mass"][s, h, src]
    st["lens"].copy_(start + (kept[:, 0] >= 0).sum(-1))


def run(st):
    op = st["case"]["op"]
    if own:
        st["call"]()
        if op == "tree":
            out, lse = st["call"].outputs
            return {"out": out, "lse": lse}
        if op == "pick":
            return {"ids": st["call"].outputs}
    elif op == "tree":
        return _plain_tree(st)
    elif op == "pick":
        return _plain_pick(st)
    elif op == "mass":
        _plain_mass(st)
    else:
        _plain_keep(st)
    if op == "mass":
        return {"mass": st["mass"]}
    return {"k": st["k"], "v": st["v"], "mass": st["mass"], "lens": st["lens"]}


# ---------------------------------------------------------------- work

def work(case):
    lens, new = _lens(case)
    S, H, P = case["seqs"], case["kv_heads"], case["page"]
    eb = 2 if case.get("dtype", "bf16") == "bf16" else 4
    pages = sum(-(-L // P) for L in lens)
    if case["op"] == "pick":
        return {"bytes": H * (4 * sum(lens) + 4 * case["keep"] * S), "flops": 0}
    if case["op"] == "keep":
        # (what is in its place already is not many rows)
        n = sum(min(case["width"] if not case["new"] else (case["width"] + 1) / 2, L) for L in lens)
        lists = S * case["width"] * 4 * (1 if case["new"] else H)
        return {"bytes": n * H * (4 * D * eb + 8) + lists, "flops": 0}
    Hq, n = case["q_heads"], sum(new)
    pairs = sum(t * (L - t) + sum(b.bit_count() if hasattr(b, "bit_count") else bin(b).count("1") for b in bits)
                for L, t, bits in zip(lens, new, _seen(case)))
    if case["op"] == "tree":
        ob = 2 if case["out"] == "bf16" else 4
        moved = sum(lens) * H * 2 * D * eb + n * Hq * (D * (eb + ob) + 4) + 4 * pages
        return {"bytes": moved, "flops": 4 * D * Hq * pairs}
    moved = sum(lens) * H * (D * eb + 8) + n * Hq * (D * eb + 4) + 4 * pages
    return {"bytes": moved, "flops": 2 * D * Hq * pairs}


# ---------------------------------------------------------------- 64-bit results

def _exact_seq(case, st, s, h):
    """Of one sequence and KV head: keys in order, and for every new token the logits of the
    group's heads over the tokens, -inf where it does not see one; all in 64 bits."""
    lens, new = _lens(case)
    P, G, L, n = case["page"], case["q_heads"] // case["kv_heads"], lens[s], new[s]
    blocks = st["pt"][s, :-(-L // P)].long()
    k = st["k"][blocks, h].reshape(-1, D)[:L].double()
    off = sum(new[:s])
    q = st["q"][off:off + n, h * G:(h + 1) * G].double()
    hidden = torch.zeros(n, L, dtype=torch.bool)
    for i, bits in enumerate(_seen(case)[s]):
        hidden[i, L - n:] = torch.tensor([not bits >> j & 1 for j in range(n)])
    return k, q, hidden.to(k.device), blocks


def exact(case, seed):
    if case["op"] == "pick":                  # whole numbers
        return None
    st = prepare(case, seed)
    lens, new = _lens(case)
    S, H, P, dev = case["seqs"], case["kv_heads"], case["page"], st["sl"].device
    if case["op"] == "tree":
        Hq, n = case["q_heads"], sum(new)
        G = Hq // H
        out = torch.zeros(n, Hq, D, dtype=torch.float64, device=dev)
        lse = torch.zeros(n, Hq, dtype=torch.float64, device=dev)
        for s in range(S):
            for h in range(H):
                k, q, hidden, blocks = _exact_seq(case, st, s, h)
                v = st["v"][blocks, h].reshape(-1, D)[:lens[s]].double()
                off = sum(new[:s])
                for g in range(G):
                    z = torch.mm(q[:, g], k.t().contiguous()) / math.sqrt(D)
                    z = z.masked_fill(hidden, -math.inf)
                    e = torch.logsumexp(z, 1)
                    w = torch.exp(z - torch.where(torch.isinf(e), torch.zeros_like(e), e)[:, None])
                    out[off:off + new[s], h * G + g] = torch.mm(w, v)
                    lse[off:off + new[s], h * G + g] = e
        return {"out": out, "lse": lse}
    if case["op"] == "mass":
        mass, G = st["mass"].double(), case["q_heads"] // H
        for s in range(S):
            L, n, off = lens[s], new[s], sum(new[:s])
            for h in range(H):
                k, q, hidden, _ = _exact_seq(case, st, s, h)
                mass[s, h, :L - n] *= case["decay"]
                mass[s, h, L - n:L] = 0.0
                for g in range(G):
                    z = torch.mm(q[:, g], k.t().contiguous()) / math.sqrt(D)
                    e = st["lse"][off:off + n, h * G + g, None].double()
                    w = torch.exp(z.masked_fill(hidden, -math.inf) - torch.where(torch.isinf(e), torch.zeros_like(e), e))
                    mass[s, h, :L] += torch.where(torch.isinf(e), torch.zeros_like(w), w).sum(0)
        return {"mass": mass}
    k, v, mass = st["k"].double(), st["v"].double(), st["mass"].double()
    kept, pt = st["kept"].tolist(), st["pt"].tolist()
    for s in range(S):
        first = lens[s] - case["new"] if case["new"] else 0
        for h in range(H):
            src = [t for t in kept[s][h if len(kept[s]) > 1 else 0] if t >= 0]
            at = [torch.tensor(x, device=dev) for x in (
                [pt[s][t // P] for t in src], [t % P for t in src],
                [pt[s][(first + i) // P] for i in range(len(src))], [(first + i) % P for i in range(len(src))])]
            for x, y in ((k, st["k"]), (v, st["v"])):
                x[at[2], h, at[3]] = y[at[0], h, at[1]].double()
            mass[s, h, first:first + len(src)] = st["mass"][s, h, torch.tensor(src, device=dev)].double()
    return {"k": k, "v": v, "mass": mass, "lens": None}
