"""Performance cases of the rollout side's operators: the append of new tokens to a paged key/value cache
(per-head norm and position rotation on the way), the attention of those tokens over the cache, and the
verification of drafted tokens against the target's probabilities.

`run` computes them in their plain form with elementary torch operations, or through the package's entry points
where `own` is true.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"


def _append(name, **kw):
    base = dict(name=name, kind="append", dtype="bf16", seqs=8, ctx_min=0, ctx_max=4096, new_min=1, new_max=1, heads=32,
                kv_heads=8, dim=128, rot=128, style="half", norm=True, page=64, depth=False)
    base.update(kw)
    return base


def _attend(name, **kw):
    base = dict(name=name, kind="attend", dtype="bf16", seqs=8, ctx_min=1024, ctx_max=8192, new_min=1, new_max=1, heads=32,
                kv_heads=8, dim=128, page=64, node=0)
    base.update(kw)
    return base


def _verify(name, **kw):
    base = dict(name=name, kind="verify", dtype="f32", seqs=1, drafts_min=4, drafts_max=4, V=151936, dist=True,
                temperature=1.0)
    base.update(kw)
    return base


def listed():
    return [
        # One generated token for each of eight rollouts: nothing but latency.
        _append("append_decode"),
        # The fp32 debugging type, sizes that fill nothing: interleaved pairs, half of each head rotated, no norm,
        # one token to a chunk of 37, pages of 16.
        _append("append_ragged_fp32", dtype="f32", seqs=13, ctx_max=1000, new_max=37, heads=10, kv_heads=2, dim=80, rot=40,
                style="pairs", norm=False, page=16),
        # The forward pass over packed trees, 32K positions in one call: positions are depths, not slots.
        _append("append_trees", seqs=8, ctx_max=0, new_min=2048, new_max=6144, depth=True),
        # One rollout with a long history generating a token: few rows, the keys are all the work.
        _attend("attend_decode_one", seqs=1, ctx_min=32767, ctx_max=32767),
        # A whole batch of rollouts generating one token each, histories of all lengths.
        _attend("attend_decode", seqs=128, ctx_min=500, ctx_max=8000),
        # Five drafted tokens per rollout checked at once, larger model (five query heads to a key head).
        _attend("attend_drafts", seqs=32, ctx_min=100, ctx_max=16000, new_min=1, new_max=6, heads=40),
        # Tool output of some 2,000 tokens read after a history of up to 14K.
        _attend("attend_chunk", seqs=4, ctx_min=2000, ctx_max=14000, new_min=1990, new_max=2048),
        # The last chunk of packed prefix trees: branches do not see each other; heads of 64.
        _attend("attend_trees", seqs=6, ctx_min=1500, ctx_max=7001, new_min=700, new_max=1333, heads=16, kv_heads=16, dim=64,
                page=16, node=150),
        # The fp32 debugging type over a small ragged batch, head size off the tiles.
        _attend("attend_ragged_fp32", dtype="f32", seqs=7, ctx_min=0, ctx_max=900, new_min=0, new_max=130, heads=10, kv_heads=2,
                dim=80, page=16),
        # One rollout, four drafts of a draft model over the whole vocabulary: latency.
        _verify("verify_one"),
        # Drafts without probabilities (text of an earlier rollout), none to seven per rollout, a vocabulary off every
        # power of two, another temperature.
        _verify("verify_reuse", seqs=24, drafts_min=0, drafts_max=7, V=50021, dist=False, temperature=0.8),
        # The batch: 128 rollouts with four drafts each, bf16 logits.
        _verify("verify_batch", dtype="bf16", seqs=128),
    ]


def _log(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "verify", "verify"])
    fp32 = rng.random() < 0.25
    if kind == "verify":
        V = int(_log(rng, 500, 152000))
        lo = rng.randint(0, 3)
        hi = lo + rng.randint(0, 5)
        most = min(128, max(1, int(1.5e8 / (V * (2 * hi + 1)))))
        c = _verify("", dtype="f32" if fp32 else "bf16", seqs=int(_log(rng, 1, most + 0.99)), drafts_min=lo, drafts_max=hi, V=V,
                    dist=rng.random() < 0.6, temperature=rng.choice([1.0, 1.0, 0.7, 1.3]))
        del c["name"]
        return c
    dim = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
    kvh = rng.choice([1, 2, 4, 8])
    heads = kvh * rng.choice([1, 2, 4, 5, 7, 8])
    page = rng.choice([8, 16, 32, 64, 256])
    seqs = int(_log(rng, 1, 129))
    new_max = int(_log(rng, 1, 2049)) if rng.random() < 0.6 else rng.randint(1, 8)
    new_max = max(1, min(new_max, 30000 // seqs))
    new_min = rng.choice([0, 1, (new_max + 1) // 2, new_max])
    ctx_max = int(_log(rng, 16, 16000))
    ctx_min = rng.choice([0, ctx_max // 8, ctx_max // 2])
    if kind == "append":
        tokens = max(1, min(seqs * new_max, int(5e7 / ((heads + 2 * kvh) * dim))))
        new_max = max(1, tokens // seqs)
        c = _append("", dtype="f32" if fp32 else "bf16", seqs=seqs, ctx_min=0, ctx_max=min(ctx_max, 4000), new_min=min(new_min, new_max),
                    new_max=new_max, heads=heads, kv_heads=kvh, dim=dim, rot=rng.choice([dim, dim, dim // 2 // 16 * 16]),
                    style=rng.choice(["half", "half", "pairs"]), norm=rng.random() < 0.6, page=page, depth=rng.random() < 0.3)
    else:
        # the plain form holds keys, values and all scores in 32 bits
        while (seqs * (ctx_max + new_max) * kvh * dim > 8e8 or seqs * heads * new_max * (ctx_max + new_max) > 1.5e9
               or seqs * heads * dim * new_max * (ctx_max + new_max) > 6e10):
            if ctx_max > 4 * new_max:
                ctx_max = ctx_max * 3 // 4
            elif seqs > 1:
                seqs = (seqs + 1) // 2
            else:
                new_max = (new_max + 1) // 2
        c = _attend("", dtype="f32" if fp32 else "bf16", seqs=seqs, ctx_min=min(ctx_min, ctx_max), ctx_max=ctx_max,
                    new_min=min(new_min, new_max), new_max=new_max, heads=heads, kv_heads=kvh, dim=dim, page=page,
                    node=rng.choice([0, 0, 20, 150]))
    del c["name"]
    return c


# ---- inputs ----

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _spread(lo, hi, n):
    """n sizes evenly over [lo, hi] (their total does not depend on the seed); one alone: the largest."""
    return np.array([hi]) if n == 1 else np.linspace(lo, hi, n).round().astype(np.int64)


def _sizes(case, rng=None):
    """New tokens and cached tokens before them, of each sequence."""
    new = _spread(case["new_min"], case["new_max"], case["seqs"])
    ctx = _spread(case["ctx_min"], case["ctx_max"], case["seqs"])
    at = np.random.default_rng(7).permutation(case["seqs"])  # which chunk goes with which history
    if rng is None:
        return new, ctx[at]
    order = rng.permutation(case["seqs"])
    return new[order], ctx[at][order]


def _tree(length, node, rng):
    """Where the subtree of every position ends, in a depth-first packed tree of nodes of `node` tokens on average."""
    end = np.full(length, length, np.int64)
    path, at = [], 0
    while at < length:
        keep = len(path) if rng.random() < 0.6 else int(rng.integers(min(1, len(path)), len(path) + 1))
        for start, stop in path[keep:]:
            end[start:stop] = at
        n = min(length - at, int(rng.geometric(1.0 / node)) if path else max(1, length // 6))
        path = path[:keep] + [(at, at + n)]
        at += n
    return end


def _randn(shape, std, dtype, gen):
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat = out.view(-1)
    for r in range(0, flat.numel(), 1 << 27):
        part = flat[r:r + (1 << 27)]
        part.copy_(torch.randn(part.shape, generator=gen, device=DEV) * std)
    return out


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a), device=DEV).to(dtype)


def _cache(case, rng, gen):
    """The paged cache after the chunk's append: pages of the sequences in no order, a few of them unused."""
    new, ctx = _sizes(case, rng)
    B, ps = case["seqs"], case["page"]
    used = -(-(new + ctx) // ps)
    cols = max(1, int(used.max()))
    pool = int(used.sum()) + 5
    table = rng.integers(0, pool, (B, cols))  # entries behind a sequence's last page are never read
    pages = rng.permutation(pool)[:used.sum()]
    table[np.arange(cols)[None, :] < used[:, None]] = pages
    shape = (pool, case["kv_heads"], ps, case["dim"])
    return new, ctx, dict(
        case=case, k_pages=_randn(shape, 1.0, _dtype(case), gen), v_pages=_randn(shape, 1.0, _dtype(case), gen), page_table=_dev(table),
        kv_len=_dev(new + ctx), cu_new=_dev(np.concatenate([[0], np.cumsum(new)])), new_max=int(new.max()))


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    if case["kind"] == "verify":
        return _prepare_verify(case, rng, gen)
    new, ctx, s = _cache(case, rng, gen)
    T, H, K, D = int(new.sum()), case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "append":
        qkv = _randn((T, H + 2 * K, D), 1.0, _dtype(case), gen)  # the output of one fused projection
        s.update(q=qkv[:, :H], k=qkv[:, H:H + K], v=qkv[:, H + K:], q_norm=None, k_norm=None, positions=None,
                 freq=1e6 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=DEV) / max(1, case["rot"])))
        if case["norm"]:
            s.update(q_norm=1 + _randn((D,), 0.2, _dtype(case), gen), k_norm=1 + _randn((D,), 0.2, _dtype(case), gen))
        if case["depth"]:
            s["positions"] = _dev(np.concatenate([rng.permutation(c + n)[:n] for n, c in zip(new, ctx)]))
        return s
    # scores of a standard deviation of 1.5: some keys stand out, none takes all
    s.update(q=_randn((T, H, D), 1.5, _dtype(case), gen), scale=1.0 / math.sqrt(D), slot_end=None)
    if case["node"]:
        tree = np.random.default_rng(11)
        ends = np.zeros((case["seqs"], int((new + ctx).max())), np.int64)
        order = np.lexsort((ctx, new))
        for b in order:
            ends[b, :new[b] + ctx[b]] = _tree(int(new[b] + ctx[b]), case["node"], tree)
        s["slot_end"] = _dev(ends)
    return s


def _prepare_verify(case, rng, gen):
    """Logits of a policy that mostly knows its next token; the draft model's are near them.  Drafts are the
    likely token more often than not."""
    V, B = case["V"], case["seqs"]
    n = _spread(case["drafts_min"], case["drafts_max"], B)[rng.permutation(B)]
    cu = np.concatenate([[0], np.cumsum(n)])
    nd, rows = int(cu[-1]), int(cu[-1]) + B
    z = _randn((rows, V), 1.3, torch.float32, gen)
    likely = torch.randint(0, V, (rows,), generator=gen, device=DEV)
    z[torch.arange(rows, device=DEV), likely] += 6.0 + 9.0 * torch.rand(rows, generator=gen, device=DEV)
    at = _dev(np.concatenate([cu[b] + b + np.arange(n[b]) for b in range(B)]) if nd else np.zeros(0), torch.int64)
    other = torch.randint(0, V, (nd,), generator=gen, device=DEV)
    draft = torch.where(torch.rand(nd, generator=gen, device=DEV) < 0.8, likely[at], other)
    draft_logits = None
    if case["dist"]:
        draft_logits = z[at] + 0.7 * torch.randn(nd, V, generator=gen, device=DEV)
        draft_logits = draft_logits.to(_dtype(case))
    return dict(case=case, logits=z.to(_dtype(case)), draft_logits=draft_logits, draft=draft.to(torch.int32), cu=_dev(cu),
                u_accept=torch.rand(nd, generator=gen, device=DEV), u_sample=torch.rand(B, generator=gen, device=DEV),
                n_max=int(n.max()))


# ---- one pass ----

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "verify": _own_verify}[kind](s)
    return {"append": _plain_append, "attend": _plain_attend, "verify": _plain_verify}[kind](s)


def _own_append(s):
    import paper_2608_16798_amd as rlk

    q, s["ws"] = rlk.kv_append(s["k_pages"], s["v_pages"], s["page_table"], s["kv_len"], s["cu_new"], s["q"], s["k"], s["v"],
                               freq=s["freq"], positions=s["positions"], q_norm=s["q_norm"], k_norm=s["k_norm"], norm_eps=1e-6,
                               rot_style=s["case"]["style"], ws=s.get("ws"))
    return dict(q=q, k_pages=s["k_pages"], v_pages=s["v_pages"])


def _own_attend(s):
    import paper_2608_16798_amd as rlk

    if "lse" not in s:
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEV)
    out, lse, s["ws"] = rlk.kv_attention(s["q"], s["k_pages"], s["v_pages"], s["page_table"], s["kv_len"], s["cu_new"],
                                         scale=s["scale"], slot_end=s["slot_end"], max_new=s["new_max"], lse=s["lse"],
                                         ws=s.get("ws"))
    return dict(out=out, lse=lse)


def _own_verify(s):
    import paper_2608_16798_amd as rlk

    tokens, accepted, logp, s["ws"] = rlk.draft_verify(s["logits"], s["draft"], s["cu"], s["u_accept"], s["u_sample"],
                                                       draft_logits=s["draft_logits"], temperature=s["case"]["temperature"],
                                                       ws=s.get("ws"))
    return dict(tokens=tokens, accepted=accepted, logp=logp)


def _places(s, T):
    """Sequence and cache slot of each new token."""
    t = torch.arange(T, device=DEV)
    cu = s["cu_new"].long()
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    return seq, s["kv_len"].long()[seq] - cu[seq + 1] + t


def _rotated(x, w, cos, sin, style, rot):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
    if rot == 0:
        return x
    head, rest = x[..., :rot], x[..., rot:]
    if style == "half":
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        head = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([head, rest], -1)


def _plain_append(s):
    case, ps = s["case"], s["case"]["page"]
    seq, slot = _places(s, s["q"].shape[0])
    pos = slot if s["positions"] is None else s["positions"]
    angle = pos.double()[:, None] * s["freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q = _rotated(s["q"], s["q_norm"], cos, sin, case["style"], case["rot"]).to(s["q"].dtype)
    k = _rotated(s["k"], s["k_norm"], cos, sin, case["style"], case["rot"]).to(s["k"].dtype)
    page = s["page_table"].long()[seq, slot // ps]
    s["k_pages"][page, :, slot % ps] = k
    s["v_pages"][page, :, slot % ps] = s["v"]
    return dict(q=q, k_pages=s["k_pages"], v_pages=s["v_pages"])


def _plain_attend(s):
    case, T = s["case"], s["q"].shape[0]
    B, H, K, D, n = case["seqs"], case["heads"], case["kv_heads"], case["dim"], s["new_max"]
    table = s["page_table"].long()
    k = s["k_pages"][table].permute(0, 2, 1, 3, 4).reshape(B, K, -1, D).float()
    v = s["v_pages"][table].permute(0, 2, 1, 3, 4).reshape(B, K, -1, D).float()
    seq, slot = _places(s, T)
    row = torch.arange(T, device=DEV) - s["cu_new"].long()[seq]
    q = torch.zeros(B, n, H, D, device=DEV)
    q[seq, row] = s["q"].float() * s["scale"]
    q = q.view(B, n, K, H // K, D).permute(0, 2, 3, 1, 4).reshape(B, K, -1, D)
    x = (q @ k.transpose(2, 3)).view(B, H, n, -1)
    at = (s["kv_len"] - (s["cu_new"][1:] - s["cu_new"][:-1])).long()[:, None] + torch.arange(n, device=DEV)  # slot of each row
    keys = torch.arange(x.shape[3], device=DEV)
    seen = keys[None, None, :] <= at[:, :, None]
    if s["slot_end"] is not None:
        end = torch.zeros(B, x.shape[3], dtype=torch.int64, device=DEV)
        end[:, :s["slot_end"].shape[1]] = s["slot_end"]
        seen &= at[:, :, None] < end[:, None, :]
    x.masked_fill_(~seen[:, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp_min(-1e38)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x.view(B, K, -1, x.shape[3]) @ v).view(B, H, n, D) / total.clamp_min(1e-38)
    lse = (total.log() + top)[..., 0]
    return dict(out=o.permute(0, 2, 1, 3)[seq, row].to(s["q"].dtype), lse=lse.permute(0, 2, 1)[seq, row])


def _softmax64(z, tau):
    x = z.double() / tau
    x = x - x.amax(-1, keepdim=True)
    e = x.exp()
    return e / e.sum(-1, keepdim=True), x - e.sum(-1, keepdim=True).log()


def _plain_verify(s):
    case = s["case"]
    B, nm = case["seqs"], s["n_max"]
    cu, draft = s["cu"].long(), s["draft"].long()
    n, nd, rows = cu[1:] - cu[:-1], draft.shape[0], s["logits"].shape[0]
    p, logp = _softmax64(s["logits"], case["temperature"])
    t = torch.arange(nd, device=DEV)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    ok = torch.zeros(B, nm + 1, dtype=torch.bool, device=DEV)
    q = None
    if nd:
        py = p[t + seq, draft]
        if case["dist"]:
            q, _ = _softmax64(s["draft_logits"], case["temperature"])
            ok[seq, t - cu[seq]] = s["u_accept"].double() * q[t, draft] < py
        else:
            ok[seq, t - cu[seq]] = s["u_accept"].double() < py
    acc = ok.long().cumprod(1).sum(1)
    b = torch.arange(B, device=DEV)
    last = cu[:-1] + b + acc  # the row that the last token is drawn from
    mass = p[last]
    if nd:
        cut, i = acc < n, (cu[:-1] + acc).clamp_max(nd - 1)
        if case["dist"]:
            mass = torch.where(cut[:, None], (mass - q[i]).clamp_min(0.0), mass)
        else:
            mass[b, draft[i]] = torch.where(cut, 0.0, mass[b, draft[i]])
    cum = mass.cumsum(1)
    drawn = (cum <= s["u_sample"].double()[:, None] * cum[:, -1:]).sum(1)
    r = torch.arange(rows, device=DEV)
    of = torch.searchsorted((cu[1:] + b + 1).contiguous(), r, right=True)
    i = r - cu[of] - of
    proposed = draft[(r - of).clamp_max(max(0, nd - 1))] if nd else torch.zeros_like(r)
    token = torch.where(i < acc[of], proposed, drawn[of])
    emitted = i <= acc[of]
    return dict(tokens=torch.where(emitted, token, -1).to(torch.int32), accepted=acc.to(torch.int32),
                logp=torch.where(emitted, logp[r, token], 0.0).float())


# ---- what a pass cannot do without ----

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "verify":
        n = int(_spread(case["drafts_min"], case["drafts_max"], case["seqs"]).sum())
        rows = n + case["seqs"] + (n if case["dist"] else 0)
        return {"bytes": rows * case["V"] * e, "flops": rows * case["V"] * 4}
    new, ctx = _sizes(case)
    H, K, D, T = case["heads"], case["kv_heads"], case["dim"], int(new.sum())
    if case["kind"] == "append":
        return {"bytes": 2 * T * (H + 2 * K) * D * e, "flops": T * (H + K) * D * 8}
    pairs = int((new * ctx + new * (new + 1) // 2).sum())
    if case["node"]:
        tree, pairs = np.random.default_rng(11), 0
        for b in np.lexsort((ctx, new)):
            end = _tree(int(new[b] + ctx[b]), case["node"], tree)
            slots = np.arange(len(end))
            pairs += int(np.maximum(0, end - np.maximum(slots, ctx[b])).sum())
    return {"bytes": (2 * T * H * D + 2 * int((new + ctx)[new > 0].sum()) * K * D) * e + T * H * 4, "flops": 4 * pairs * H * D}


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "verify": _exact_verify}[case["kind"]](s)


def _exact_append(s):
    case, ps, rot = s["case"], s["case"]["page"], s["case"]["rot"]
    cu, lens, table = s["cu_new"].tolist(), s["kv_len"].tolist(), s["page_table"].long()
    q_all = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    pools = [s["k_pages"].double(), s["v_pages"].double()]

    def turned(x, w, pos):
        x = x.double()
        if w is not None:
            x = w.double() * x / torch.sqrt(1e-6 + torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / x.shape[-1])
        h = rot // 2
        re, im = (x[..., :h], x[..., h:rot]) if case["style"] == "half" else (x[..., :rot:2], x[..., 1:rot:2])
        y = torch.complex(re, im) * torch.polar(torch.ones_like(pos)[:, None], pos[:, None] * s["freq"])[:, None]
        y = torch.cat([y.real, y.imag], -1) if case["style"] == "half" else torch.view_as_real(y).reshape(*x.shape[:-1], rot)
        return torch.cat([y, x[..., rot:]], -1)

    for b, n in enumerate(np.diff(cu).tolist()):
        rows = slice(cu[b], cu[b] + n)
        slots = torch.arange(lens[b] - n, lens[b], device=DEV)
        pos = (slots if s["positions"] is None else s["positions"][rows]).double()
        q_all[rows] = turned(s["q"][rows], s["q_norm"], pos)
        where = (table[b, slots // ps], slice(None), slots % ps)
        pools[0][where] = turned(s["k"][rows], s["k_norm"], pos)
        pools[1][where] = s["v"][rows].double()
    return dict(q=q_all, k_pages=pools[0], v_pages=pools[1])


def _exact_attend(s):
    case, ps = s["case"], s["case"]["page"]
    H, K = case["heads"], case["kv_heads"]
    cu, lens = s["cu_new"].tolist(), s["kv_len"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    for b, n in enumerate(np.diff(cu).tolist()):
        if n == 0:
            continue
        L = lens[b]
        slots = torch.arange(L, device=DEV)
        pages = s["page_table"][b, :-(-L // ps)].long()
        hidden = slots[None, :] > slots[L - n:, None]
        if s["slot_end"] is not None:
            hidden = hidden | (s["slot_end"][b, :L][None, :] <= slots[L - n:, None])
        for h in range(H):
            k = s["k_pages"][pages, h // (H // K)].reshape(-1, case["dim"])[:L].double()
            v = s["v_pages"][pages, h // (H // K)].reshape(-1, case["dim"])[:L].double()
            x = s["q"][cu[b]:cu[b + 1], h].double() @ k.T * s["scale"]
            x = torch.where(hidden, -math.inf, x)
            z = torch.logsumexp(x, 1)
            lse[cu[b]:cu[b + 1], h] = z
            out[cu[b]:cu[b + 1], h] = torch.exp(x - z[:, None]) @ v
    return dict(out=out, lse=lse)


def _exact_verify(s):
    case, tau = s["case"], s["case"]["temperature"]
    cu, draft = s["cu"].tolist(), s["draft"].tolist()
    ua, us = s["u_accept"].double().tolist(), s["u_sample"].double().tolist()
    rows = s["logits"].shape[0]
    tokens, accepted, logp = np.full(rows, -1, np.int32), np.zeros(case["seqs"], np.int32), np.zeros(rows)
    for b in range(case["seqs"]):
        n, r0 = cu[b + 1] - cu[b], cu[b] + b
        a = 0
        while True:
            lp = s["logits"][r0 + a].double() / tau
            lp = lp - torch.logsumexp(lp, 0)
            if a == n:
                mass = lp.exp()
                break
            y = draft[cu[b] + a]
            if s["draft_logits"] is None:
                lq = torch.full_like(lp, -math.inf)
                lq[y] = 0.0
            else:
                lq = s["draft_logits"][cu[b] + a].double() / tau
                lq = lq - torch.logsumexp(lq, 0)
            if ua[cu[b] + a] * math.exp(lq[y]) < math.exp(lp[y]):
                tokens[r0 + a], logp[r0 + a] = y, float(lp[y])
                a += 1
                continue
            mass = (lp.exp() - lq.exp()).clamp_min(0.0)
            break
        cum = torch.cumsum(mass, 0)
        y = int(torch.searchsorted(cum, us[b] * cum[-1], right=True))
        tokens[r0 + a], logp[r0 + a], accepted[b] = y, float(lp[y]), a
    return dict(tokens=torch.from_numpy(tokens), accepted=torch.from_numpy(accepted), logp=torch.from_numpy(logp))
