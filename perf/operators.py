"""Speculative decoding over the tiered cache: what its operators are timed on, with a plain form of each.

A drafted tree of n nodes hangs on the committed context.  Node i's parent is a node before it, or -1 for the context's end; a
parent outside -1 .. i - 1 marks a node that is not there (a batch padded to one tree size).  Three kinds of pass:

  attend   attention of the tree's queries (`attend_tree`), one call per layer: a node sees the live context and, of the
           tree's rows, its ancestors and itself.
  step     the cache's part of a whole speculative step: the tree's rows are appended to every layer, every layer is attended, the
           nodes of an accepted path are kept and the others given back, and the kept queries' weights enter the scores
           (`append`, `attend_tree`, `accept_tree`).  What the pass before has kept is taken back first, and the scores are set, so
           that every pass does the same.
  verify   the walk of the tree against the target's probabilities, from given random numbers (`verify_tree`), and the next token.

Contexts are synthetic and reasoning-shaped: standard normal keys, values and queries; one key element carries a per-position
importance z ~ N(0, 1) and the matching query element is sqrt(head_dim).  Rows lie in tiers at random, in the shares of this
repository's benchmark policies: full precision (in HBM, or staged from the host), int8 / int4 codes, evicted.  Shapes are
those of its benchmark configurations, with the layers cut where one layer more adds nothing but time.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SINK, WINDOW = 4, 128                     # protected positions at the context's beginning and end
MIX_7B = dict(f1=100_000, f2=100_000, f3=50_000)      # of a million: staged rows, compressed, evicted; the rest in HBM
MIX_14B = dict(f1=100_000, f2=150_000, f3=30_000)
MIX_PROD = dict(f1=0, f2=200_000, f3=30_000)
ATTEND = dict(kind="attend", layers=1, batch=1, q_heads=8, kv_heads=2, dim=128, dtype="bf16", out="f32", t2="int8_row", context=512,
              nodes=8, span=4, pad=False, roots=False, keep=0, scorer="attention", **MIX_7B)
VERIFY = dict(kind="verify", batch=1, nodes=8, span=4, vocab=32000, dtype="f32", drafted=True)


def listed():
    b7 = dict(q_heads=28, kv_heads=4, **MIX_7B)
    b14 = dict(batch=8, q_heads=40, kv_heads=8, **MIX_14B)
    return [
        # the smallest calls: one sequence of a small binary32 layer, a line of four tokens
        dict(ATTEND, name="attend_tiny_f32", dim=64, dtype="f32", context=257, nodes=4, span=1),
        # one user on the 7B shape, a tree of odd size: few rows a layer, latency and the number of launches count
        dict(ATTEND, name="attend_solo_7b", layers=4, context=1422, nodes=25, **b7),
        # the 14B benchmark shape, 160 columns a kv head, binary32 output
        dict(ATTEND, name="attend_14b_32", context=4133, nodes=32, pad=True, **b14),
        # the same with a large tree and 16-bit output, as a 16-bit model takes it
        dict(ATTEND, name="attend_14b_60_bf16", out="bf16", context=4133, nodes=60, span=12, **b14),
        # a long context in binary16, a small tree beside it: bound by the rows
        dict(ATTEND, name="attend_32b_f16", batch=4, q_heads=40, kv_heads=8, dtype="f16", out="f16", context=8201, nodes=13, **MIX_14B),
        # the production batch's lists in int4, a line of eight drafted tokens (the largest)
        dict(ATTEND, name="attend_prod_int4", batch=32, q_heads=28, kv_heads=4, t2="int4_g32", context=16384, nodes=8, span=1, **MIX_PROD),
        # one user's whole step at full depth
        dict(ATTEND, name="step_solo_7b", kind="step", layers=28, context=1422, nodes=25, keep=5, **b7),
        # a batch's step on the 14B shape, sequences that keep different numbers of nodes
        dict(ATTEND, name="step_14b", kind="step", layers=8, context=4133, nodes=32, keep=6, **b14),
        # one sequence, a line of five tokens drafted by a small model
        dict(VERIFY, name="verify_line", nodes=6, span=1),
        # a batch of large trees of most likely tokens, 16-bit probabilities over a large vocabulary
        dict(VERIFY, name="verify_ranked_tree", batch=32, nodes=60, span=12, vocab=128_000, dtype="bf16", drafted=False),
        # trees whose children were drawn from the draft's distribution: rejected ones leave a residual
        dict(VERIFY, name="verify_drawn_tree", batch=8, nodes=25, span=8, vocab=100_003, dtype="f32"),
    ]


def _columns(c):
    return c["nodes"] * c["q_heads"] // c["kv_heads"]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    if rng.random() < 0.3:
        c = dict(VERIFY, batch=log_int(1, 32), nodes=rng.randint(2, 64), span=rng.choice([1, 4, 12]), vocab=log_int(1000, 128_000),
                 dtype=rng.choice(["f32", "bf16", "f16"]), drafted=rng.random() < 0.5)
        c["batch"] = max(1, min(c["batch"], int(32 * 60 * 128_000 / (c["nodes"] * c["vocab"] * (4 if c["drafted"] else 1)))))
        return c
    heads = rng.choice([(8, 2), (28, 4), (28, 4), (40, 8), (40, 8), (10, 2), (8, 8), (16, 4), (64, 8), (12, 2)])
    c = dict(ATTEND, kind=rng.choice(["attend", "attend", "step"]), q_heads=heads[0], kv_heads=heads[1], dim=rng.choice([64, 128, 128, 128]),
             dtype=rng.choice(["bf16", "bf16", "bf16", "f16", "f32"]), out=rng.choice(["f32", "f32", "bf16"]), t2=rng.choice(["int8_row", "int8_row", "int4_g32"]),
             layers=rng.randint(1, 12), batch=log_int(1, 32), context=log_int(200, 16384), nodes=rng.choice([rng.randint(1, 16), rng.randint(8, 64)]),
             span=rng.choice([1, 4, 12]), pad=rng.random() < 0.3, roots=rng.random() < 0.2)
    c.update(rng.choice([MIX_7B, MIX_14B, MIX_PROD]))
    if c["dtype"] == "f32":
        c.update(out="f32", nodes=min(c["nodes"], 16))
    if c["kind"] == "step":
        c.update(keep=rng.randint(1, 8), scorer=rng.choice(["attention", "attention", "vatp"]), layers=max(2, c["layers"]))
    # no more than the largest listed case: its rows, and the products of them
    rows = c["batch"] * c["kv_heads"] * c["dim"]
    c["context"] = max(200, min(c["context"], int(32 * 4 * 128 * 16384 / rows), int(2.0e10 / (rows * _columns(c)))))
    c["layers"] = max(1, min(c["layers"], int(32 * 4 * 128 * 16384 / (rows * c["context"])), int(2.0e10 / (rows * c["context"] * _columns(c)))))
    return c


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _generator(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1_000_003 + tag * 7919 + 12345) & 0x7FFFFFFFFFFFFFFF)
    return g


def _trees(c, seed):
    """Parents [B, n] and accepted paths [B, keep] (-1 beyond a path's end), on the host."""
    r = np.random.RandomState((int(seed) * 31 + 7) % (1 << 31))
    B, n = c["batch"], c["nodes"]
    parents = np.full((B, n), -1, np.int32)
    for b in range(B):
        for i in range(1, n):
            parents[b, i] = r.randint(max(0, i - c["span"]), i)
        if c.get("roots") and n > 2:
            parents[b, n // 2] = -1
        if c.get("pad") and b % 2 and n > 3:
            parents[b, n - 1 - r.randint(n // 3 + 1):] = -2
    path = np.full((B, max(1, c.get("keep", 0))), -1, np.int32)
    for b in range(B):
        cur, m = 0, r.randint(1, path.shape[1] + 1)
        for j in range(m):
            path[b, j] = cur
            kids = np.nonzero(parents[b] == cur)[0]
            if not len(kids):
                break
            cur = kids[r.randint(len(kids))]
    return parents, path


def _tiers(c, seed):
    """Tier of every context position [B, N], on the host: the policy's shares of the unprotected ones, at random."""
    r = np.random.RandomState((int(seed) * 131 + 77) % (1 << 31))
    t = np.zeros((c["batch"], c["context"]), np.uint8)
    lo, hi = SINK, c["context"] - WINDOW
    if hi > lo:
        m = hi - lo
        n1, n2, n3 = (m * c[f] // 1_000_000 for f in ("f1", "f2", "f3"))
        for b in range(c["batch"]):
            at = lo + r.permutation(m)
            t[b, at[:n3]], t[b, at[n3:n3 + n2]], t[b, at[n3 + n2:n3 + n2 + n1]] = 3, 2, 1
    return t


def _rows(c, seed, layer, n, tag, z):
    g = _generator(seed, 1000 + 64 * layer + tag)
    shape = (c["batch"], n, c["kv_heads"], c["dim"])
    k = torch.randn(shape, generator=g, device="cuda", dtype=DTYPES[c["dtype"]])
    v = torch.randn(shape, generator=g, device="cuda", dtype=DTYPES[c["dtype"]])
    k[..., 0] = z[:, :, None].to(k.dtype)
    return k, v


def _attention_inputs(c, seed):
    """Context rows and tree rows per layer, queries, trees, tiers, scores: everything a step is given."""
    B, N, n = c["batch"], c["context"], c["nodes"]
    z = torch.randn((B, N + n), generator=_generator(seed, 1), device="cuda")
    s = torch.exp(z[:, :N] + 0.25 * torch.randn((B, N), generator=_generator(seed, 4), device="cuda"))
    score = torch.zeros((B, N + n), device="cuda")
    score[:, :N] = s / s.sum(1, keepdim=True)
    q = torch.randn((c["layers"], B, n, c["q_heads"], c["dim"]), generator=_generator(seed, 2), device="cuda", dtype=DTYPES[c["dtype"]])
    q[..., 0] = math.sqrt(c["dim"])
    context = [_rows(c, seed, l, N, 0, z[:, :N]) for l in range(c["layers"])]
    tree = [_rows(c, seed, l, n, 1, z[:, N:]) for l in range(c["layers"])]
    parents, path = _trees(c, seed)
    return context, tree, q, score.cpu().numpy(), torch.from_numpy(parents).cuda(), torch.from_numpy(path).cuda(), _tiers(c, seed)


def _encoded(x, t2):
    """Codes and scales of rows [..., D] as the compressed tier holds them (binary32 arithmetic, true divisions)."""
    x = x.float()
    y = x if t2 == "int8_row" else x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top, a = (127.0 if t2 == "int8_row" else 7.0), y.abs().amax(-1, keepdim=True)
    scale = a / torch.full_like(a, top)
    if t2 != "int8_row":
        scale = scale.half().float()
    code = torch.where(scale > 0, torch.round(y / torch.where(scale > 0, scale, torch.ones_like(scale))).clamp(-top, top), torch.zeros_like(y))
    return code.to(torch.int8), scale


def _probabilities(c, seed):
    B, n, V, dt = c["batch"], c["nodes"], c["vocab"], DTYPES[c["dtype"]]
    parents, _ = _trees(c, seed)
    pa = torch.from_numpy(parents).cuda()
    up = pa.clamp(min=0).long()
    logits = 2.0 * torch.randn((B, n, V), generator=_generator(seed, 1), device="cuda")
    if c["drafted"]:
        # the draft's distribution is the target's with noise, and every child is drawn from its parent's
        q = torch.softmax(logits + 0.6 * torch.randn((B, n, V), generator=_generator(seed, 2), device="cuda"), -1).to(dt)
        cum = torch.cumsum(q.double(), -1)
        at = torch.rand((B, n, n), generator=_generator(seed, 3), device="cuda").double() * cum[..., -1:]
        drawn = torch.searchsorted(cum, at, right=True).clamp(max=V - 1)                       # n draws from every node
        tokens = torch.gather(drawn, 1, up[:, None, :]).squeeze(1)
        del cum, at, drawn
    else:
        # children are likely tokens of their parent, each another one
        q = None
        first = torch.randint(0, V, (B, n), generator=_generator(seed, 3), device="cuda")
        tokens = (torch.gather(first, 1, up) + 13 * torch.arange(n, device="cuda")) % V
        lift = math.log(V) + 0.5 * torch.randn((B, n), generator=_generator(seed, 2), device="cuda")
        b = torch.arange(B, device="cuda")[:, None]
        logits[b, up, tokens] = lift + 1.0
    p = torch.softmax(logits, -1).to(dt)
    u = torch.rand((B, n + 1), generator=_generator(seed, 5), device="cuda")
    return pa, tokens.to(torch.int32), p, q, u[:, :n].contiguous(), u[:, n].contiguous()


def _cache(c, context, tiers):
    import paper_2605_09490_amd as tkv

    N, n = c["context"], c["nodes"]
    most = lambda t: int((tiers == t).sum(1).max()) + 8
    kv = tkv.TieredKV(c["layers"], c["batch"], c["q_heads"], c["kv_heads"], c["dim"], N + n, kv_dtype=c["dtype"], t2_format=c["t2"], out_dtype=c["out"],
                      k_sink=SINK, k_window=WINDOW, prefetch_mode="lazy", scorer=c["scorer"], staging_rows=most(1), t2_rows=most(2),
                      host_rows=int((tiers == 1).sum()) + 8, bounce_bytes=16 << 20)
    for l, (k, v) in enumerate(context):
        kv.append(l, k, v)
    kv.set_tiers(tiers)
    kv.migrate()
    kv.wait_prefetch()
    return kv


def prepare(case, seed):
    c = case
    st = {"case": c}
    if c["kind"] == "verify":
        st["args"] = _probabilities(c, seed)
        if own:
            import paper_2605_09490_amd as tkv
            st["kv"] = tkv.TieredKV(1, c["batch"], 1, 1, 64, 64, staging_rows=1, t2_rows=1, host_rows=1, bounce_bytes=1 << 16)
        return st
    context, tree, q, score, parents, path, tiers = _attention_inputs(c, seed)
    out = torch.zeros(q.shape, dtype=DTYPES[c["out"]], device="cuda")
    st.update(tree=tree, q=q, score=score, parents=parents, path=path, out=out)
    if own:
        kv = _cache(c, context, tiers)
        st.update(kv=kv, kept=0)
        if c["kind"] == "attend":
            for l, (k, v) in enumerate(tree):
                kv.append(l, k, v)
        return st
    t = torch.from_numpy(tiers).cuda()
    n2 = int((tiers == 2).sum(1).max())
    at2 = torch.nonzero(t == 2)[:, 1].reshape(c["batch"], n2)
    b = torch.arange(c["batch"], device="cuda")[:, None]
    st.update(tier=t, at2=at2, rows=[(k, v) for k, v in context], codes=[(_encoded(k[b, at2], c["t2"]), _encoded(v[b, at2], c["t2"])) for k, v in context])
    return st


# ---- the plain forms -----------------------------------------------------------------------------------------------------
def _ancestors(parents):
    """seen [B, n, n]: node j is node i or above it; here [B, n]: i and all above it are there."""
    n = parents.shape[1]
    i = torch.arange(n, device="cuda")
    bad = (parents < -1) | (parents >= i)
    up = (parents[:, :, None] == i) & ~bad[:, :, None]
    seen = (up | torch.eye(n, dtype=torch.bool, device="cuda")).float()
    for _ in range(7):                                    # trees of up to 128 nodes
        seen = (torch.matmul(seen, seen) > 0).float()
    here = torch.matmul(seen, bad.float()[:, :, None])[..., 0] == 0
    return seen > 0, here


def _full(rows, codes, at2, tree):
    """Rows of context and tree in 32 bits, [B, N + n, Hkv, D]."""
    x = torch.cat([rows, tree], 1).float()
    code, scale = codes
    b = torch.arange(x.shape[0], device="cuda")[:, None]
    x[b, at2] = (code.float() * scale).reshape(x[b, at2].shape)
    return x


def _plain_attend(st, l, visible, here):
    c = st["case"]
    B, n, Hq, Hkv, D = c["batch"], c["nodes"], c["q_heads"], c["kv_heads"], c["dim"]
    G = Hq // Hkv
    (k, v), (kc, vc), (tk, tv) = st["rows"][l], st["codes"][l], st["tree"][l]
    k = _full(k, kc, st["at2"], tk).permute(0, 2, 3, 1).contiguous()                      # [B, Hkv, D, N + n]
    v = _full(v, vc, st["at2"], tv).permute(0, 2, 1, 3).contiguous()
    q = st["q"][l].float().reshape(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D).contiguous()
    x = torch.matmul(q, k) * (1.0 / math.sqrt(D))
    x = torch.where(visible.repeat_interleave(G, 1)[:, None], x, torch.full_like(x, -math.inf))
    w = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-1e30))
    w = w / w.sum(-1, keepdim=True).clamp(min=1e-30)
    o = torch.matmul(w, v).reshape(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    st["out"][l] = torch.where(here[:, :, None, None], o, torch.zeros_like(o)).to(st["out"].dtype)
    return w, v


def _plain_step(st):
    c = st["case"]
    B, n, N, Hkv, G = c["batch"], c["nodes"], c["context"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    seen, here = _ancestors(st["parents"])
    visible = torch.cat([(st["tier"] != 3)[:, None].expand(B, n, N), seen], 2) & here[:, :, None]
    path = st["path"]
    taken = torch.where(path >= 0, path, torch.zeros_like(path)).long()                  # [B, keep]
    live = path >= 0
    b = torch.arange(B, device="cuda")[:, None]
    gain = torch.zeros((B, N + n), device="cuda")
    for l in range(c["layers"]):
        w, v = _plain_attend(st, l, visible, here)
        if c["kind"] == "step":
            w = w.reshape(B, Hkv, n, G, N + n).sum(3)                                     # [B, Hkv, n, N + n]
            if c["scorer"] == "vatp":
                norm = torch.cat([st["rows"][l][1], st["tree"][l][1]], 1).float().square().sum(-1).sqrt()
                w = w * norm.permute(0, 2, 1)[:, :, None]
            w = w.sum(1)[b, taken] * live[:, :, None]                                     # the kept queries'
            gain += w.sum(1)
    if c["kind"] == "attend":
        return {"out": st["out"]}
    gain *= 1.0 / (c["layers"] * c["q_heads"])
    kept = int(live.sum(1).max())
    score = torch.zeros((B, N + n), device="cuda")
    score[:, :N] = torch.from_numpy(st["score"]).cuda()[:, :N] + gain[:, :N]
    score[:, N:N + kept] = torch.where(live, gain[b, N + taken], torch.zeros_like(gain[b, N + taken]))[:, :kept]
    tier = torch.zeros((B, N + n), dtype=torch.uint8, device="cuda")
    tier[:, :N] = st["tier"]
    tier[:, N:N + kept] = torch.where(live, 0, 3).to(torch.uint8)[:, :kept]
    return {"out": st["out"], "scores": score.cpu().numpy(), "tiers": tier.cpu().numpy(), "kept": kept}


def _plain_verify(args):
    parents, tokens, p, q, u, u_draw = args
    B, n, V = p.shape
    b = torch.arange(B, device="cuda")
    cur = torch.zeros(B, dtype=torch.long, device="cuda")
    left, total = p[:, 0].double(), torch.ones(B, dtype=torch.float64, device="cuda")
    path = torch.full((B, n), -1, dtype=torch.int32, device="cuda")
    path[:, 0] = 0
    count = torch.ones(B, dtype=torch.long, device="cuda")
    for i in range(1, n):                                  # a node's children come after it: one sweep sees them all in order
        asked = parents[:, i] == cur
        x = tokens[:, i].long()
        t = left[b, x]
        drafted = q[b, cur].double() if q is not None else None
        yes = asked & (u[:, i].double() * total * (drafted[b, x] if drafted is not None else 1.0) < t)
        no = asked & ~yes
        if drafted is not None:
            rest = (left - total[:, None] * drafted).clamp(min=0.0)
            mass = rest.sum(-1)
        else:
            rest = left.clone()
            rest[b, x] = 0.0
            mass = total - t
        no = no & (mass > 0)                               # nothing left (rounded inputs): what was there stays
        left = torch.where(yes[:, None], p[:, i].double(), torch.where(no[:, None], rest, left))
        total = torch.where(yes, torch.ones_like(total), torch.where(no, mass, total))
        path[b, count.clamp(max=n - 1)] = torch.where(yes, torch.full_like(path[:, 0], i), path[b, count.clamp(max=n - 1)])
        count += yes
        cur = torch.where(yes, torch.full_like(cur, i), cur)
    cum = torch.cumsum(left, -1)
    token = torch.searchsorted(cum, (u_draw.double() * cum[:, -1])[:, None], right=True)[:, 0].clamp(max=V - 1)
    return {"path": path, "n_path": count.to(torch.int32), "next": token.to(torch.int32)}


def run(st):
    c = st["case"]
    if c["kind"] == "verify":
        if not own:
            return _plain_verify(st["args"])
        parents, tokens, p, q, u, u_draw = st["args"]
        path, n_path, token = st["kv"].verify_tree(parents, tokens, p, u, u_draw, q)
        return {"path": path, "n_path": n_path, "next": token}
    if not own:
        return _plain_step(st)
    kv = st["kv"]
    if c["kind"] == "attend":
        for l in range(c["layers"]):
            kv.attend_tree(l, st["q"][l], st["parents"], st["out"][l])
        return {"out": st["out"]}
    if st["kept"]:
        kv.accept_tree(st["kept"])
    kv.set_scores(st["score"])
    for l, (k, v) in enumerate(st["tree"]):
        kv.append(l, k, v)
        kv.attend_tree(l, st["q"][l], st["parents"], st["out"][l])
    st["kept"] = kv.accept_tree(c["nodes"], st["path"], st["q"])
    return {"out": st["out"], "scores": kv.get_scores(), "tiers": kv.get_tiers(), "kept": st["kept"]}


def work(case):
    """One pass: every row that is attended read once a layer, queries read, outputs written; a step stores the tree's rows and
    updates a score per position.  A walk: the gathered values, and one residual per sequence."""
    c = case
    if c["kind"] == "verify":
        es = 4 if c["dtype"] == "f32" else 2
        rows = c["batch"] * c["vocab"]
        return {"bytes": float(rows * es * (2 if c["drafted"] else 1)), "flops": 4.0 * rows}
    es, oes = (4 if c["dtype"] == "f32" else 2), (4 if c["out"] == "f32" else 2)
    D, n = c["dim"], c["nodes"]
    t2 = 2 * (D + 4) if c["t2"] == "int8_row" else 2 * (D // 2 + D // 16)
    u = max(0, c["context"] - SINK - WINDOW)
    n2, n3 = u * c["f2"] // 1_000_000, u * c["f3"] // 1_000_000
    full = c["context"] + n - n2 - n3
    heads = c["batch"] * n * c["q_heads"] * D
    total = c["layers"] * (c["batch"] * c["kv_heads"] * (full * 2 * D * es + n2 * t2) + heads * (es + oes))
    flops = c["layers"] * 4.0 * heads * (full + n2)
    if c["kind"] == "step":
        total += 2.0 * c["layers"] * c["batch"] * n * c["kv_heads"] * 2 * D * es + 8.0 * c["batch"] * (full + n2)
        flops += c["layers"] * 2.0 * heads / n * c["keep"] * (full + n2)
    return {"bytes": float(total), "flops": float(flops)}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------------
def _exact_verify(case, seed):
    parents, tokens, p, q, u, u_draw = _probabilities(case, seed)
    B, n, V = p.shape
    pa, tok, u, u_draw = parents.cpu().numpy(), tokens.cpu().numpy(), u.cpu().numpy(), u_draw.cpu().numpy()
    path, count, nxt = np.full((B, n), -1, np.int32), np.zeros(B, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        cur, line, mass = 0, [0], 1.0
        t = p[b, 0].double().cpu().numpy()
        kids = [i for i in range(1, n) if pa[b, i] == 0]
        while kids:
            i = kids.pop(0)
            x = int(tok[b, i])
            qx = float(q[b, cur, x]) if q is not None else 1.0
            if float(u[b, i]) * mass * qx < t[x]:
                cur, mass = i, 1.0
                line.append(i)
                t = p[b, i].double().cpu().numpy()
                kids = [j for j in range(i + 1, n) if pa[b, j] == i]
                continue
            if q is not None:
                rest = np.maximum(t - mass * q[b, cur].double().cpu().numpy(), 0.0)
                left = float(rest.sum())
            else:
                rest = t.copy()
                rest[x] = 0.0
                left = mass - t[x]
            if left > 0:
                t, mass = rest, left
        run = np.cumsum(t)
        path[b, :len(line)], count[b] = line, len(line)
        nxt[b] = min(int(np.searchsorted(run, float(u_draw[b]) * run[-1], side="right")), V - 1)
    return {"path": torch.from_numpy(path), "n_path": torch.from_numpy(count), "next": torch.from_numpy(nxt)}


def exact(case, seed):
    c = case
    if c["kind"] == "verify":
        return _exact_verify(c, seed)
    if c["layers"] * c["batch"] * c["kv_heads"] * c["context"] * _columns(c) * c["dim"] > 3.0e11:
        return None
    context, tree, q, score0, parents, path, tiers = _attention_inputs(c, seed)
    B, N, n, Hkv, G, D = c["batch"], c["context"], c["nodes"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    pa, path = parents.cpu().numpy(), path.cpu().numpy()
    out = torch.zeros((c["layers"], B, n, c["q_heads"], D), dtype=torch.float64, device="cuda")
    score = torch.zeros((B, N + n), dtype=torch.float64)
    kept = int((path >= 0).sum(1).max())
    for b in range(B):
        sees = torch.zeros((n, N + n), dtype=torch.bool)
        for i in range(n):
            j, line = i, []
            while -1 <= pa[b, j] < j:
                line.append(j)
                if pa[b, j] == -1:
                    break
                j = int(pa[b, j])
            else:
                line = []                                 # the chain ends at a node that is not there
            if line:
                sees[i, :N] = torch.from_numpy(tiers[b] != 3)
                sees[i, [N + j for j in line]] = True
        sees = sees.cuda()
        mine = [int(i) for i in path[b] if i >= 0]
        gain = torch.zeros(N + n, dtype=torch.float64, device="cuda")
        two = torch.from_numpy(tiers[b] == 2).cuda()
        for l in range(c["layers"]):
            kb, vb = [torch.cat([x[b], y[b]]).double() for x, y in zip(context[l], tree[l])]     # [N + n, Hkv, D]
            norm = vb.norm(dim=-1)
            for full, stored in ((kb, context[l][0][b]), (vb, context[l][1][b])):
                code, scale = _encoded(stored[two], c["t2"])
                full[:N][two] = (code.double() * scale.double()).reshape(-1, Hkv, D)
            for h in range(Hkv):
                qh = q[l, b, :, h * G:(h + 1) * G].double().reshape(n * G, D).contiguous()
                x = (qh @ kb[:, h].t().contiguous()) / math.sqrt(D)
                x[~sees.repeat_interleave(G, 0)] = -math.inf
                w = torch.nan_to_num(torch.softmax(x, -1))
                out[l, b, :, h * G:(h + 1) * G] = (w @ vb[:, h].contiguous()).reshape(n, G, D)
                if c["kind"] == "step":
                    w = w.reshape(n, G, N + n)[mine].sum((0, 1))
                    gain += w * norm[:, h] if c["scorer"] == "vatp" else w
        gain = gain.cpu() / (c["layers"] * c["q_heads"])
        score[b, :N] = torch.from_numpy(score0[b, :N]).double() + gain[:N]
        score[b, N:N + len(mine)] = gain[N:][mine]
    if c["kind"] == "attend":
        return {"out": out}
    return {"out": out, "scores": score.numpy(), "tiers": None, "kept": kept}
