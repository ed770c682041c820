"""The cases whose speed the operators of drafted trees are measured by.

A round of speculative decoding in which a drafter proposes a tree: the tree's keys and values
go into the 8-bit cache, rotated by their positions on the way, as are its queries
(``api.cache_append_rotary``); every node attends over the context and its own ancestors
(``api.tree_attend``); the tree is verified (``api.tree_verify``), and the rows of the accepted
path are moved to where the next round expects them (``api.cache_keep``).  ``run`` makes those
calls where ``own`` is true and computes the same in elementary torch operations elsewhere;
``exact`` restates the definitions in 64 bits.

Node 0 of a tree is the last emitted token, parents come before their children.  Cache layout:
codes are float8_e4m3fn, keys [pages, heads, block, dim], values [pages, heads, dim, block], one
float32 scale per page and head for each.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ------------------------------------------------------------------------------ cases
def _append(name, B, W, H, G, D, block, max_len, dtype="bf16", ragged=False, tree=False, rot=0, pairs="halves"):
    return dict(name=name, kind="append", B=B, W=W, H=H, G=G, D=D, block=block, max_len=max_len, dtype=dtype,
                ragged=ragged, tree=tree, rot=rot or D, pairs=pairs)


def _attend(name, B, W, H, G, D, block, max_len, dtype="bf16", ragged=False, fan=4):
    return dict(name=name, kind="attend", B=B, W=W, H=H, G=G, D=D, block=block, max_len=max_len, dtype=dtype,
                ragged=ragged, fan=fan)


def _verify(name, B, W, V, dtype, fan=4, chosen=False, ragged=False, temperature=1.0):
    return dict(name=name, kind="verify", B=B, W=W, V=V, dtype=dtype, fan=fan, chosen=chosen, ragged=ragged,
                temperature=temperature)


def _keep(name, B, W, H, D, block, max_len, deep):
    return dict(name=name, kind="keep", B=B, W=W, H=H, D=D, block=block, max_len=max_len, deep=deep)


def listed():
    return [
        # single tokens of a serving batch, far positions: latency
        _append("append_tokens", 64, 1, 8, 4, 128, 64, 16000, ragged=True),
        # the trees of a serving batch: positions go by depth
        _append("append_trees", 32, 32, 8, 4, 128, 64, 16000, ragged=True, tree=True),
        # prompts of several users, neighbouring pairs, half of each head rotated: the largest read and write
        _append("append_prompts", 4, 8000, 8, 4, 128, 64, 500, rot=64, pairs="neighbours"),
        # one user's small tree: latency
        _attend("attend_one", 1, 16, 8, 4, 128, 64, 3000),
        # trees of a serving batch, 128 rows a key head: the bulk of such an engine's time
        _attend("attend_batch", 32, 32, 8, 4, 128, 64, 16000, ragged=True),
        # large trees of few users over long contexts, many query heads a key head
        _attend("attend_long", 2, 60, 8, 8, 128, 32, 65000, "f16", fan=6),
        # one user's tree, the verification between two model calls: latency
        _verify("verify_one", 1, 16, 32768, "bf16"),
        # the trees of a serving batch
        _verify("verify_batch", 16, 32, 131072, "bf16"),
        # a drafter's likeliest tokens in place of drawn ones, odd vocabulary, free slots, 32 bits
        _verify("verify_chosen", 48, 24, 50001, "f32", fan=6, chosen=True, ragged=True, temperature=0.9),
        # the accepted paths of a small batch: latency
        _keep("keep_few", 8, 32, 8, 128, 64, 4000, 6),
        # of a large one, in small pages
        _keep("keep_many", 256, 64, 8, 128, 16, 1000, 12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "verify", "verify", "keep"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    D = rng.choice([64, 128, 128])
    H = rng.choice([1, 2, 4, 8, 8])
    block = rng.choice([16, 32, 48, 64, 64, 128])
    if kind == "append":
        G = rng.choice([1, 2, 4, 5, 8])
        tree = rng.random() < 0.5
        W = rng.randint(1, 64) if tree else _log_int(rng, 1, 8000)
        B = _log_int(rng, 1, max(1, min(256, 150_000_000 // (W * H * D * (G + 2)))))
        c = _append("", B, W, H, G, D, block, _log_int(rng, 1, 100_000 if B * H * D < 16000 else 4000), dtype,
                    rng.random() < 0.6, tree, rng.choice([D, D, D // 2]), rng.choice(["halves", "neighbours"]))
    elif kind == "attend":
        G = rng.choice([1, 2, 4, 5, 8, 16])
        W = rng.randint(1, 64)
        most = 60_000_000_000 // (H * D * W * G)
        max_len = _log_int(rng, W + 1, max(W + 2, min(100_000, most)))
        B = _log_int(rng, 1, max(1, min(128, 200_000_000 // (max_len * H * D), most // max_len)))
        c = _attend("", B, W, H, G, D, block, max_len, rng.choice(["bf16", "bf16", "f16"]), rng.random() < 0.6,
                    rng.randint(1, 8))
    elif kind == "verify":
        V = _log_int(rng, 1000, 200_000)
        if rng.random() < 0.6:                            # a vocabulary padded for the matrix product before
            V = V // 64 * 64
        W = rng.randint(1, 64)
        B = _log_int(rng, 1, max(1, min(128, 60_000_000 // (V * W))))
        c = _verify("", B, W, V, dtype, rng.randint(1, 8), rng.random() < 0.4, rng.random() < 0.4,
                    rng.choice([1.0, 1.0, 0.8, 1.2]))
    else:
        W = rng.randint(1, 64)
        B = _log_int(rng, 1, 256)
        c = _keep("", B, W, H, D, block, _log_int(rng, 1, 2000), rng.randint(1, 16))
    del c["name"]
    return c


# ------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 17)


def _scale_for(amax):
    """The least power of two (2^-126 or more) whose 448-fold holds amax."""
    m, e = torch.frexp(amax)
    k = (e - 9 + (m > 0.875)).clamp(min=-126)
    return ((k + 127).to(torch.int32) << 23).view(torch.float32)


def _quantised(x, dims):
    """e4m3 codes of x with one power-of-two scale for each group along `dims`, and the scales."""
    s = _scale_for(x.abs().amax(dims, keepdim=True))
    return (x / s).to(torch.float8_e4m3fn), s


def _cache(g, pages, H, D, block):
    """A cache filled with tokens that have passed: keys and values of normal size, heads of different size."""
    kc = torch.empty(pages, H, block, D, dtype=torch.float8_e4m3fn, device=DEV)
    vc = torch.empty(pages, H, D, block, dtype=torch.float8_e4m3fn, device=DEV)
    ks = torch.empty(pages, H, device=DEV)
    vs = torch.empty(pages, H, device=DEV)
    step = max(1, 30_000_000 // (H * D * block))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        size = 0.5 + torch.rand(n, H, 1, 1, generator=g, device=DEV)
        c, s = _quantised(size * torch.randn(n, H, block, D, generator=g, device=DEV), (2, 3))
        kc[p:p + n], ks[p:p + n] = c, s[:, :, 0, 0]
        c, s = _quantised(size * torch.randn(n, H, D, block, generator=g, device=DEV), (2, 3))
        vc[p:p + n], vs[p:p + n] = c, s[:, :, 0, 0]
    return dict(k=kc, v=vc, k_scale=ks, v_scale=vs)


def _trees(seed, B, W, fan):
    """Parents [B, W] of random trees with at most `fan` children a node, and each node's depth and rank
    among its parent's children."""
    rng = random.Random(seed * 31 + 7)
    parents, depths, ranks = [], [], []
    for _ in range(B):
        p, d, r, n = [-1], [0], [0], [0] * W
        for i in range(1, W):
            u = rng.randint(max(0, (i - 1) // (fan + 1) - 1), i - 1)
            while n[u] == fan:
                u = (u + 1) % i
            p.append(u)
            d.append(d[u] + 1)
            r.append(n[u])
            n[u] += 1
        parents.append(p)
        depths.append(d)
        ranks.append(r)
    return [torch.tensor(t, dtype=torch.int32, device=DEV) for t in (parents, depths, ranks)]


def _lengths(g, case, lo):
    """Tokens of each sequence: all max_len, or spread from a sixth of it to the whole (one slot free)."""
    B, most = case["B"], case["max_len"]
    if not case.get("ragged", True):
        return torch.full((B,), most, dtype=torch.int32, device=DEV)
    n = torch.randint(max(lo, most // 6), most + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    if B > 2:
        n[B // 2] = 0
    return n


def _freqs(rot):
    """Radians a position of each pair, in 64 bits."""
    return 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)


def _prepare_verify(case, g, seed, st):
    B, W, V, fan, T = (case[k] for k in ("B", "W", "V", "fan", "temperature"))
    dt = DTYPES[case["dtype"]]
    parents, _, ranks = _trees(seed, B, W, fan)
    target = torch.empty(B, W, V, dtype=dt, device=DEV)
    draft = torch.empty(B, W, V, dtype=dt, device=DEV)
    near = torch.empty(B, W, fan, dtype=torch.int64, device=DEV)
    for i in range(W):                                # sharper and flatter rows; a drafter near its target
        row = (1.5 + 2.5 * torch.rand(B, 1, generator=g, device=DEV)) * torch.randn(B, V, generator=g, device=DEV)
        target[:, i] = row
        draft[:, i] = row + 0.6 * torch.randn(B, V, generator=g, device=DEV)
        near[:, i] = draft[:, i].float().topk(fan, 1).indices
    row = torch.arange(B, device=DEV)
    tokens = torch.zeros(B, W, dtype=torch.int32, device=DEV)
    for i in range(1, W):
        u = parents[:, i].long()
        if case["chosen"]:
            tokens[:, i] = near[row, u, ranks[:, i].long()]
        else:
            e = torch.empty(B, V, device=DEV).exponential_(generator=g)
            tokens[:, i] = (draft[row, u].float() / T - e.log()).argmax(1)
    st.update(target=target, draft=None if case["chosen"] else draft, tokens=tokens, parents=parents, counts=None,
              coins=torch.rand(B, W, generator=g, device=DEV),
              race=torch.empty(B, V, device=DEV).exponential_(generator=g))
    if case["ragged"]:
        st["counts"] = torch.randint(1, W + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        if B > 2:
            st["counts"][B // 2] = 0                  # a free slot


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case)
    kind = case["kind"]
    if kind == "verify":
        _prepare_verify(case, g, seed, st)
        return st
    B, W, H, D, block = (case[k] for k in ("B", "W", "H", "D", "block"))
    M = (case["max_len"] + (0 if kind == "attend" else W)) // block + 2
    st["cache"] = _cache(g, B * M, H, D, block)
    st["pages"] = torch.randperm(B * M, generator=g, device=DEV).to(torch.int32).view(B, M)
    n = _lengths(g, case, W if kind == "attend" else 0)
    st["lengths"] = n
    st["counts"] = None
    if kind == "keep":
        # paths as they come from trees in order of depth: kept rows that lie in place, then ones further back
        rng = random.Random(seed * 37 + 5)
        path = torch.full((B, W), -1, dtype=torch.int32)
        for b in range(B):
            keep = rng.randint(1, min(W, case["deep"]))
            still = rng.randint(min(1, keep), keep)
            back = sorted(rng.sample(range(keep, W), min(keep - still, W - keep)))
            nodes = list(range(keep - len(back))) + back
            path[b, :len(nodes)] = torch.tensor(nodes, dtype=torch.int32)
        st["path"] = path.to(DEV)
        return st
    if case["ragged"]:
        c = torch.randint(1, W + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        st["counts"] = torch.minimum(c, n) if kind == "attend" else c
    dt = DTYPES[case["dtype"]]
    HQ = H * case["G"]
    if kind == "attend":
        st["parents"] = _trees(seed, B, W, case["fan"])[0]
        st["q"] = torch.randn(B, W, HQ, D, generator=g, device=DEV).to(dt)
        st["scale"] = D ** -0.5
        return st
    rows = torch.empty(B, W, HQ + 2 * H, D, dtype=dt, device=DEV)              # one projection gives all three
    for b in range(B):
        rows[b] = 0.8 * torch.randn(W, HQ + 2 * H, D, generator=g, device=DEV)
    st.update(q=rows[:, :, :HQ], k_new=rows[:, :, HQ:HQ + H], v_new=rows[:, :, HQ + H:])
    st["freqs"] = _freqs(case["rot"])
    st["positions"] = n[:, None] + _trees(seed, B, W, 4)[1] if case["tree"] else None
    return st


# ------------------------------------------------------------------------------ plain forms
def _rotated(x, st):
    """x [B, W, heads, D], its first `rot` elements turned by their positions, in 32 bits."""
    rot, W = st["rot"], st["W"]
    pos = st["positions"]
    pos = st["lengths"][:, None] + torch.arange(W, device=x.device) if pos is None else pos
    turn = (pos.double()[..., None] * st["freqs"])[:, :, None]                 # far angles want 64 bits
    cos, sin = turn.cos().float(), turn.sin().float()
    x = x.float()
    if st["pairs"] == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., :rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _put(st, codes, scale, x, turn, at, page, old, fresh):
    """Writes the rows x[b, at] into pages of codes; `turn`: the tokens are the last axis."""
    B, nb = page.shape
    row = torch.arange(B, device=page.device)[:, None]
    x = x.float()[row, at].view(B, nb, st["block"], x.shape[2], x.shape[3]).transpose(2, 3)
    x = torch.where(fresh, x, 0.0)                    # [B, nb, H, block, D]
    was = codes.view(torch.uint8)[page].view(torch.float8_e4m3fn)
    was = was.transpose(3, 4) if turn else was
    need = _scale_for(x.abs().amax((3, 4)))
    s_old = scale[page]
    s = torch.where(old.any(3)[..., 0], torch.maximum(s_old, need), need)
    s = torch.where(fresh.any(3)[..., 0], s, s_old)[..., None, None]
    kept = torch.where(old & (s != s_old[..., None, None]),
                       (was.float() * (s_old[..., None, None] / s)).to(torch.float8_e4m3fn).float(), was.float())
    out = torch.where(fresh, (x / s).to(torch.float8_e4m3fn).float(), kept).to(torch.float8_e4m3fn)
    out = out.transpose(3, 4) if turn else out
    codes.view(torch.uint8)[page] = out.contiguous().view(torch.uint8)
    scale[page] = s[..., 0, 0]


def _plain_append(st):
    c, W, block, n = st["cache"], st["W"], st["block"], st["lengths"].long()
    new = torch.full_like(n, W) if st["counts"] is None else st["counts"].long()
    nb = (W + 2 * block - 2) // block
    first = n // block
    page = st["pages"].long().gather(1, first[:, None] + torch.arange(nb, device=n.device))
    pos = first[:, None] * block + torch.arange(nb * block, device=n.device)          # [B, nb * block]
    at = (pos - n[:, None]).clamp(0, W - 1)
    old = (pos < n[:, None]).view(-1, nb, 1, block, 1)
    fresh = ((pos >= n[:, None]) & (pos < (n + new)[:, None])).view(-1, nb, 1, block, 1)
    _put(st, c["k"], c["k_scale"], _rotated(st["k_new"], st), False, at, page, old, fresh)
    _put(st, c["v"], c["v_scale"], st["v_new"], True, at, page, old, fresh)
    q = _rotated(st["q"], st)
    if st["counts"] is not None:                      # queries behind a sequence's own count are left zero
        live = (torch.arange(W, device=q.device) < new[:, None])[..., None, None]
        q = torch.where(live, q, 0.0)
    return dict(k=c["k"], v=c["v"], k_scale=c["k_scale"], v_scale=c["v_scale"], q=q.to(st["q"].dtype))


def _keep_one(st, codes, scale, turn):
    """Moves the codes' rows; `turn`: the tokens are the last axis."""
    W, block, n = st["W"], st["block"], st["lengths"].long()
    path = st["path"].long()
    at = n[:, None] + path.clamp(min=0)
    page, place = st["pages"].long().gather(1, at // block), at % block
    raw = codes.view(torch.uint8)
    x = (raw[page, :, :, place] if turn else raw[page, :, place]).view(torch.float8_e4m3fn).float() * scale[page][..., None]
    moves = (path >= 0) & (path != torch.arange(W, device=n.device))
    nb = (W + 2 * block - 2) // block
    first = n // block
    page = st["pages"].long().gather(1, first[:, None] + torch.arange(nb, device=n.device))
    to = first[:, None] * block + torch.arange(nb * block, device=n.device) - n[:, None]
    fresh = (moves.gather(1, to.clamp(0, W - 1)) & (to >= 0) & (to < W)).view(-1, nb, 1, block, 1)
    row = torch.arange(n.shape[0], device=n.device)[:, None]
    x = x[row, to.clamp(0, W - 1)].view(-1, nb, block, x.shape[2], x.shape[3]).transpose(2, 3)
    x = torch.where(fresh, x, 0.0)                    # [B, nb, H, block, D]
    was = raw[page].view(torch.float8_e4m3fn)
    was = was.transpose(3, 4) if turn else was
    s_old = scale[page]
    s = torch.where(fresh.any(3)[..., 0], torch.maximum(s_old, _scale_for(x.abs().amax((3, 4)))), s_old)
    old, new = s_old[..., None, None], s[..., None, None]
    kept = torch.where(new != old, (was.float() * (old / new)).to(torch.float8_e4m3fn).float(), was.float())
    out = torch.where(fresh, (x / new).to(torch.float8_e4m3fn).float(), kept).to(torch.float8_e4m3fn)
    out = out.transpose(3, 4) if turn else out
    raw[page] = out.contiguous().view(torch.uint8)
    scale[page] = s


def _plain_keep(st):
    c = st["cache"]
    _keep_one(st, c["k"], c["k_scale"], False)
    _keep_one(st, c["v"], c["v_scale"], True)
    return dict(k=c["k"], v=c["v"], k_scale=c["k_scale"], v_scale=c["v_scale"])


def _ancestors(parents):
    """[B, W, W]: whether node j is node i or one of those above it."""
    B, W = parents.shape
    eye = torch.eye(W, device=parents.device).expand(B, W, W)
    up = eye[:, :, :W] * 0
    up = up.scatter(2, parents.long().clamp(min=0)[..., None], (parents >= 0).float()[..., None]) + eye
    for _ in range(max(1, (W - 1).bit_length())):     # one step up; then two, four, ...
        up = ((up @ up) > 0).float()
    return up > 0


def _plain_attend(st):
    c, B, W, H, G, D, block = st["cache"], st["B"], st["W"], st["H"], st["G"], st["D"], st["block"]
    page = st["pages"].long()
    M = page.shape[1]
    n = st["lengths"].long()
    new = torch.full_like(n, W) if st["counts"] is None else st["counts"].long()
    k = c["k"].view(torch.uint8)[page].view(torch.float8_e4m3fn).float() * c["k_scale"][page][..., None, None]
    k = k.transpose(1, 2).reshape(B, H, M * block, D)
    q = st["q"].float().view(B, W, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, W * G, D)
    s = (q @ k.transpose(2, 3)).view(B, H, W, G, M * block) * st["scale"]
    del k
    key = torch.arange(M * block, device=n.device) - (n - new)[:, None]               # in the tree from 0 on
    above = _ancestors(st["parents"]).gather(2, key.clamp(0, W - 1)[:, None].expand(B, W, M * block))
    seen = ((key < 0)[:, None] | above) & (key < new[:, None])[:, None]
    seen &= (torch.arange(W, device=n.device) < new[:, None])[..., None]
    seen = seen[:, None, :, None, :]
    s = torch.where(seen, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = (s - m).exp()
    del s
    total = p.sum(-1, keepdim=True)
    lse = (total.log() + m)[..., 0].permute(0, 2, 1, 3).reshape(B, W, H * G)
    p = p / torch.where(total == 0, 1.0, total)
    v = c["v"].view(torch.uint8)[page].view(torch.float8_e4m3fn).float() * c["v_scale"][page][..., None, None]
    v = v.permute(0, 2, 3, 1, 4).reshape(B, H, D, M * block)
    o = p.view(B, H, W * G, M * block) @ v.transpose(2, 3)
    o = o.view(B, H, W, G, D).permute(0, 2, 1, 3, 4).reshape(B, W, H * G, D)
    return dict(out=o.to(st["q"].dtype), lse=lse)


def _log_probs(x, T):
    x = x.float()
    d = (x - x.amax(2, keepdim=True)) / T
    return d - d.exp().sum(2, keepdim=True).log()


def _plain_verify(st):
    T, B, W, fan = st["temperature"], st["B"], st["W"], st["fan"]
    tok, parents, coins = st["tokens"].long(), st["parents"].long(), st["coins"]
    dev = tok.device
    n = torch.full((B,), W, device=dev) if st["counts"] is None else st["counts"].long()
    node = torch.arange(W, device=dev)
    here = (node < n[:, None]) & (parents >= 0)       # nodes with a parent
    up = parents.clamp(min=0)
    rank = ((parents[:, :, None] == parents[:, None, :]) & (node < node[:, None])).sum(2)
    child = torch.full((B, W * fan + 1), -1, device=dev)
    child.scatter_(1, torch.where(here, up * fan + rank, W * fan), node.expand(B, W).contiguous())
    child = child[:, :-1].view(B, W, fan)
    q = _log_probs(st["target"], T).exp_()
    p = None if st["chosen"] else _log_probs(st["draft"], T).exp_()
    beta, mass = torch.zeros(B, W, device=dev), torch.ones(B, W, device=dev)
    took = torch.full((B, W), -1, device=dev)
    ratio = torch.zeros(B, W + 1, device=dev)
    left = q if p is not None else q.clone()          # chosen children: what they leave of each row
    for k in range(fan):
        c = child[:, :, k]
        live = (c >= 0) & (took < 0)
        x = tok.gather(1, c.clamp(min=0).view(B, -1)).view(B, W, 1)
        qx = q.gather(2, x)[..., 0]
        px = torch.ones_like(qx) if p is None else p.gather(2, x)[..., 0]
        value = left.gather(2, x)[..., 0] if p is None else qx / px - beta
        eta = coins.gather(1, c.clamp(min=0).view(B, -1)).view(B, W)
        hit = live & (eta * mass < value)
        ratio.scatter_(1, torch.where(live, c, W), (qx.log() - px.log()))
        took = torch.where(hit, c, took)
        miss = live & ~hit
        if p is None:
            left.scatter_(2, x, torch.where(miss[..., None], 0.0, left.gather(2, x)))
            mass = torch.where(miss, left.sum(2), mass)
        else:
            beta = torch.where(miss, beta + mass, beta)
            mass = torch.where(miss, (q - beta[..., None] * p).clamp(min=0).sum(2), mass)
    at = torch.where(n > 0, 0, -1)
    path = [at]
    for _ in range(W - 1):
        step = took.gather(1, at.clamp(min=0)[:, None])[:, 0]
        step = torch.where((at >= 0) & (step >= 0), step, -1)
        path.append(step)
        at = step
    path = torch.stack(path, 1)
    long = (path >= 0).sum(1)
    end = path.gather(1, (long - 1).clamp(min=0)[:, None])[:, 0].clamp(min=0)
    row = torch.arange(B, device=dev)
    r = left[row, end] if p is None else q[row, end] - beta[row, end][:, None] * p[row, end]
    nxt = torch.where(r > 0, r / st["race"], -1.0).argmax(1)
    free = n <= 0
    on = torch.zeros(B, W + 1, dtype=torch.bool, device=dev).scatter_(1, torch.where(path >= 0, path, W), True)
    first = took.gather(1, up)                        # the child taken there: later ones are not tried
    tried = here & on[:, :W].gather(1, up) & ((first < 0) | (node <= first))
    return dict(accepted_len=(long - 1).clamp(min=0).to(torch.int32), path=path.to(torch.int32),
                next_token=torch.where(free, -1, nxt).to(torch.int32),
                log_ratio=torch.where(tried, ratio[:, :W], 0.0))


# ------------------------------------------------------------------------------ the calls
def _own(st):
    from paper_2606_13426_gb300 import api
    kind = st["kind"]
    if kind == "append":
        q = api.cache_append_rotary(st["cache"], st["k_new"], st["v_new"], st["pages"], st["lengths"], st["freqs"],
                                    pairs=st["pairs"], q=st["q"], positions=st["positions"], counts=st["counts"])
        return dict(st["cache"], q=q)
    if kind == "attend":
        r = api.tree_attend(st["q"], st["cache"], st["pages"], st["lengths"], st["parents"], counts=st["counts"],
                            scale=st["scale"])
        return dict(out=r["out"], lse=r["lse"])
    if kind == "verify":
        r = api.tree_verify(st["target"], st["draft"], st["tokens"], st["parents"], counts=st["counts"],
                            temperature=st["temperature"], coins=st["coins"], race=st["race"])
        return {k: r[k] for k in ("accepted_len", "path", "next_token", "log_ratio")}
    api.cache_keep(st["cache"], st["path"], st["pages"], st["lengths"])
    return dict(st["cache"])


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "attend": _plain_attend, "verify": _plain_verify,
            "keep": _plain_keep}[state["kind"]](state)


# ------------------------------------------------------------------------------ work
def work(case):
    kind, B, W = case["kind"], case["B"], case["W"]
    if kind == "verify":
        V, es = case["V"], BYTES[case["dtype"]]
        # about three nodes of a drawn tree are on the path (two of one with chosen tokens), the last of them
        # often without children; a shorter tree ends sooner
        on = min(W, 2 if case["chosen"] else 3) * (0.75 if case["ragged"] else 1)
        rows = on if case["chosen"] else 2 * on - 0.5
        return dict(bytes=B * rows * V * es + B * V * 4 + B * W * 20, flops=4 * B * rows * V)
    H, D = case["H"], case["D"]
    if kind == "keep":
        rows = min(W, case["deep"]) / 2 + 0.5
        return dict(bytes=4 * B * rows * H * D, flops=4 * B * rows * H * D)
    G = case["G"]
    steps = (W + 1) / 2 if case["ragged"] else W
    if kind == "append":
        es = BYTES[case["dtype"]]
        return dict(bytes=B * steps * H * D * (2 * es + 2 + G * es) + B * W * H * G * D * es,
                    flops=B * steps * H * D * (3 * (G + 1) + 4))
    mean = case["max_len"] * (7 / 12 if case["ragged"] else 1)
    if case["ragged"] and B > 2:
        mean *= (B - 1) / B
    return dict(bytes=2 * B * mean * H * D + 2 * B * steps * H * G * D * 2, flops=4 * B * mean * steps * H * G * D)


# ------------------------------------------------------------------------------ 64 bits
def _e4m3(x):
    """The nearest e4m3 value (ties to even) of x, |x| < 464, in 64 bits."""
    _, e = torch.frexp(x.abs().clamp(min=2.0 ** -6))
    unit = _power(e - 4)
    return torch.round(x / unit) * unit


def _power(k):
    """2^k in 64 bits, exactly."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _exact_rows(st, rows):
    """What appending the rows (a function of the sequence: keys and values [n, H, D]) makes of the cache."""
    c, block = st["cache"], st["block"]
    got = dict(k=c["k"].double(), v=c["v"].double(), k_scale=c["k_scale"].double(), v_scale=c["v_scale"].double())
    lengths, pages = st["lengths"].tolist(), st["pages"].tolist()
    for b in range(st["B"]):
        x = rows(b)
        n, new = lengths[b], x[0].shape[0]
        for j in range(n // block, (n + new + block - 1) // block):
            page = pages[b][j]
            lo, hi = max(n, j * block), min(n + new, (j + 1) * block)
            kept = max(0, n - j * block)
            for codes, scales, y, turn in ((got["k"], got["k_scale"], x[0], False), (got["v"], got["v_scale"], x[1], True)):
                y = y[lo - n:hi - n].transpose(0, 1)                                  # [H, tokens, D]
                here = codes[page].transpose(1, 2) if turn else codes[page]
                scale = _power_above(y.abs().amax((1, 2)) / 448)
                if kept:
                    scale = torch.maximum(scale, scales[page])
                    here[:, :kept] = _e4m3(here[:, :kept] * (scales[page] / scale)[:, None, None])
                here[:, lo - j * block:hi - j * block] = _e4m3(y / scale[:, None, None])
                scales[page] = scale
    return got


def _power_above(x):
    """The least power of two that is x or more (2^-126 at least)."""
    m, e = torch.frexp(x.clamp(min=2.0 ** -126))
    return _power(e - (m == 0.5).to(e.dtype))


def _turned(st, x, b, n):
    """Sequence b's first n rows of x [B, W, heads, D] as complex numbers, turned."""
    rot, x = st["rot"], x[b, :n].double()
    first = float(st["lengths"][b])
    pos = first + torch.arange(n, device=DEV, dtype=torch.float64) if st["positions"] is None else st["positions"][b, :n].double()
    unit = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos[:, None, None] * st["freqs"])
    out = x.clone()
    if st["pairs"] == "halves":
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * unit
        out[..., :rot // 2], out[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.view_as_complex(x[..., :rot].reshape(x.shape[:-1] + (rot // 2, 2)).contiguous()) * unit
        out[..., :rot] = torch.view_as_real(z).flatten(-2)
    return out


def _exact_append(st):
    counts = [st["W"]] * st["B"] if st["counts"] is None else st["counts"].tolist()
    got = _exact_rows(st, lambda b: (_turned(st, st["k_new"], b, counts[b]), st["v_new"][b, :counts[b]].double()))
    q = torch.zeros(st["q"].shape, dtype=torch.float32, device=DEV)
    for b in range(st["B"]):
        q[b, :counts[b]] = _turned(st, st["q"], b, counts[b])
    got["q"] = q
    return got


def _exact_keep(st):
    c, block = st["cache"], st["block"]
    got = dict(k=c["k"].double(), v=c["v"].double(), k_scale=c["k_scale"].double(), v_scale=c["v_scale"].double())
    held = dict(k=got["k"] * got["k_scale"][..., None, None], v=got["v"] * got["v_scale"][..., None, None])
    lengths, path, pages = st["lengths"].tolist(), st["path"].tolist(), st["pages"].tolist()
    for b in range(st["B"]):
        into = {}                                     # of each page: rows, and where they come from
        for j, i in enumerate(path[b]):
            if i >= 0 and i != j:
                to, at = lengths[b] + j, lengths[b] + i
                into.setdefault(pages[b][to // block], []).append((to % block, pages[b][at // block], at % block))
        for page, rows in into.items():
            for name in ("k", "v"):
                x = torch.stack([held[name][p, :, :, r] if name == "v" else held[name][p, :, r] for _, p, r in rows], 1)
                was = got[name + "_scale"][page].clone()
                scale = torch.maximum(was, _power_above(x.abs().amax((1, 2)) / 448))
                here = got[name][page].transpose(1, 2) if name == "v" else got[name][page]
                here[:] = torch.where((scale != was)[:, None, None], _e4m3(here * (was / scale)[:, None, None]), here)
                here[:, [t for t, _, _ in rows]] = _e4m3(x / scale[:, None, None])
                got[name + "_scale"][page] = scale
    return got


def _exact_attend(st):
    c, B, W, H, G, D, block = st["cache"], st["B"], st["W"], st["H"], st["G"], st["D"], st["block"]
    out = torch.zeros(B, W, H * G, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, W, H * G), -math.inf, dtype=torch.float64, device=DEV)
    lengths, parents = st["lengths"].tolist(), st["parents"].tolist()
    counts = [W] * B if st["counts"] is None else st["counts"].tolist()
    for b in range(B):
        n, new = lengths[b], counts[b]
        if not n or not new:
            continue
        seen = torch.ones(new, n, dtype=torch.bool)
        seen[:, n - new:] = False
        for i in range(new):
            u = i
            while u >= 0:
                seen[i, n - new + u] = True
                u = parents[b][u]
        seen = seen.to(DEV).repeat_interleave(G, 0)
        page = st["pages"][b, : (n + block - 1) // block].long()
        for h in range(H):
            k = c["k"].view(torch.uint8)[page, h].view(torch.float8_e4m3fn).double() * c["k_scale"][page, h].double()[:, None, None]
            v = c["v"].view(torch.uint8)[page, h].view(torch.float8_e4m3fn).double() * c["v_scale"][page, h].double()[:, None, None]
            k = k.reshape(-1, D)[:n]
            v = v.transpose(1, 2).reshape(-1, D)[:n]
            s = st["scale"] * (st["q"][b, :new, h * G:(h + 1) * G].double().reshape(new * G, D) @ k.T)
            s = s.masked_fill(~seen, -math.inf)
            out[b, :new, h * G:(h + 1) * G] = (torch.softmax(s, 1) @ v).view(new, G, D)
            lse[b, :new, h * G:(h + 1) * G] = torch.logsumexp(s, 1).view(new, G)
    return dict(out=out, lse=lse)


def _exact_verify(st):
    B, W, T = st["B"], st["W"], st["temperature"]
    ratio = torch.zeros(B, W, dtype=torch.float64)
    counts = [W] * B if st["counts"] is None else st["counts"].tolist()
    parents, tokens, coins = st["parents"].tolist(), st["tokens"].tolist(), st["coins"].tolist()
    for b in range(B):
        at = 0 if counts[b] > 0 else None
        while at is not None:
            children = [i for i in range(1, counts[b]) if parents[b][i] == at]
            went = None
            if children:
                q = torch.softmax(st["target"][b, at].double() / T, 0)
                p = None if st["chosen"] else torch.softmax(st["draft"][b, at].double() / T, 0)
                rest = q                              # the distribution that is left, normalised
            for i in children:
                x = tokens[b][i]
                ratio[b, i] = math.log(q[x]) - (0.0 if p is None else math.log(p[x]))
                if coins[b][i] < float(rest[x]) / (1.0 if p is None else float(p[x])):
                    went = i
                    break
                if p is None:
                    rest = rest.clone()
                    rest[x] = 0
                else:
                    rest = (rest - p).clamp(min=0)
                rest = rest / rest.sum()
            at = went
    return dict(accepted_len=None, path=None, next_token=None, log_ratio=ratio.to(DEV))


def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "verify": _exact_verify, "keep": _exact_keep}[case["kind"]](st)
