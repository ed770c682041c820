"""The cases whose speed the token operators are measured by.

A round of speculative decoding over tokens appends the window's keys and values to a
cache held in 8 bits (``api.cache_append``), attends over it (``api.cache_attend``), scores
tokens under the logits (``api.token_scores``; ``api.token_scores_train`` with the gradient, where
the model is trained on them) and verifies the drafted window (``api.token_verify``).  ``run`` makes
those calls where ``own`` is true and computes the same in elementary torch operations
elsewhere; ``exact`` restates the definitions in 64 bits.

Cache layout: codes are float8_e4m3fn, keys [pages, heads, block, dim], values
[pages, heads, dim, block], one float32 scale per page and head for each; a sequence's
tokens are in the pages that its row of the page table lists.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ------------------------------------------------------------------------------ cases
def _scores(name, N, V, dtype, top_k=0, masked=False, temperature=1.0, pad=0):
    return dict(name=name, kind="scores", N=N, V=V, dtype=dtype, top_k=top_k, masked=masked,
                temperature=temperature, pad=pad)


def _train(name, N, V, dtype, entropy=True, pad=0):
    return dict(name=name, kind="train", N=N, V=V, dtype=dtype, entropy=entropy, pad=pad)


def _verify(name, B, L, V, dtype, mode="block", ragged=False, temperature=1.0):
    return dict(name=name, kind="verify", B=B, L=L, V=V, dtype=dtype, mode=mode, ragged=ragged,
                temperature=temperature)


def _append(name, B, W, H, D, block, max_len, dtype="bf16", ragged=False):
    return dict(name=name, kind="append", B=B, W=W, H=H, D=D, block=block, max_len=max_len,
                dtype=dtype, ragged=ragged)


def _attend(name, B, W, H, G, D, block, max_len, dtype="bf16", ragged=False, span=0):
    return dict(name=name, kind="attend", B=B, W=W, H=H, G=G, D=D, block=block, max_len=max_len,
                dtype=dtype, ragged=ragged, span=span)


def listed():
    return [
        # one decoding step of a few users who asked for log probabilities: latency
        _scores("scores_step", 8, 65536, "bf16", top_k=8),
        # every position of a batch of verified windows, some under a grammar's mask
        _scores("scores_window", 144, 131072, "bf16", top_k=20, masked=True, temperature=0.8),
        # a training step of a drafter on its tokens, with an entropy bonus: the largest read and write
        _train("train_batch", 4096, 65536, "bf16"),
        # the same in 32 bits, an odd vocabulary in a padded buffer (rows on no 16-byte boundary)
        _train("train_odd", 333, 50001, "f32", entropy=False, pad=6),
        # one user's window, the verification between two model calls
        _verify("verify_one", 1, 4, 32768, "bf16"),
        # a serving batch
        _verify("verify_batch", 16, 8, 131072, "bf16"),
        # chains with shorter windows and free slots, sample verification, odd vocabulary, 32 bits
        _verify("verify_ragged", 48, 7, 50001, "f32", mode="sample", ragged=True, temperature=0.9),
        # the window's keys and values of one round of a serving batch
        _append("append_window", 64, 9, 8, 128, 64, 4096, ragged=True),
        # prompts of several users
        _append("append_prompts", 4, 8000, 8, 128, 64, 500),
        # one user's single token: latency
        _attend("attend_one", 1, 1, 8, 4, 128, 64, 3000),
        # verification windows of a serving batch: the bulk of such an engine's time
        _attend("attend_window", 32, 9, 8, 4, 128, 64, 16000, ragged=True),
        # single tokens over long contexts, few sequences: the longest read for few rows
        _attend("attend_long", 2, 1, 8, 8, 128, 32, 131000, "f16", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["scores", "train", "verify", "append", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    V = _log_int(rng, 1000, 200_000)
    if rng.random() < 0.6:                            # a vocabulary padded for the matrix product before
        V = V // 64 * 64
    pad = rng.choice([0, 0, 1, 5, 64])
    if kind == "scores":
        top_k = rng.choice([0, 1, 5, 8, 20, 32])
        N = _log_int(rng, 1, max(2, min(600, 20_000_000 // V)))
        c = _scores("", N, V, dtype, top_k, rng.random() < 0.4, rng.choice([1.0, 1.0, 0.7, 1.3]), pad)
    elif kind == "train":
        N = _log_int(rng, 16, max(32, min(8000, 500_000_000 // (V * BYTES[dtype]))))
        c = _train("", N, V, dtype, rng.random() < 0.5, pad)
    elif kind == "verify":
        L = rng.randint(1, 12)
        B = _log_int(rng, 1, max(1, min(128, 40_000_000 // (V * (2 * L + 1)))))
        c = _verify("", B, L, V, dtype, rng.choice(["block", "block", "sample"]), rng.random() < 0.4,
                    rng.choice([1.0, 1.0, 0.8, 1.2]))
    else:
        D = rng.choice([64, 128, 128])
        H = rng.choice([1, 2, 4, 8, 8])
        block = rng.choice([16, 32, 64, 64, 128])
        ragged = rng.random() < 0.6
        if kind == "append":
            W = _log_int(rng, 1, 8000)
            B = _log_int(rng, 1, max(1, min(256, 30_000_000 // (W * H * D))))
            c = _append("", B, W, H, D, block, rng.randint(0, 2000), dtype, ragged)
        else:
            W = rng.choice([1, 1, 2, 4, 5, 8, 9, 13, 17])
            G = rng.choice([1, 2, 4, 5, 8, 16])
            max_len = _log_int(rng, W + 1, min(100_000, 10_000_000_000 // (H * D * W * G)))
            B = _log_int(rng, 1, max(1, min(128, 200_000_000 // (max_len * H * D), 10_000_000_000 // (max_len * H * D * W * G))))
            c = _attend("", B, W, H, G, D, block, max_len, rng.choice(["bf16", "bf16", "f16"]), ragged,
                        rng.choice([0, 0, 0, 1000]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 17)


def _logits(g, rows, V, dtype, pad):
    """[rows, V] logits, sharper and flatter rows, a view of a buffer padded by `pad` columns."""
    buf = torch.empty(rows, V + pad, dtype=DTYPES[dtype], device=DEV)
    step = max(1, 50_000_000 // (V + pad))
    for r in range(0, rows, step):
        n = min(step, rows - r)
        sharp = 1.5 + 2.5 * torch.rand(n, 1, generator=g, device=DEV)
        buf[r:r + n] = sharp * torch.randn(n, V + pad, generator=g, device=DEV)
    return buf[:, :V]


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


def _lengths(g, case, lo):
    """Tokens of each sequence: all max_len, or spread from a sixth of it to the whole (one slot free)."""
    B, most = case["B"], case["max_len"]
    if not case["ragged"]:
        return torch.full((B,), most, dtype=torch.int32, device=DEV)
    n = torch.randint(max(lo, most // 6), most + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    if B > 2:
        n[B // 2] = 0
    return n


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case)
    kind = case["kind"]
    if kind in ("scores", "train"):
        N, V = case["N"], case["V"]
        x = _logits(g, N, V, case["dtype"], case["pad"])
        if case.get("masked"):                        # a third of the rows allow a few hundred tokens, one none
            for r in range(0, N, 3):
                keep = torch.randint(0, V, (300,), generator=g, device=DEV)
                row = torch.full_like(x[r], -math.inf)
                row[keep] = x[r, keep]
                x[r] = row
            if N > 4:
                x[N // 2] = -math.inf
        likely = x[:, : min(V, 256)].argmax(1)        # half the tokens are likely ones
        other = torch.randint(0, V, (N,), generator=g, device=DEV)
        tok = torch.where(torch.rand(N, generator=g, device=DEV) < 0.5, likely, other).to(torch.int32)
        if N > 8:
            tok[torch.rand(N, generator=g, device=DEV) < 0.05] = -1      # padding
        st.update(logits=x, tokens=tok)
        if kind == "train":
            st["g_logprob"] = -torch.rand(N, generator=g, device=DEV) / N
            st["g_entropy"] = torch.full((N,), -0.01 / N, device=DEV) if case["entropy"] else None
    elif kind == "verify":
        B, L, V = case["B"], case["L"], case["V"]
        dt = DTYPES[case["dtype"]]
        tl = _logits(g, B * (L + 1), V, "f32", 0).view(B, L + 1, V)
        dl = torch.empty(B, L, V, dtype=dt, device=DEV)
        tok = torch.empty(B, L, dtype=torch.int32, device=DEV)
        for b in range(B):                            # a drafter near its target; tokens drawn from it
            dl[b] = tl[b, :L] + 0.6 * torch.randn(L, V, generator=g, device=DEV)
            e = torch.empty(L, V, device=DEV).exponential_(generator=g)
            tok[b] = (dl[b].float() / case["temperature"] - e.log()).argmax(1).to(torch.int32)
        st.update(target=tl.to(dt), draft=dl, tokens=tok,
                  coins=torch.rand(B, L, generator=g, device=DEV),
                  race=torch.empty(B, V, device=DEV).exponential_(generator=g), L_eff=None)
        if case["ragged"]:
            n = torch.randint(0, L + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
            if B > 2:
                n[B // 2] = -1                        # a free slot
            st["L_eff"] = n
    else:
        B, W, H, D, block = (case[k] for k in ("B", "W", "H", "D", "block"))
        room = case["max_len"] + (W if kind == "append" else 0)
        M = room // block + 2
        st["cache"] = _cache(g, B * M, H, D, block)
        st["pages"] = torch.randperm(B * M, generator=g, device=DEV).to(torch.int32).view(B, M)
        n = _lengths(g, case, W if kind == "attend" else 0)
        st["lengths"] = n
        st["counts"] = None
        if case["ragged"]:
            c = torch.randint(1, W + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
            st["counts"] = torch.minimum(c, n) if kind == "attend" else c
        dt = DTYPES[case["dtype"]]
        if kind == "append":
            st["k_new"] = (0.8 * torch.randn(B, W, H, D, generator=g, device=DEV)).to(dt)
            st["v_new"] = (0.8 * torch.randn(B, W, H, D, generator=g, device=DEV)).to(dt)
        else:
            st["q"] = torch.randn(B, W, H * case["G"], D, generator=g, device=DEV).to(dt)
            st["scale"] = D ** -0.5
    return st


# ------------------------------------------------------------------------------ plain forms
def _plain_scores(st):
    x, T, k = st["logits"].float(), st.get("temperature", 1.0), st.get("top_k", 0)
    m = x.amax(1)
    empty = m == -math.inf
    d = (x - torch.where(empty, 0.0, m)[:, None]) / T
    e = d.exp()
    s = e.sum(1)
    ls = s.log()
    mean = torch.where(x == -math.inf, 0.0, e * d).sum(1) / s
    tok = st["tokens"].long()
    lp = d.gather(1, tok.clamp(min=0)[:, None])[:, 0] - ls
    r = dict(logprob=torch.where(tok < 0, 0.0, torch.where(empty, -math.inf, lp)),
             entropy=torch.where(empty, 0.0, ls - mean), row_max=m, log_sum=ls)
    if k:                                             # value first, then the lower index
        bits = (x + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + (x.shape[1] - 1 - torch.arange(x.shape[1], device=x.device))
        key = key.topk(k, 1).values
        ids = x.shape[1] - 1 - (key & 0xFFFFFFFF)
        top = x.gather(1, ids)
        gone = top == -math.inf
        r["top_ids"] = torch.where(gone, -1, ids).to(torch.int32)
        r["top_logprob"] = torch.where(gone, -math.inf, (top - m[:, None]) / T - ls[:, None])
    return r


def _plain_train(st):
    r = _plain_scores(st)
    x, tok = st["logits"].float(), st["tokens"].long()
    d = x - r["row_max"][:, None]
    lp = d - r["log_sum"][:, None]
    p = lp.exp()
    gl = torch.where(tok < 0, 0.0, st["g_logprob"])
    dx = -gl[:, None] * p
    dx.scatter_add_(1, tok.clamp(min=0)[:, None], gl[:, None])
    if st["g_entropy"] is not None:
        dx -= st["g_entropy"][:, None] * p * (lp + r["entropy"][:, None])
    return dict(logprob=r["logprob"], entropy=r["entropy"], d_logits=dx.to(st["logits"].dtype))


def _log_probs(x, T):
    x = x.float()
    d = (x - x.amax(2, keepdim=True)) / T
    return d - d.exp().sum(2, keepdim=True).log()


def _plain_verify(st):
    T, L = st["temperature"], st["L"]
    lq, lp = _log_probs(st["target"], T), _log_probs(st["draft"], T)
    tok = st["tokens"].long()[..., None]
    B, dev = tok.shape[0], tok.device
    n = torch.full((B,), L, device=dev) if st["L_eff"] is None else st["L_eff"].long()
    step = torch.arange(L, device=dev)
    inside = step < n[:, None]
    ell = torch.where(inside, (lq[:, :L].gather(2, tok) - lp.gather(2, tok))[..., 0], 0.0)
    if st["mode"] == "sample":
        ok = (st["coins"] < ell.exp()) & inside
        acc = ok.long().cumprod(1).sum(1)
        la = torch.zeros(B, L + 1, device=dev)
    else:
        total = torch.cat([torch.zeros(B, 1, device=dev), ell.cumsum(1)], 1)
        la = total - total.cummax(1).values           # log alpha_0 .. log alpha_L
        alpha = la.exp()
        mass = (alpha[:, 1:L, None] * lq[:, 1:L].exp() - lp[:, 1:].exp()).clamp(min=0).sum(2)
        mass = torch.cat([mass, torch.zeros(B, 1, device=dev)], 1)
        a = alpha[:, 1:]
        h = torch.where(a == 1, 1.0, mass / (mass + 1 - a))
        h = torch.where(step == n[:, None] - 1, a, h)
        ok = (st["coins"] < h) & inside
        acc = (ok * (step + 1)).amax(1)
    row = torch.arange(B, device=dev)
    last = lq[row, acc].exp()
    rest = last * la[row, acc].exp()[:, None] - lp[row, acc.clamp(max=L - 1)].exp()
    r = torch.where((acc == n.clamp(min=0))[:, None], last, rest)
    score = torch.where(r > 0, r / st["race"], -1.0)
    nxt = score.argmax(1)
    free = n < 0
    return dict(accepted_len=torch.where(free, 0, acc).to(torch.int32),
                next_token=torch.where(free, -1, nxt).to(torch.int32), log_ratio=ell)


def _plain_append(st):
    c, B, W, block = st["cache"], st["B"], st["W"], st["block"]
    n = st["lengths"].long()
    new = torch.full_like(n, W) if st["counts"] is None else st["counts"].long()
    nb = (W + 2 * block - 2) // block
    first = n // block
    page = st["pages"].long().gather(1, first[:, None] + torch.arange(nb, device=n.device))
    pos = first[:, None] * block + torch.arange(nb * block, device=n.device)          # [B, nb * block]
    at = (pos - n[:, None]).clamp(0, W - 1)
    old = (pos < n[:, None]).view(B, nb, 1, block, 1)
    fresh = ((pos >= n[:, None]) & (pos < (n + new)[:, None])).view(B, nb, 1, block, 1)
    row = torch.arange(B, device=n.device)[:, None]
    for codes, scale, x, turn in ((c["k"], c["k_scale"], st["k_new"], False), (c["v"], c["v_scale"], st["v_new"], True)):
        x = x.float()[row, at].view(B, nb, block, x.shape[2], x.shape[3]).transpose(2, 3)
        x = torch.where(fresh, x, 0.0)                # [B, nb, H, block, D]
        was = codes.view(torch.uint8)[page].view(torch.float8_e4m3fn)
        was = was.transpose(3, 4) if turn else was
        need = _scale_for(x.abs().amax((3, 4)))
        s_old = scale[page]
        s = torch.where(old.any(3)[..., 0], torch.maximum(s_old, need), need)
        s = torch.where(fresh.any(3)[..., 0], s, s_old)[..., None, None]
        kept = torch.where(old & (s != s_old[..., None, None]), (was.float() * (s_old[..., None, None] / s)).to(torch.float8_e4m3fn).float(), was.float())
        out = torch.where(fresh, (x / s).to(torch.float8_e4m3fn).float(), kept).to(torch.float8_e4m3fn)
        out = out.transpose(3, 4) if turn else out
        codes.view(torch.uint8)[page] = out.contiguous().view(torch.uint8)
        scale[page] = s[..., 0, 0]
    return dict(k=c["k"], v=c["v"], k_scale=c["k_scale"], v_scale=c["v_scale"])


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
    at = (n - new)[:, None] + torch.arange(W, device=n.device)                        # positions of the queries
    key = torch.arange(M * block, device=n.device)
    seen = (key <= at[..., None]) & (torch.arange(W, device=n.device) < new[:, None])[..., None]
    if st["span"]:
        seen &= key > at[..., None] - st["span"]
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


# ------------------------------------------------------------------------------ the calls
def _own(st):
    from paper_2606_13426_gb300 import api
    kind = st["kind"]
    if kind == "scores":
        r = api.token_scores(st["logits"], st["tokens"], top_k=st["top_k"], temperature=st["temperature"])
        names = ["logprob", "entropy", "row_max", "log_sum"] + (["top_ids", "top_logprob"] if st["top_k"] else [])
        return {k: r[k] for k in names}
    if kind == "train":
        r = api.token_scores_train(st["logits"], st["tokens"], st["g_logprob"], st["g_entropy"])
        return {k: r[k] for k in ("logprob", "entropy", "d_logits")}
    if kind == "verify":
        r = api.token_verify(st["target"], st["draft"], st["tokens"], mode=st["mode"], temperature=st["temperature"],
                             L_eff=st["L_eff"], coins=st["coins"], race=st["race"])
        return {k: r[k] for k in ("accepted_len", "next_token", "log_ratio")}
    if kind == "append":
        api.cache_append(st["cache"], st["k_new"], st["v_new"], st["pages"], st["lengths"], counts=st["counts"])
        return dict(st["cache"])
    r = api.cache_attend(st["q"], st["cache"], st["pages"], st["lengths"], counts=st["counts"], scale=st["scale"],
                         span=st["span"])
    return dict(out=r["out"], lse=r["lse"])


def run(state):
    if own:
        return _own(state)
    return {"scores": _plain_scores, "train": _plain_train, "verify": _plain_verify, "append": _plain_append,
            "attend": _plain_attend}[state["kind"]](state)


# ------------------------------------------------------------------------------ work
def work(case):
    kind = case["kind"]
    if kind in ("scores", "train"):
        N, V, es = case["N"], case["V"], BYTES[case["dtype"]]
        if kind == "scores":
            return dict(bytes=N * V * es + N * (20 + 8 * case["top_k"]), flops=5 * N * V)
        return dict(bytes=2 * N * V * es + N * 16, flops=10 * N * V)
    if kind == "verify":
        B, L, V, es = case["B"], case["L"], case["V"], BYTES[case["dtype"]]
        steps = L / 2 if case["ragged"] else L        # the windows of a ragged batch are half as long on average
        rows = B * (2 * steps + 1)
        return dict(bytes=rows * V * es + B * V * 4 + B * L * 12, flops=4 * rows * V)
    B, W, H, D = case["B"], case["W"], case["H"], case["D"]
    steps = (W + 1) / 2 if case["ragged"] else W
    if kind == "append":
        return dict(bytes=2 * B * steps * H * D * (BYTES[case["dtype"]] + 1), flops=2 * 2 * B * steps * H * D)
    mean = case["max_len"] * (7 / 12 if case["ragged"] else 1)
    if case["ragged"] and B > 2:
        mean *= (B - 1) / B
    if case["span"]:
        mean = min(mean, case["span"] + steps)
    return dict(bytes=2 * B * mean * H * D + 2 * B * steps * H * case["G"] * D * 2,
                flops=4 * B * mean * steps * H * case["G"] * D)


# ------------------------------------------------------------------------------ 64 bits
def _exact_rows(st, grad):
    x, V, T = st["logits"], st["V"], st.get("temperature", 1.0)
    got = {k: [] for k in ("logprob", "entropy", "row_max", "log_sum", "top_logprob", "d_logits")}
    step = max(1, 20_000_000 // V)
    for r in range(0, st["N"], step):
        z = x[r:r + step].double()
        tok = st["tokens"][r:r + step].long()
        top = z.max(1).values
        lse = torch.logsumexp(z / T, 1)
        logp = z / T - lse[:, None]
        logp[top == -math.inf] = -math.inf
        p = logp.exp()
        plogp = torch.where(p > 0, p * logp, 0.0)
        H = -plogp.sum(1)
        taken = logp.gather(1, tok.clamp(min=0)[:, None])[:, 0]
        got["logprob"].append(torch.where(tok >= 0, taken, 0.0))
        got["entropy"].append(H)
        got["row_max"].append(top)
        got["log_sum"].append(torch.where(top == -math.inf, -math.inf, lse - top / T))
        if st.get("top_k"):
            got["top_logprob"].append(logp.sort(1, descending=True).values[:, : st["top_k"]])
        if grad:
            up = torch.where(tok >= 0, st["g_logprob"][r:r + step].double(), 0.0)
            onehot = torch.zeros_like(p).scatter_(1, tok.clamp(min=0)[:, None], 1.0)
            dx = up[:, None] * (onehot - p)
            if st["g_entropy"] is not None:
                dx -= st["g_entropy"][r:r + step].double()[:, None] * (plogp + p * H[:, None])
            got["d_logits"].append(dx.float() if st["N"] * V > 100_000_000 else dx)
    return {k: torch.cat(v) for k, v in got.items() if v}


def _exact_verify(st):
    B, L, T = st["B"], st["L"], st["temperature"]
    ell = torch.zeros(B, L, dtype=torch.float64)
    for b in range(B):
        n = L if st["L_eff"] is None else int(st["L_eff"][b])
        for j in range(max(n, 0)):
            t = int(st["tokens"][b, j])
            q, p = st["target"][b, j].double() / T, st["draft"][b, j].double() / T
            ell[b, j] = (q[t] - q.logsumexp(0)) - (p[t] - p.logsumexp(0))
    return dict(accepted_len=None, next_token=None, log_ratio=ell.to(DEV))


def _e4m3(x):
    """The nearest e4m3 value (ties to even) of x, |x| < 464, in 64 bits."""
    _, e = torch.frexp(x.abs().clamp(min=2.0 ** -6))
    unit = _power(e - 4)
    return torch.round(x / unit) * unit


def _power(k):
    """2^k in 64 bits, exactly."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _exact_append(st):
    c, block, W = st["cache"], st["block"], st["W"]
    got = dict(k=c["k"].double(), v=c["v"].double(), k_scale=c["k_scale"].double(), v_scale=c["v_scale"].double())
    lengths, pages = st["lengths"].tolist(), st["pages"].tolist()
    counts = [W] * st["B"] if st["counts"] is None else st["counts"].tolist()
    for b in range(st["B"]):
        n, new = lengths[b], counts[b]
        for j in range(n // block, (n + new + block - 1) // block):
            page = pages[b][j]
            lo, hi = max(n, j * block), min(n + new, (j + 1) * block)
            kept = max(0, n - j * block)
            for codes, scales, x, turn in ((got["k"], got["k_scale"], st["k_new"], False), (got["v"], got["v_scale"], st["v_new"], True)):
                y = x[b, lo - n:hi - n].double().transpose(0, 1)                      # [H, tokens, D]
                here = codes[page].transpose(1, 2) if turn else codes[page]
                least = (y.abs().amax((1, 2)) / 448).clamp(min=2.0 ** -126)
                scale = _power(torch.ceil(torch.log2(least)))
                if kept:
                    scale = torch.maximum(scale, scales[page])
                    here[:, :kept] = _e4m3(here[:, :kept] * (scales[page] / scale)[:, None, None])
                here[:, lo - j * block:hi - j * block] = _e4m3(y / scale[:, None, None])
                scales[page] = scale
    return got


def _exact_attend(st):
    c, B, W, H, G, D, block = st["cache"], st["B"], st["W"], st["H"], st["G"], st["D"], st["block"]
    out = torch.zeros(B, W, H * G, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, W, H * G), -math.inf, dtype=torch.float64, device=DEV)
    lengths = st["lengths"].tolist()
    counts = [W] * B if st["counts"] is None else st["counts"].tolist()
    for b in range(B):
        n, new = lengths[b], counts[b]
        if not n or not new:
            continue
        page = st["pages"][b, : (n + block - 1) // block].long()
        for h in range(H):
            k = c["k"].view(torch.uint8)[page, h].view(torch.float8_e4m3fn).double() * c["k_scale"][page, h].double()[:, None, None]
            v = c["v"].view(torch.uint8)[page, h].view(torch.float8_e4m3fn).double() * c["v_scale"][page, h].double()[:, None, None]
            k = k.reshape(-1, D)[:n]
            v = v.transpose(1, 2).reshape(-1, D)[:n]
            for i in range(new):
                end = n - new + i + 1
                lo = max(0, end - st["span"]) if st["span"] else 0
                s = st["scale"] * (st["q"][b, i, h * G:(h + 1) * G].double() @ k[lo:end].T)
                out[b, i, h * G:(h + 1) * G] = torch.softmax(s, 1) @ v[lo:end]
                lse[b, i, h * G:(h + 1) * G] = torch.logsumexp(s, 1)
    return dict(out=out, lse=lse)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "scores":
        r = _exact_rows(st, False)
        if case["top_k"]:
            r["top_ids"] = None
        return r
    if kind == "train":
        r = _exact_rows(st, True)
        return {k: r[k] for k in ("logprob", "entropy", "d_logits")}
    if kind == "verify":
        return _exact_verify(st)
    if kind == "append":
        return _exact_append(st)
    return _exact_attend(st)
