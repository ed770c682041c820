"""Torch-facing helpers over the C ABI: allocate outputs and workspace, pass pointers.

PyTorch provides device memory and the current stream only; every step of the
verification path runs in libspecdiff's kernels.  Inputs must be CUDA tensors
(this module never computes anything itself and has no CPU path).
"""
import functools

import torch

from . import binding as B

_DTYPES = {torch.float32: B.SDV_F32, torch.bfloat16: B.SDV_BF16}
_MODES = {"sample": B.SDV_MODE_SAMPLE, "block": B.SDV_MODE_BLOCK,
          B.SDV_MODE_SAMPLE: B.SDV_MODE_SAMPLE, B.SDV_MODE_BLOCK: B.SDV_MODE_BLOCK}
_TOKEN_DTYPES = {torch.float32: B.SDV_F32, torch.bfloat16: B.SDV_BF16, torch.float16: B.SDV_F16}
_RESIDUALS = {"decomposition": B.SDV_RESIDUAL_DECOMPOSITION,
              "reflection": B.SDV_RESIDUAL_REFLECTION}


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _stream():
    # the handle alone: building a Stream object takes longer than a small call's launch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _need_cuda(*ts):
    for t in ts:
        if t is not None and not (t.is_cuda and t.is_contiguous()):
            raise ValueError("libspecdiff needs contiguous CUDA tensors")


def workspace_bytes(B_, L, d, dtype=torch.float32):
    return B.sdv_workspace_bytes(B_, L, d, _DTYPES[dtype])


def make_workspace(B_, L, d, dtype=torch.float32, device="cuda"):
    """A workspace for calls of up to (B_, L, d) (zeroed, though no call needs that)."""
    return torch.zeros(max(workspace_bytes(B_, L, d, dtype), 256), dtype=torch.uint8, device=device)


def _sigma_args(sigma, Bn, L):
    if sigma.dim() == 1:
        if sigma.shape[0] != L:
            raise ValueError("sigma [L] expected")
        return sigma, 0
    if tuple(sigma.shape) != (Bn, L):
        raise ValueError("sigma [B, L] expected")
    return sigma, L


def verify(x_draft, mu_target, mu_draft, sigma, seed, mode="block", *, L_eff=None,
           mu_target_bonus=None, sigma_bonus=None, residual="decomposition", omega=1.0,
           with_ratios=True, with_aux=False, workspace=None, out=None, pipelined=False):
    """One verification call (sdv_verify_ex) on [B, L, d] CUDA tensors; returns a dict of outputs.

    pipelined=True calls sdv_verify_pipelined instead: the call may overlap the end of the
    previous kernel on the stream (see its preconditions in include/specdiff.h)."""
    _need_cuda(x_draft, mu_target, mu_draft, sigma, L_eff, mu_target_bonus, sigma_bonus)
    Bn, L, d = x_draft.shape
    dt = x_draft.dtype
    if mu_target.dtype != dt or mu_draft.dtype != dt or dt not in _DTYPES:
        raise ValueError("x_draft, mu_target, mu_draft must share a float32/bfloat16 dtype")
    if sigma.dtype != torch.float32:
        raise ValueError("sigma must be float32")
    sigma, sstride = _sigma_args(sigma, Bn, L)
    dev = x_draft.device
    if out is None:
        out = {}
    acc = out.get("accepted_len")
    if acc is None:
        acc = torch.empty(Bn, dtype=torch.int32, device=dev)
    y = out.get("y")
    if y is None:
        y = torch.empty(Bn, d, dtype=dt, device=dev)
    lr = dn = None
    if with_ratios:
        lr = out.get("log_ratio")
        lr = torch.empty(Bn, L, dtype=torch.float32, device=dev) if lr is None else lr
        dn = out.get("delta_norm")
        dn = torch.empty(Bn, L, dtype=torch.float32, device=dev) if dn is None else dn
    st = out.get("status")
    st = torch.empty(Bn, dtype=torch.int32, device=dev) if st is None else st
    aux = None
    if with_aux:
        aux = out.get("aux")
        aux = torch.empty(Bn, 4, dtype=torch.float32, device=dev) if aux is None else aux
    if workspace is None:
        workspace = make_workspace(Bn, L, d, dt, dev)
    # straight to the C entry point (the binding's function of that name has the same arguments)
    B._call("sdv_verify_pipelined" if pipelined else "sdv_verify_ex",
            x_draft.data_ptr(), mu_target.data_ptr(), mu_draft.data_ptr(), sigma.data_ptr(), sstride,
            Bn, L, d, _DTYPES[dt], int(seed) & 0xFFFFFFFFFFFFFFFF, _MODES[mode],
            _ptr(L_eff), _ptr(mu_target_bonus), _ptr(sigma_bonus),
            _RESIDUALS[residual], float(omega),
            acc.data_ptr(), y.data_ptr(), _ptr(lr), _ptr(dn), st.data_ptr(), _ptr(aux),
            workspace.data_ptr(), workspace.numel(), _stream())
    res = dict(accepted_len=acc, y=y, status=st)
    if with_ratios:
        res.update(log_ratio=lr, delta_norm=dn)
    if with_aux:
        res["aux"] = aux
    return res


def verify_host(x_draft, mu_target, mu_draft, sigma, seed, mode="block", *, dev_bufs=None):
    """End-to-end call from pinned host tensors: copy in, verify, copy accepted_len and y back.

    ``dev_bufs`` (from ``make_device_buffers``) holds the device copies and
    outputs so repeated calls allocate nothing.  Returns (accepted_len, y) as
    host tensors, synchronised.
    """
    Bn, L, d = x_draft.shape
    if dev_bufs is None:
        dev_bufs = make_device_buffers(Bn, L, d, x_draft.dtype, sigma.shape)
    db = dev_bufs
    db["x"].copy_(x_draft, non_blocking=True)
    db["mq"].copy_(mu_target, non_blocking=True)
    db["mp"].copy_(mu_draft, non_blocking=True)
    db["sigma"].copy_(sigma, non_blocking=True)
    verify(db["x"], db["mq"], db["mp"], db["sigma"], seed, mode, with_ratios=False,
           workspace=db["ws"], out=db)
    db["h_acc"].copy_(db["accepted_len"], non_blocking=True)
    db["h_y"].copy_(db["y"], non_blocking=True)
    torch.cuda.current_stream().synchronize()
    return db["h_acc"], db["h_y"]


class HostStream:
    """End-to-end verification of a sequence of windows held in pinned host memory.

    Each window is one pinned host tensor [3, B, L, d] (x_draft, mu_target, mu_draft
    stacked, so that it crosses to the device in one copy) plus sigma.  ``depth`` device
    slots are used in turn: the copy of a window into its slot (on a copy stream)
    overlaps the verification of the previous one (on a compute stream), and each slot's
    accepted lengths and states come back to pinned host memory on the compute stream.
    ``submit`` returns the slot index; ``result`` waits for that slot and returns its
    host tensors (valid until the slot is submitted again).  torch only allocates
    memory and supplies the streams and events; the verification runs in libspecdiff.
    """

    def __init__(self, Bn, L, d, dtype=torch.float32, sigma_shape=None, depth=2, device="cuda"):
        self.Bn, self.L, self.d, self.depth = Bn, L, d, depth
        sigma_shape = (Bn, L) if sigma_shape is None else tuple(sigma_shape)
        self.copy_stream = torch.cuda.Stream(device=device)
        self.compute_stream = torch.cuda.Stream(device=device)
        self.ws = torch.zeros(max(workspace_bytes(Bn, L, d, dtype), 256), dtype=torch.uint8, device=device)
        self.slots = []
        for _ in range(depth):
            self.slots.append(dict(
                win=torch.empty(3, Bn, L, d, dtype=dtype, device=device),
                sigma=torch.empty(*sigma_shape, dtype=torch.float32, device=device),
                accepted_len=torch.empty(Bn, dtype=torch.int32, device=device),
                y=torch.empty(Bn, d, dtype=dtype, device=device),
                status=torch.empty(Bn, dtype=torch.int32, device=device),
                h_acc=torch.empty(Bn, dtype=torch.int32, pin_memory=True),
                h_y=torch.empty(Bn, d, dtype=dtype, pin_memory=True),
                copied=torch.cuda.Event(), done=torch.cuda.Event(), busy=False))
        self.next = 0

    def submit(self, window, sigma, seed, mode="block"):
        i = self.next
        self.next = (i + 1) % self.depth
        sl = self.slots[i]
        if sl["busy"]:
            self.copy_stream.wait_event(sl["done"])      # the slot's previous window is verified
        with torch.cuda.stream(self.copy_stream):
            sl["win"].copy_(window, non_blocking=True)
            sl["sigma"].copy_(sigma, non_blocking=True)
            sl["copied"].record(self.copy_stream)
        self.compute_stream.wait_event(sl["copied"])
        with torch.cuda.stream(self.compute_stream):
            w = sl["win"]
            verify(w[0], w[1], w[2], sl["sigma"], seed, mode, with_ratios=False, workspace=self.ws, out=sl)
            sl["h_acc"].copy_(sl["accepted_len"], non_blocking=True)
            sl["h_y"].copy_(sl["y"], non_blocking=True)
            sl["done"].record(self.compute_stream)
        sl["busy"] = True
        return i

    def result(self, i):
        sl = self.slots[i]
        sl["done"].synchronize()
        return sl["h_acc"], sl["h_y"]


def make_device_buffers(Bn, L, d, dtype, sigma_shape, device="cuda"):
    return dict(
        x=torch.empty(Bn, L, d, dtype=dtype, device=device),
        mq=torch.empty(Bn, L, d, dtype=dtype, device=device),
        mp=torch.empty(Bn, L, d, dtype=dtype, device=device),
        sigma=torch.empty(*sigma_shape, dtype=torch.float32, device=device),
        accepted_len=torch.empty(Bn, dtype=torch.int32, device=device),
        y=torch.empty(Bn, d, dtype=dtype, device=device),
        status=torch.empty(Bn, dtype=torch.int32, device=device),
        ws=make_workspace(Bn, L, d, dtype, device),
        h_acc=torch.empty(Bn, dtype=torch.int32, pin_memory=True),
        h_y=torch.empty(Bn, d, dtype=dtype, pin_memory=True),
    )


def log_ratios(x_draft, mu_target, mu_draft, sigma, L_eff=None, workspace=None):
    """ell_j and |Delta_j| only (sdv_log_ratios)."""
    _need_cuda(x_draft, mu_target, mu_draft, sigma, L_eff)
    Bn, L, d = x_draft.shape
    sigma, sstride = _sigma_args(sigma, Bn, L)
    lr = torch.empty(Bn, L, dtype=torch.float32, device=x_draft.device)
    dn = torch.empty_like(lr)
    if workspace is None:
        workspace = make_workspace(Bn, L, d, x_draft.dtype, x_draft.device)
    B.sdv_log_ratios(_ptr(x_draft), _ptr(mu_target), _ptr(mu_draft), _ptr(sigma), sstride,
                     Bn, L, d, _DTYPES[x_draft.dtype], _ptr(L_eff), _ptr(lr), _ptr(dn),
                     _ptr(workspace), workspace.numel(), _stream())
    return lr, dn


def accept_scan(log_ratio, delta_norm, seed, mode="block", L_eff=None, omega=1.0):
    """tau and log alpha_{tau-1} from given ell, |Delta| (sdv_accept_scan)."""
    _need_cuda(log_ratio, delta_norm, L_eff)
    Bn, L = log_ratio.shape
    tau = torch.empty(Bn, dtype=torch.int32, device=log_ratio.device)
    la = torch.empty(Bn, dtype=torch.float32, device=log_ratio.device)
    B.sdv_accept_scan(_ptr(log_ratio), _ptr(delta_norm), Bn, L, _ptr(L_eff),
                      int(seed) & 0xFFFFFFFFFFFFFFFF, _MODES[mode], float(omega),
                      _ptr(tau), _ptr(la), _stream())
    return tau, la


def usample(delta_norm, log_alpha, w_bits):
    """U = Psi_alpha^{-1}(w) for each item (sdv_usample); w_bits is int32 holding uint32 words."""
    _need_cuda(delta_norm, log_alpha, w_bits)
    n = delta_norm.numel()
    U = torch.empty(n, dtype=torch.float32, device=delta_norm.device)
    st = torch.empty(n, dtype=torch.int32, device=delta_norm.device)
    B.sdv_usample(_ptr(delta_norm), _ptr(log_alpha), _ptr(w_bits), n, _ptr(U), _ptr(st), _stream())
    return U, st


def philox(ctr, seed):
    """Raw Philox4x32-10 blocks for counters ctr [n, 4] (int32 holding uint32 words)."""
    _need_cuda(ctr)
    out = torch.empty_like(ctr)
    B.sdv_philox(_ptr(ctr), int(seed) & 0xFFFFFFFFFFFFFFFF, ctr.shape[0], _ptr(out), _stream())
    return out


def normals(seed, Bn, d, stream_id, sub=0, device="cuda"):
    out = torch.empty(Bn, d, dtype=torch.float32, device=device)
    B.sdv_normals(int(seed) & 0xFFFFFFFFFFFFFFFF, Bn, d, stream_id, sub, _ptr(out), _stream())
    return out


def special(which, z):
    """The device special functions (sdv_special): 'erfcx', 'log_ndtr' or 'gprime' at z (fp32)."""
    _need_cuda(z)
    out = torch.empty_like(z)
    B.sdv_special({"erfcx": 0, "log_ndtr": 1, "gprime": 2}[which], _ptr(z), z.numel(), _ptr(out), _stream())
    return out


class GmmTarget:
    """Analytic Gaussian-mixture target and its variance-preserving schedule (device copies)."""

    def __init__(self, means, log_weights, comp_var, K, churn, beta_min=0.1, beta_max=20.0,
                 t_floor=1e-4, device="cuda"):
        self.means = torch.as_tensor(means, dtype=torch.float32).to(device).contiguous()
        self.log_weights = torch.as_tensor(log_weights, dtype=torch.float32).to(device).contiguous()
        self.C, self.d = self.means.shape
        self.comp_var = float(comp_var)
        self.K = int(K)
        self.churn = float(churn)
        self.beta_min, self.beta_max, self.t_floor = float(beta_min), float(beta_max), float(t_floor)

    def sched(self):
        return (self.K, self.churn, self.beta_min, self.beta_max, self.t_floor)

    def params(self):
        return (_ptr(self.means), _ptr(self.log_weights), self.C, self.comp_var) + self.sched()


def gmm_target(states, k, target):
    """m^q_k(state) and the score for rows of states [n, d] (sdv_gmm_target)."""
    _need_cuda(states, k)
    n, d = states.shape
    mq = torch.empty_like(states)
    sc = torch.empty_like(states)
    B.sdv_gmm_target(_ptr(states), _ptr(k), n, d, *target.params(), _ptr(mq), _ptr(sc), _stream())
    return mq, sc


def free_draft(y, score, k, L_eff, L, target, seed):
    """The drafter's gamma_b steps (sdv_free_draft): x_draft, mu_draft [B, L, d], sigma [B, L]."""
    _need_cuda(y, score, k, L_eff)
    Bn, d = y.shape
    x = torch.zeros(Bn, L, d, dtype=torch.float32, device=y.device)
    mp = torch.zeros_like(x)
    sg = torch.zeros(Bn, L, dtype=torch.float32, device=y.device)
    B.sdv_free_draft(_ptr(y), _ptr(score), _ptr(k), _ptr(L_eff), Bn, L, d, *target.sched(),
                     int(seed) & 0xFFFFFFFFFFFFFFFF, _ptr(x), _ptr(mp), _ptr(sg), _stream())
    return x, mp, sg


def sampler_run(Bn, L, target, seed, mode="block", drafter="free", max_rounds=None,
                workspace=None):
    """Speculative sampling of Bn chains to step K (sdv_sampler_run); returns a dict."""
    dev = target.means.device
    d = target.d
    if workspace is None:
        workspace = torch.empty(B.sdv_sampler_workspace_bytes(Bn, L, d), dtype=torch.uint8,
                                device=dev)
    y = torch.empty(Bn, d, dtype=torch.float32, device=dev)
    k = torch.empty(Bn, dtype=torch.int32, device=dev)
    cr = torch.empty(Bn, dtype=torch.int32, device=dev)
    ts = torch.empty(Bn, dtype=torch.int32, device=dev)
    dr = {"free": B.SDV_DRAFTER_FREE, "frozen": B.SDV_DRAFTER_FROZEN}[drafter]
    mr = target.K if max_rounds is None else int(max_rounds)
    rounds = B.sdv_sampler_run(Bn, L, d, *target.params(), int(seed) & 0xFFFFFFFFFFFFFFFF,
                               _MODES[mode], dr, mr, _ptr(y), _ptr(k), _ptr(cr), _ptr(ts),
                               _ptr(workspace), workspace.numel(), _stream())
    return dict(y=y, k=k, chain_rounds=cr, tau_sum=ts, rounds=rounds)


def sampler_rounds(Bn, L, target, seed, rounds, mode="block", drafter="free", workspace=None):
    """The same sampler driven from the host: sdv_sampler_begin, `rounds` calls of
    sdv_sampler_round, sdv_sampler_end; returns the dict of sampler_run."""
    dev = target.means.device
    d = target.d
    if workspace is None:
        workspace = torch.empty(B.sdv_sampler_workspace_bytes(Bn, L, d), dtype=torch.uint8,
                                device=dev)
    y = torch.empty(Bn, d, dtype=torch.float32, device=dev)
    k = torch.empty(Bn, dtype=torch.int32, device=dev)
    cr = torch.empty(Bn, dtype=torch.int32, device=dev)
    ts = torch.empty(Bn, dtype=torch.int32, device=dev)
    dr = {"free": B.SDV_DRAFTER_FREE, "frozen": B.SDV_DRAFTER_FROZEN}[drafter]
    sd = int(seed) & 0xFFFFFFFFFFFFFFFF
    ws, nb, st = _ptr(workspace), workspace.numel(), _stream()
    B.sdv_sampler_begin(Bn, L, d, *target.params(), sd, ws, nb, st)
    for _ in range(int(rounds)):
        B.sdv_sampler_round(Bn, L, d, *target.params(), sd, _MODES[mode], dr, ws, nb, st)
    r = B.sdv_sampler_end(Bn, L, d, ws, nb, _ptr(y), _ptr(k), _ptr(cr), _ptr(ts), st)
    return dict(y=y, k=k, chain_rounds=cr, tau_sum=ts, rounds=r)


def em_sample(Bn, target, seed):
    """The plain Euler-Maruyama chain (sdv_em_sample)."""
    y = torch.empty(Bn, target.d, dtype=torch.float32, device=target.means.device)
    B.sdv_em_sample(Bn, target.d, *target.params(), int(seed) & 0xFFFFFFFFFFFFFFFF, _ptr(y),
                    _stream())
    return y


# ---- speculative decoding over tokens: scores, verification, 8-bit cache


def _dense(what, t, dtype, shape):
    """A contiguous CUDA tensor of the type and shape, or None."""
    if t is not None and not (t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous()):
        raise ValueError("%s: a contiguous CUDA %s tensor of shape %s expected" % (what, dtype, tuple(shape)))


def _out(out, name, shape, dtype, dev):
    t = out.get(name) if out else None
    if t is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    _dense(name, t, dtype, shape)
    return t


def _outs(out, names, n, dtype, dev):
    """Outputs [n] of one type by name: the caller's, or new ones (an allocation takes 1.5 us here, a
    view of one more)."""
    if not out:
        return {k: torch.empty(n, dtype=dtype, device=dev) for k in names}
    return {k: _out(out, k, (n,), dtype, dev) for k in names}


def _workspace(t, need, dev):
    """A workspace of `need` bytes: the caller's (whose size the entry point checks), or a new one."""
    if t is None:
        return torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    _need_cuda(t)
    return t


@functools.lru_cache(maxsize=1024)
def _verify_workspace(Bn, L):
    return B.sdv_token_verify_workspace_bytes(Bn, L)


@functools.lru_cache(maxsize=1024)
def _attend_workspace(device, *sizes):
    """The size depends on the current device's SMs too, which `device` stands for."""
    return B.sdv_attend_workspace_bytes(*sizes)


def _rows(what, t, dims):
    """A CUDA tensor of logits (or keys, queries) whose last axis is contiguous; its type's code."""
    dt = _TOKEN_DTYPES.get(t.dtype)
    if dt is None or not t.is_cuda or t.dim() != dims or t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError("%s: a %d-d CUDA float32/bfloat16/float16 tensor with a contiguous last axis expected" % (what, dims))
    return dt


def _row_stride(t):
    """Elements between rows of [..., N, V] (rows of a single one may be anywhere)."""
    return t.stride(-2) if t.shape[-2] > 1 else max(t.stride(-2), t.shape[-1])


def token_scores(logits, tokens=None, *, top_k=0, temperature=1.0, entropy=True, with_status=False, out=None):
    """Log probabilities of given tokens, entropy and top alternatives of logits [N, V]
    (sdv_token_scores); returns a dict: logprob [N] (with tokens [N] int32, -1 for none), entropy
    [N], row_max, log_sum [N], status [N] if wanted, and top_ids, top_logprob [N, top_k]."""
    dt = _rows("logits", logits, 2)
    N, V = logits.shape
    dev, f32 = logits.device, torch.float32
    _dense("tokens", tokens, torch.int32, (N,))
    names = ("row_max", "log_sum") + (("logprob",) if tokens is not None else ()) + (("entropy",) if entropy else ())
    r = _outs(out, names, N, f32, dev)
    if with_status:
        r["status"] = _out(out, "status", (N,), torch.int32, dev)
    if top_k:
        r["top_ids"] = _out(out, "top_ids", (N, top_k), torch.int32, dev)
        r["top_logprob"] = _out(out, "top_logprob", (N, top_k), f32, dev)
    B._call("sdv_token_scores", logits.data_ptr(), _row_stride(logits), N, V, dt, _ptr(tokens), float(temperature), int(top_k),
            _ptr(r.get("logprob")), _ptr(r.get("entropy")), r["row_max"].data_ptr(), r["log_sum"].data_ptr(),
            _ptr(r.get("top_ids")), _ptr(r.get("top_logprob")), _ptr(r.get("status")), _stream())
    return r


def _grad_like(logits, d_logits):
    """The gradient's tensor: rows laid out as the logits' where they are (nearly) dense, so that
    both meet 16-byte boundaries at the same places."""
    N, V = logits.shape
    if d_logits is None:
        st = _row_stride(logits)
        if V < st <= V + 128:
            return torch.empty(N, st, dtype=logits.dtype, device=logits.device)[:, :V]
        return torch.empty(N, V, dtype=logits.dtype, device=logits.device)
    if not d_logits.is_cuda or d_logits.dtype != logits.dtype or d_logits.shape != logits.shape or d_logits.stride(1) != 1 and V > 1:
        raise ValueError("d_logits: a CUDA tensor of the logits' type and shape with a contiguous last axis expected")
    return d_logits


def token_scores_grad(logits, tokens, scores, g_logprob=None, g_entropy=None, *, temperature=1.0, d_logits=None):
    """The gradient of sum g_logprob logprob + g_entropy entropy with respect to the logits, from
    the dict of token_scores (sdv_token_scores_grad); d_logits may be the logits themselves."""
    dt = _rows("logits", logits, 2)
    N, V = logits.shape
    _dense("tokens", tokens, torch.int32, (N,))
    for what, t in (("g_logprob", g_logprob), ("g_entropy", g_entropy), ("row_max", scores["row_max"]),
                    ("log_sum", scores["log_sum"]), ("entropy", scores.get("entropy"))):
        _dense(what, t, torch.float32, (N,))
    dx = _grad_like(logits, d_logits)
    B._call("sdv_token_scores_grad", logits.data_ptr(), _row_stride(logits), N, V, dt,
            _ptr(tokens) if g_logprob is not None else 0, float(temperature), scores["row_max"].data_ptr(),
            scores["log_sum"].data_ptr(), _ptr(scores.get("entropy")), _ptr(g_logprob), _ptr(g_entropy), dx.data_ptr(),
            _row_stride(dx), _stream())
    return dx


def token_scores_train(logits, tokens, g_logprob=None, g_entropy=None, *, temperature=1.0, d_logits=None,
                       with_status=False, out=None):
    """Scores and gradient in one call that reads the logits once (sdv_token_scores_train);
    returns the dict of token_scores with d_logits."""
    dt = _rows("logits", logits, 2)
    N, V = logits.shape
    dev, f32 = logits.device, torch.float32
    _dense("tokens", tokens, torch.int32, (N,))
    _dense("g_logprob", g_logprob, f32, (N,))
    _dense("g_entropy", g_entropy, f32, (N,))
    r = _outs(out, ("entropy", "row_max", "log_sum") + (("logprob",) if tokens is not None else ()), N, f32, dev)
    if with_status:
        r["status"] = _out(out, "status", (N,), torch.int32, dev)
    r["d_logits"] = dx = _grad_like(logits, d_logits)
    B._call("sdv_token_scores_train", logits.data_ptr(), _row_stride(logits), N, V, dt, _ptr(tokens), float(temperature),
            _ptr(g_logprob), _ptr(g_entropy), _ptr(r.get("logprob")), r["entropy"].data_ptr(), r["row_max"].data_ptr(),
            r["log_sum"].data_ptr(), _ptr(r.get("status")), dx.data_ptr(), _row_stride(dx), _stream())
    return r


def token_verify(target_logits, draft_logits, tokens, seed=0, mode="block", *, L_eff=None, temperature=1.0,
                 draft_temperature=None, coins=None, race=None, with_status=False, workspace=None, out=None):
    """Verification of drafted tokens [B, L] from target logits [B, L + 1, V] and draft logits
    [B, L, V] (sdv_token_verify); returns accepted_len, next_token [B], log_ratio [B, L], and
    status [B] if wanted.  draft_temperature defaults to temperature; coins [B, L] and race [B, V] (exponential
    variates) replace the draws from `seed`."""
    dt = _rows("target_logits", target_logits, 3)
    if _rows("draft_logits", draft_logits, 3) != dt:
        raise ValueError("target_logits and draft_logits must share a type")
    Bn, L, V = draft_logits.shape
    if tuple(target_logits.shape) != (Bn, L + 1, V):
        raise ValueError("target_logits [B, L + 1, V] expected")
    i32, f32, dev = torch.int32, torch.float32, target_logits.device
    _dense("tokens", tokens, i32, (Bn, L))
    _dense("L_eff", L_eff, i32, (Bn,))
    _dense("coins", coins, f32, (Bn, L))
    _dense("race", race, f32, (Bn, V))
    r = _outs(out, ("accepted_len", "next_token", "status") if with_status else ("accepted_len", "next_token"), Bn, i32, dev)
    r["log_ratio"] = _out(out, "log_ratio", (Bn, L), f32, dev)
    workspace = _workspace(workspace, _verify_workspace(Bn, L), dev)
    B._call("sdv_token_verify", target_logits.data_ptr(), target_logits.stride(0), _row_stride(target_logits),
            draft_logits.data_ptr(), draft_logits.stride(0), _row_stride(draft_logits), tokens.data_ptr(), Bn, L, V, dt,
            float(temperature), float(temperature if draft_temperature is None else draft_temperature), _MODES[mode],
            _ptr(L_eff), int(seed) & 0xFFFFFFFFFFFFFFFF, _ptr(coins), _ptr(race), r["accepted_len"].data_ptr(),
            r["next_token"].data_ptr(), r["log_ratio"].data_ptr(), _ptr(r.get("status")), workspace.data_ptr(),
            workspace.numel(), _stream())
    return r


def make_token_cache(pages, heads, block, dim, device="cuda"):
    """An empty 8-bit cache: codes k [pages, heads, block, dim] and v [pages, heads, dim, block]
    (float8_e4m3fn), k_scale and v_scale [pages, heads]."""
    f8 = torch.float8_e4m3fn
    return dict(k=torch.zeros(pages, heads, block, dim, dtype=torch.uint8, device=device).view(f8),
                v=torch.zeros(pages, heads, dim, block, dtype=torch.uint8, device=device).view(f8),
                k_scale=torch.ones(pages, heads, dtype=torch.float32, device=device),
                v_scale=torch.ones(pages, heads, dtype=torch.float32, device=device))


def _cache_args(cache, page_table, lengths, counts):
    k = cache["k"]
    P, H, block, D = k.shape
    f8 = torch.float8_e4m3fn
    _dense("cache k", k, f8, (P, H, block, D))
    _dense("cache v", cache["v"], f8, (P, H, D, block))
    _dense("cache k_scale", cache["k_scale"], torch.float32, (P, H))
    _dense("cache v_scale", cache["v_scale"], torch.float32, (P, H))
    Bn, M = page_table.shape
    _dense("page_table", page_table, torch.int32, (Bn, M))
    _dense("lengths", lengths, torch.int32, (Bn,))
    _dense("counts", counts, torch.int32, (Bn,))
    return P, H, block, D, Bn, M


def _same_layout(a, b):
    """One shape, and one stride along every axis of more than one place."""
    if a.shape != b.shape:
        return False
    s, t = a.stride(), b.stride()
    return s == t or all(x == y or n == 1 for n, x, y in zip(a.shape, s, t))


def cache_append(cache, k_new, v_new, page_table, lengths, *, counts=None, status=None):
    """Appends k_new, v_new [B, W, H, D] behind the lengths [B] tokens that the cache holds of each
    sequence (sdv_cache_append); status [B] int32 gets bits added to it."""
    P, H, block, D, Bn, M = _cache_args(cache, page_table, lengths, counts)
    dt = _rows("k_new", k_new, 4)
    W = k_new.shape[1]
    if tuple(k_new.shape) != (Bn, W, H, D) or v_new.dtype != k_new.dtype or not v_new.is_cuda or not _same_layout(k_new, v_new):
        raise ValueError("k_new and v_new: [B, W, heads, dim] of one type and layout expected")
    _dense("status", status, torch.int32, (Bn,))
    B._call("sdv_cache_append", k_new.data_ptr(), v_new.data_ptr(), k_new.stride(0), k_new.stride(1), k_new.stride(2), dt, Bn, W, H,
            D, block, cache["k"].data_ptr(), cache["v"].data_ptr(), cache["k_scale"].data_ptr(), cache["v_scale"].data_ptr(), P,
            page_table.data_ptr(), M, lengths.data_ptr(), _ptr(counts), _ptr(status), _stream())


def cache_attend(q, cache, page_table, lengths, *, counts=None, scale=None, span=0, status=None, workspace=None, out=None):
    """Attention of the window q [B, W, Hq, D], whose tokens are the last ones of the cache, over
    the lengths [B] tokens that it holds (sdv_cache_attend); returns out [B, W, Hq, D] and lse
    [B, W, Hq].  scale defaults to D^-1/2."""
    P, H, block, D, Bn, M = _cache_args(cache, page_table, lengths, counts)
    dt = _rows("q", q, 4)
    W, Hq = q.shape[1], q.shape[2]
    if tuple(q.shape) != (Bn, W, Hq, D):
        raise ValueError("q: [B, W, query heads, dim] expected")
    _dense("status", status, torch.int32, (Bn,))
    dev = q.device
    r = dict(out=_out(out, "out", (Bn, W, Hq, D), q.dtype, dev), lse=_out(out, "lse", (Bn, W, Hq), torch.float32, dev))
    workspace = _workspace(workspace, _attend_workspace(torch.cuda.current_device(), Bn, W, Hq, H, D), dev)
    B._call("sdv_cache_attend", q.data_ptr(), q.stride(0), q.stride(1), q.stride(2), dt, Bn, W, Hq, H, D, block,
            cache["k"].data_ptr(), cache["v"].data_ptr(), cache["k_scale"].data_ptr(), cache["v_scale"].data_ptr(), P,
            page_table.data_ptr(), M, lengths.data_ptr(), _ptr(counts), float(D ** -0.5 if scale is None else scale), int(span),
            r["out"].data_ptr(), r["lse"].data_ptr(), _ptr(status), workspace.data_ptr(), workspace.numel(), _stream())
    return r


# ---- speculative decoding with trees of drafted tokens


@functools.lru_cache(maxsize=1024)
def _tree_attend_workspace(device, *sizes):
    """The size depends on the current device's SMs too, which `device` stands for."""
    return B.sdv_tree_attend_workspace_bytes(*sizes)


def _here(*ts):
    """All on the current device, whose stream the call goes to."""
    dev = torch.cuda.current_device()
    for t in ts:
        if t is not None and t.get_device() != dev:
            raise ValueError("a tensor on cuda:%d, the current device, expected (got %s)" % (dev, t.device))


def _cache_here(cache, *ts):
    _here(cache["k"], cache["v"], cache["k_scale"], cache["v_scale"], *ts)


def rotary_freqs(rot, base=10000.0, device="cuda"):
    """Radians a position of the pairs of a head's first `rot` elements, base^(-2 i / rot), float64
    [rot / 2], as cache_append_rotary takes them; scaled variants are the caller's own tensor."""
    if rot < 2 or rot % 2:
        raise ValueError("rot: an even number of elements expected")
    return float(base) ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)


def cache_append_rotary(cache, k_new, v_new, page_table, lengths, freqs, *, pairs="halves", q=None, positions=None,
                        counts=None, status=None, out=None):
    """cache_append with the keys turned by their positions on the way (sdv_cache_append_rotary): positions
    [B, W] int32, by default lengths[b] + i (a tree's nodes take lengths[b] + depth); freqs [rot / 2] float64
    (rotary_freqs); pairs "halves" (i, i + rot / 2) or "neighbours" (2 i, 2 i + 1).  q [B, W, Hq, D] is
    turned too and returned as a new tensor, or in `out`, which may be q itself."""
    P, H, block, D, Bn, M = _cache_args(cache, page_table, lengths, counts)
    dt = _rows("k_new", k_new, 4)
    W = k_new.shape[1]
    if tuple(k_new.shape) != (Bn, W, H, D) or v_new.dtype != k_new.dtype or not v_new.is_cuda or not _same_layout(k_new, v_new):
        raise ValueError("k_new and v_new: [B, W, heads, dim] of one type and layout expected")
    if pairs not in ("halves", "neighbours"):
        raise ValueError("pairs: \"halves\" or \"neighbours\" expected")
    _dense("freqs", freqs, torch.float64, (freqs.numel(),))
    _dense("positions", positions, torch.int32, (Bn, W))
    _dense("status", status, torch.int32, (Bn,))
    Hq, qs, os_ = 0, (0, 0, 0), (0, 0, 0)
    if q is not None:
        if _rows("q", q, 4) != dt or tuple(q.shape) != (Bn, W, q.shape[2], D):
            raise ValueError("q: [B, W, query heads, dim] of the keys' type expected")
        Hq, qs = q.shape[2], q.stride()[:3]
        if out is None:
            out = torch.empty((Bn, W, Hq, D), dtype=q.dtype, device=q.device)
        elif _rows("out", out, 4) != dt or out.shape != q.shape:
            raise ValueError("out: a tensor like q expected")
        os_ = out.stride()[:3]
        if out.data_ptr() == q.data_ptr():
            if not _same_layout(q, out):
                raise ValueError("out: q itself or a tensor apart from it expected")
            os_ = qs
    elif out is not None:
        raise ValueError("out without q")
    _cache_here(cache, k_new, v_new, page_table, lengths, freqs, q, out, positions, counts, status)
    B._call("sdv_cache_append_rotary", k_new.data_ptr(), v_new.data_ptr(), k_new.stride(0), k_new.stride(1), k_new.stride(2),
            _ptr(q), qs[0], qs[1], qs[2], _ptr(out), os_[0], os_[1], os_[2], dt, Bn, W, Hq, H, D, block, freqs.data_ptr(),
            2 * freqs.numel(), int(pairs == "halves"), _ptr(positions), cache["k"].data_ptr(), cache["v"].data_ptr(),
            cache["k_scale"].data_ptr(), cache["v_scale"].data_ptr(), P, page_table.data_ptr(), M, lengths.data_ptr(), _ptr(counts),
            _ptr(status), _stream())
    return out


def tree_attend(q, cache, page_table, lengths, parents, *, counts=None, scale=None, status=None, workspace=None, out=None):
    """Attention of a drafted tree's nodes q [B, W, Hq, D], whose tokens are the last ones of the cache, each over
    the tokens before the tree, its ancestors and itself (sdv_tree_attend); parents [B, W] int32 (-1 for a
    root).  lengths [B] count the nodes too.  Returns out [B, W, Hq, D] and lse [B, W, Hq].  scale defaults to D^-1/2.  Outputs
    that a kernel gave up on (SDV_STATUS_STUCK) are NaN."""
    P, H, block, D, Bn, M = _cache_args(cache, page_table, lengths, counts)
    dt = _rows("q", q, 4)
    W, Hq = q.shape[1], q.shape[2]
    if tuple(q.shape) != (Bn, W, Hq, D):
        raise ValueError("q: [B, W, query heads, dim] expected")
    _dense("parents", parents, torch.int32, (Bn, W))
    _dense("status", status, torch.int32, (Bn,))
    dev = q.device
    r = dict(out=_out(out, "out", (Bn, W, Hq, D), q.dtype, dev), lse=_out(out, "lse", (Bn, W, Hq), torch.float32, dev))
    _cache_here(cache, q, page_table, lengths, parents, counts, status, r["out"], r["lse"], workspace)
    workspace = _workspace(workspace, _tree_attend_workspace(torch.cuda.current_device(), Bn, W, Hq, H, D), dev)
    B._call("sdv_tree_attend", q.data_ptr(), q.stride(0), q.stride(1), q.stride(2), dt, Bn, W, Hq, H, D, block,
            cache["k"].data_ptr(), cache["v"].data_ptr(), cache["k_scale"].data_ptr(), cache["v_scale"].data_ptr(), P,
            page_table.data_ptr(), M, lengths.data_ptr(), parents.data_ptr(), _ptr(counts), float(D ** -0.5 if scale is None else scale),
            r["out"].data_ptr(), r["lse"].data_ptr(), _ptr(status), workspace.data_ptr(), workspace.numel(), _stream())
    return r


def tree_verify(target_logits, draft_logits, tokens, parents, seed=0, *, counts=None, temperature=1.0, draft_temperature=None,
                coins=None, race=None, with_status=False, out=None):
    """Verification of drafted trees: tokens, parents [B, W], target and draft logits [B, W, V] of their nodes
    (sdv_tree_verify).  The children of a node were drawn from its draft logits; with draft_logits None they
    were chosen without chance.  Returns accepted_len [B], path [B, W] (the nodes taken from the root on, -1
    behind them, as cache_keep takes it), next_token [B], log_ratio [B, W], and status [B] if wanted."""
    dt = _rows("target_logits", target_logits, 3)
    Bn, W, V = target_logits.shape
    if draft_logits is not None and (_rows("draft_logits", draft_logits, 3) != dt or draft_logits.shape != target_logits.shape):
        raise ValueError("draft_logits: a tensor of the target's type and shape expected")
    i32, f32, dev = torch.int32, torch.float32, target_logits.device
    _dense("tokens", tokens, i32, (Bn, W))
    _dense("parents", parents, i32, (Bn, W))
    _dense("counts", counts, i32, (Bn,))
    _dense("coins", coins, f32, (Bn, W))
    _dense("race", race, f32, (Bn, V))
    r = _outs(out, ("accepted_len", "next_token", "status") if with_status else ("accepted_len", "next_token"), Bn, i32, dev)
    r["path"] = _out(out, "path", (Bn, W), i32, dev)
    r["log_ratio"] = _out(out, "log_ratio", (Bn, W), f32, dev)
    _here(target_logits, draft_logits, tokens, parents, counts, coins, race, *r.values())
    db, dr = (0, V) if draft_logits is None else (draft_logits.stride(0), _row_stride(draft_logits))
    B._call("sdv_tree_verify", target_logits.data_ptr(), target_logits.stride(0), _row_stride(target_logits), _ptr(draft_logits), db,
            dr, tokens.data_ptr(), parents.data_ptr(), Bn, W, V, dt, float(temperature),
            float(temperature if draft_temperature is None else draft_temperature), _ptr(counts), int(seed) & 0xFFFFFFFFFFFFFFFF,
            _ptr(coins), _ptr(race), r["accepted_len"].data_ptr(), r["path"].data_ptr(), r["next_token"].data_ptr(),
            r["log_ratio"].data_ptr(), _ptr(r.get("status")), _stream())
    return r


def cache_keep(cache, path, page_table, lengths, *, status=None):
    """Moves the rows of accepted paths [B, W] (tree_verify's) to the places behind the lengths [B] tokens that
    the cache held before the trees (sdv_cache_keep); status [B] int32 gets bits added to it."""
    P, H, block, D, Bn, M = _cache_args(cache, page_table, lengths, None)
    W = path.shape[-1]
    _dense("path", path, torch.int32, (Bn, W))
    _dense("status", status, torch.int32, (Bn,))
    _cache_here(cache, path, page_table, lengths, status)
    B._call("sdv_cache_keep", path.data_ptr(), Bn, W, H, D, block, cache["k"].data_ptr(), cache["v"].data_ptr(),
            cache["k_scale"].data_ptr(), cache["v_scale"].data_ptr(), P, page_table.data_ptr(), M, lengths.data_ptr(), _ptr(status),
            _stream())
