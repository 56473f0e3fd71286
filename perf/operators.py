"""Performance cases of the operators around the top-K distillation loss.

Five kinds of pass, each as a user's program makes it through the package's
public calls:

  topk      the K largest logits of each row, as the loss takes them
            (topk_entries)
  write     the same selection written to the teacher cache (12-bit codes and
            a scale per row) and read back (teacher_cache_write, _read)
  read      a training batch's rows gathered from a teacher cache
            (teacher_cache_read)
  ckpt      hidden states to 8-bit checkpoints and back (checkpoint_write,
            checkpoint_read)
  train     loss and gradients of a training step that keeps its hidden states
            in 8 bits between forward and backward (topk_kl_loss)
  verify    drafted tokens against the target's probabilities (verify_draft)

With `own` false a pass is computed in elementary torch operations instead.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CODE_MAX = 4094      # cache codes 0..4094; 4095 = no entry
REACH = 1024.0       # entries further below the row's largest are not kept


# ------------------------------------------------------------------ cases --
def listed():
    return [
        # one decoded position of a teacher that runs beside the student: the
        # target of an online distillation step, latency
        dict(name="topk_token", op="topk", dtype="f32", N=1, V=131072, K=100, pad=0,
             logprobs=False, masked=0.0),
        # a short ragged batch of a model with an odd vocabulary in a padded
        # head, log-probabilities for the partial-mass loss, some of the
        # vocabulary masked
        dict(name="write_ragged", op="write", dtype="bf16", N=777, V=50257, K=50, pad=47,
             logprobs=True, masked=0.1),
        # one 4K-token sequence of teacher logits at the loss benchmark's
        # vocabulary, as the offline cache is written
        dict(name="write_4k", op="write", dtype="bf16", N=4096, V=131072, K=100, pad=0,
             logprobs=False, masked=0.0),
        # a shuffled micro-batch from a small cache
        dict(name="read_batch", op="read", rows=100003, N=2000, K=20),
        # the tokens of a long-context step from a cache of a million positions
        dict(name="read_256k", op="read", rows=1000000, N=262144, K=100),
        # a short fp32 sample: launches and latency
        dict(name="ckpt_small", op="ckpt", dtype="f32", N=77, D=768),
        # the hidden states of the headline training step
        dict(name="ckpt_32k", op="ckpt", dtype="bf16", N=32768, D=4096),
        # a small model trained in fp32, ragged sizes, a fifth of the tokens masked
        dict(name="train_f32", op="train", dtype="f32", N=1000, D=768, V=30011, K=32, chunk=300,
             tau=2.0, ignored=0.2),
        # one 4K-token sequence at the loss benchmark's head size
        dict(name="train_4k", op="train", dtype="bf16", N=4096, D=4096, V=131072, K=100,
             chunk=4096, tau=1.0, ignored=0.0),
        # one user's decoding step with four drafted tokens, latency
        dict(name="verify_one", op="verify", dtype="bf16", B=1, T=4, V=131072, K=100, pad=0,
             tau=1.0, masked=0.0, ragged=False),
        # a small server's batch, the draft's whole distribution in fp32, odd
        # vocabulary, constrained decoding, drafts of several lengths
        dict(name="verify_dense", op="verify", dtype="f32", B=32, T=7, V=50257, K=0, pad=0,
             tau=0.8, masked=0.3, ragged=True),
        # a busy server's batch, the draft truncated to its top 100
        dict(name="verify_256", op="verify", dtype="bf16", B=256, T=5, V=131072, K=100, pad=0,
             tau=1.0, masked=0.0, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges: rows 1 to 8192, vocabularies of
    1000 to 200000 columns, 1 to 256 entries, 1 to 12 drafted tokens."""
    op = rng.choice(["topk", "write", "write", "read", "ckpt", "train", "verify", "verify"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("topk", "write"):
        V = _log_int(rng, 1000, 200000)
        return dict(op=op, dtype=dtype, N=_log_int(rng, 1, min(8192, (1 << 29) // V)), V=V,
                    K=_log_int(rng, 1, 256), pad=rng.choice([0, 0, rng.randint(1, 128)]),
                    logprobs=rng.random() < 0.4, masked=rng.choice([0.0, 0.2, 0.999]))
    if op == "read":
        return dict(op=op, rows=_log_int(rng, 1000, 500000), N=_log_int(rng, 1, 262144),
                    K=_log_int(rng, 1, 128))
    if op == "ckpt":
        D = 64 * _log_int(rng, 1, 128)
        return dict(op=op, dtype=dtype, N=_log_int(rng, 1, (1 << 27) // D), D=D)
    if op == "train":
        return dict(op=op, dtype=dtype, N=_log_int(rng, 64, 2048), D=64 * _log_int(rng, 2, 32),
                    V=_log_int(rng, 1000, 60000), K=_log_int(rng, 1, 128),
                    chunk=_log_int(rng, 64, 2048), tau=rng.choice([0.7, 1.0, 2.0]),
                    ignored=rng.choice([0.0, round(rng.uniform(0.0, 0.9), 2)]))
    V, T = _log_int(rng, 1000, 200000), rng.randint(1, 12)
    return dict(op=op, dtype=dtype, B=_log_int(rng, 1, min(256, (1 << 28) // (V * (T + 1)))), T=T,
                V=V, K=rng.choice([0, _log_int(rng, 1, 256)]),
                pad=rng.choice([0, rng.randint(1, 128)]), tau=rng.choice([0.6, 1.0, 1.3]),
                masked=rng.choice([0.0, 0.5]), ragged=rng.random() < 0.5)


# ----------------------------------------------------------------- inputs --
def _gen(seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    return g, dev


def _logits(n, V, pad, std, dtype, masked, g, dev):
    """[n, V] logits, a view of rows of V + pad; a share of the vocabulary masked."""
    x = torch.empty(n, V + pad, dtype=dtype, device=dev)
    for s in range(0, n, 1024):
        e = min(n, s + 1024)
        x[s:e] = torch.randn(e - s, V + pad, generator=g, device=dev) * std
    if masked > 0:
        hidden = torch.rand(V + pad, generator=g, device=dev) < masked
        x[:, hidden] = float("-inf")
    return x[:, :V]


def _distinct(N, K, V, g, dev):
    x = torch.randint(0, V - K + 1, (N, K), generator=g, device=dev).sort(dim=1).values
    x = x + torch.arange(K, device=dev)
    order = torch.rand(N, K, generator=g, device=dev).argsort(dim=1)
    return x.gather(1, order).to(torch.int32).contiguous()


def prepare(case, seed):
    g, dev = _gen(seed)
    s = dict(case)
    op = case["op"]
    if op in ("topk", "write"):
        # teacher logits: a spread of 5, about half of the mass in the top 100
        s["logits"] = _logits(case["N"], case["V"], case["pad"], 5.0, DTYPES[case["dtype"]],
                              case["masked"], g, dev)
        s["K"] = min(case["K"], case["V"])
    elif op == "read":
        R, K = case["rows"], case["K"]
        code = torch.randint(0, 4096, (R, K), generator=g, device=dev, dtype=torch.int32)
        idx = torch.randint(0, 131072, (R, K), generator=g, device=dev, dtype=torch.int32)
        s["entries"] = (idx << 12) | code
        top = 10.0 + 3.0 * torch.randn(R, generator=g, device=dev)
        step = 0.001 + 0.003 * torch.rand(R, generator=g, device=dev)
        # one position in a hundred holds no entry (a fully masked teacher row)
        empty = torch.rand(R, generator=g, device=dev) < 0.01
        s["scale"] = torch.stack([top.masked_fill(empty, float("-inf")), step], dim=1)
        s["rows_idx"] = torch.randint(0, R, (case["N"],), generator=g, device=dev)
    elif op == "ckpt":
        x = torch.randn(case["N"], case["D"], generator=g, device=dev)
        # a few feature columns carry much larger values than the others
        big = torch.rand(case["D"], generator=g, device=dev) < 0.01
        s["hidden"] = (x * torch.where(big, 30.0, 1.0)).to(DTYPES[case["dtype"]])
    elif op == "train":
        N, D, V, K = case["N"], case["D"], case["V"], min(case["K"], case["V"])
        dt = DTYPES[case["dtype"]]
        s["hidden"] = torch.randn(N, D, generator=g, device=dev).to(dt).requires_grad_(True)
        s["W"] = (torch.randn(V, D, generator=g, device=dev) * 0.02).to(dt).requires_grad_(True)
        s["teacher_idx"] = _distinct(N, K, V, g, dev)
        s["teacher_logit"] = (torch.randn(N, K, generator=g, device=dev) * 3).sort(
            dim=1, descending=True).values.contiguous()
        s["ignore"] = None
        if case["ignored"] > 0:
            s["ignore"] = (torch.rand(N, generator=g, device=dev) < case["ignored"]).to(torch.uint8)
            s["ignore"][0] = 0
    else:
        B, T, V, K = case["B"], case["T"], case["V"], min(case["K"], case["V"])
        dt = DTYPES[case["dtype"]]
        x = _logits(B * (T + 1), V, case["pad"], 5.0, dt, case["masked"], g, dev)
        s["target"] = x.unflatten(0, (B, T + 1))
        # the draft: the target's logits with an error, as a distilled student has
        near = torch.empty(B, T, V, dtype=dt, device=dev)
        tokens = torch.empty(B, T, dtype=torch.int32, device=dev)
        s["draft_idx"] = s["draft_logit"] = s["draft_logits"] = None
        if K > 0:
            s["draft_idx"] = torch.empty(B, T, K, dtype=torch.int32, device=dev)
            s["draft_logit"] = torch.empty(B, T, K, dtype=torch.float32, device=dev)
        for b in range(0, B, 32):
            t = s["target"][b:b + 32, :T].float()
            t = (t + 0.7 * torch.randn(t.shape, generator=g, device=dev)).to(dt)
            if K > 0:
                v, i = t.float().topk(K, dim=-1)
                s["draft_idx"][b:b + 32], s["draft_logit"][b:b + 32] = i.int(), v
            else:
                near[b:b + 32] = t
                v, i = t.float(), None
            # a draw from the draft's softmax: the largest logit with Gumbel noise
            noise = torch.rand(v.shape, generator=g, device=dev).clamp_(1e-20, 1.0 - 1e-7)
            noise = noise.log_().neg_().log_().neg_()
            pick = (v / case["tau"] + noise).argmax(dim=-1)
            tokens[b:b + 32] = pick.int() if i is None else i.gather(2, pick[..., None])[..., 0].int()
        if K == 0:
            s["draft_logits"] = near
        s["tokens"] = tokens
        s["uniform"] = torch.rand(B, T + 1, generator=g, device=dev)
        s["lengths"] = None
        if case["ragged"]:
            s["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device=dev, dtype=torch.int32)
            s["lengths"][0] = T
    return s


# ------------------------------------------------------------ plain forms --
def _plain_topk(logits, K, logprobs):
    """(index, logit, row's log-probability shift): largest first, of equals the
    lowest index first."""
    x = logits.float()
    x = torch.where(x.isnan(), float("-inf"), x) + 0.0
    bits = x.view(torch.int32).long()
    order = torch.where(bits < 0, ~bits & 0x7fffffff | -(1 << 31), bits)   # as the values compare
    last = torch.arange(x.shape[1] - 1, -1, -1, device=x.device)
    idx = (order * (1 << 20) + last).topk(K, dim=1).indices
    z = x.gather(1, idx)
    shift = torch.zeros_like(z[:, :1])
    if logprobs:
        w = torch.where(x == z[:, :1], 0.0, x - z[:, :1]).exp()
        shift = torch.where(z[:, :1] == float("-inf"), 0.0, w.sum(1, keepdim=True).log())
    return idx.int(), z, shift


def _plain_values(z, shift, logprobs):
    if not logprobs:
        return z
    return torch.where(z == z[:, :1], 0.0, z - z[:, :1]) - shift + torch.where(
        z == float("-inf"), z, 0.0)


def _plain_write(logits, K, logprobs):
    idx, z, shift = _plain_topk(logits, K, logprobs)
    empty = z[:, :1] == float("-inf")
    top = torch.where(empty, 0.0, z[:, :1]).double()
    kept = (z >= top - REACH) & ~empty
    low = torch.where(kept, z.double(), top).amin(1, keepdim=True)
    step = ((top - low) / CODE_MAX).float()
    code = ((top - z.double()) / torch.where(step > 0, step, 1.0).double()).round()
    code = torch.where(kept, code.clamp(0, CODE_MAX), 4095.0).int()
    stored = torch.where(empty, float("-inf"), _plain_values(z, shift, logprobs)[:, :1])
    return (idx << 12) | code, torch.cat([stored, torch.where(empty, 0.0, step)], dim=1)


def _plain_read(entries, scale, rows):
    e, sc = (entries, scale) if rows is None else (entries[rows], scale[rows])
    code = e & 4095
    top = sc[:, :1].double()
    empty = top == float("-inf")
    value = (top - code * sc[:, 1:].double()).float()
    value = torch.where(code == 4095, float("-inf"), value)
    return {"teacher_idx": torch.where(empty, -1, (e >> 12) & 0xfffff),
            "teacher_logit": torch.where(empty, 0.0, value),
            "ignore": empty[:, 0].to(torch.uint8)}


def _plain_checkpoint(hidden):
    """The values that an 8-bit checkpoint stands for, in fp32."""
    x = hidden.float().unflatten(1, (-1, 32))
    m, e = torch.frexp(x.abs().amax(2, keepdim=True))
    # the least power of two with amax <= 448 = 0.875 * 2^9 of it
    e = (e - 9 + (m > 0.875)).clamp(min=-127)
    e = torch.where(m == 0, -127, e)
    codes = torch.ldexp(x.double(), -e).float().to(torch.float8_e4m3fn)
    return torch.ldexp(codes.double(), e).float().flatten(1)


def _plain_train(s):
    h, W, tau = s["hidden"].detach().float(), s["W"].detach().float(), s["tau"]
    idx = s["teacher_idx"].long()
    p = torch.softmax(s["teacher_logit"] / tau, dim=1)
    keep = torch.ones_like(h[:, 0]) if s["ignore"] is None else 1.0 - s["ignore"].float()
    w = keep / keep.sum()
    y = (h @ W.t()).div_(tau)
    top = y.amax(1, keepdim=True)
    logz = (y - top).exp_().sum(1).log() + top[:, 0]
    loss = (w * ((p * p.log()).sum(1) - (p * y.gather(1, idx)).sum(1) + p.sum(1) * logz)).sum()
    # gradients at the checkpoint's hidden states
    hc = _plain_checkpoint(s["hidden"].detach())
    y = (hc @ W.t()).div_(tau)
    q = y.sub_(y.amax(1, keepdim=True)).exp_()
    q = q.div_(q.sum(1, keepdim=True)).mul_(p.sum(1, keepdim=True))
    G = q.scatter_add_(1, idx, -p).mul_(w[:, None] / tau)
    return {"loss": loss, "grad_hidden": (G @ W).to(s["hidden"].dtype),
            "grad_W": (G.t() @ hc).to(s["W"].dtype)}


def _softmax64(x, tau):
    x = x.double()
    x = torch.where(x.isnan(), float("-inf"), x)
    m = x.amax(-1, keepdim=True)
    w = torch.where(x == m, 0.0, (x - m) / tau).exp()
    w = torch.where(m == float("-inf"), 0.0, w)
    return w / w.sum(-1, keepdim=True).clamp(min=1e-300)


def _plain_verify(s):
    B, T, V = s["B"], s["T"], s["V"]
    d, u = s["tokens"].long(), s["uniform"].double()
    p = _softmax64(s["target"], s["tau"])
    if s["draft_logits"] is not None:
        q = _softmax64(s["draft_logits"], s["tau"])
    else:
        q = torch.zeros(B, T, V, dtype=torch.float64, device=d.device)
        q.scatter_add_(2, s["draft_idx"].long(), _softmax64(s["draft_logit"], s["tau"]))
    pd = p[:, :T].gather(2, d[..., None])[..., 0]
    qd = q.gather(2, d[..., None])[..., 0]
    n = torch.full_like(d[:, 0], T) if s["lengths"] is None else s["lengths"].long()
    place = torch.arange(T, device=d.device)
    drafted = place < n[:, None]
    r = ((u[:, :T] * qd < pd) & drafted).long().cumprod(1).sum(1)
    at = torch.arange(B, device=d.device)
    x = p[at, r]
    rest = (x - q[at, r.clamp(max=T - 1)]).clamp(min=0)
    rest = torch.where(rest.sum(1, keepdim=True) > 0, rest, x)
    x = torch.where((r < n)[:, None], rest, x)
    c = x.cumsum(1)
    v = (c <= u[:, T:] * c[:, -1:]).sum(1)
    last = V - 1 - (x > 0).flip(1).long().argmax(1)
    v = torch.where(c[:, -1] > 0, torch.minimum(v, last), -1)
    out = torch.cat([torch.where(place < r[:, None], d, -1), torch.full_like(d[:, :1], -1)], 1)
    out[at, r] = v
    prob = torch.where(qd > 0, (pd / qd).clamp(max=1.0), (pd > 0).double())
    return {"tokens": out.int(), "accepted": r.int(),
            "accept_prob": torch.where(drafted, prob, 0.0).float()}


# -------------------------------------------------------------------- run --
def _own(s):
    import paper_2608_03796_amd as kd
    op = s["op"]
    if op == "topk":
        return kd.topk_entries(s["logits"], s["K"], logprobs=s["logprobs"])
    if op == "write":
        cache = kd.teacher_cache_write(s["logits"], s["K"], logprobs=s["logprobs"])
        return kd.teacher_cache_read(cache["entries"], cache["scale"])
    if op == "read":
        return kd.teacher_cache_read(s["entries"], s["scale"], rows=s["rows_idx"])
    if op == "ckpt":
        c = kd.checkpoint_write(s["hidden"])
        return kd.checkpoint_read(c["codes"], c["scales"], s["hidden"].dtype)
    if op == "train":
        loss = kd.topk_kl_loss(s["hidden"], s["W"], s["teacher_idx"], s["teacher_logit"],
                               tau=s["tau"], ignore=s["ignore"], chunk=s["chunk"],
                               schedule="recompute", checkpoint=True)
        gh, gw = torch.autograd.grad(loss, (s["hidden"], s["W"]))
        return {"loss": loss.detach(), "grad_hidden": gh, "grad_W": gw}
    return kd.verify_draft(s["target"], s["tokens"], s["uniform"], draft_idx=s["draft_idx"],
                           draft_logit=s["draft_logit"], draft_logits=s["draft_logits"],
                           lengths=s["lengths"], tau=s["tau"], accept_prob=True)


def run(s):
    if own:
        return _own(s)
    op = s["op"]
    if op == "topk":
        idx, z, shift = _plain_topk(s["logits"], s["K"], s["logprobs"])
        return {"teacher_idx": idx, "teacher_logit": _plain_values(z, shift, s["logprobs"])}
    if op == "write":
        entries, scale = _plain_write(s["logits"], s["K"], s["logprobs"])
        return _plain_read(entries, scale, None)
    if op == "read":
        return _plain_read(s["entries"], s["scale"], s["rows_idx"])
    if op == "ckpt":
        return _plain_checkpoint(s["hidden"]).to(s["hidden"].dtype)
    if op == "train":
        return _plain_train(s)
    return _plain_verify(s)


def work(case):
    op = case["op"]
    eb = 2 if case.get("dtype") == "bf16" else 4
    if op in ("topk", "write"):
        N, V, K = case["N"], case["V"], min(case["K"], case["V"])
        # logits read once; (index, value) written, from the cache with its
        # entries and scales written and read
        b = N * V * eb + N * K * 8
        if op == "write":
            b += N * (2 * (4 * K + 8) + 1)
        return {"bytes": float(b), "flops": float(N * V * (5 if case["logprobs"] else 1))}
    if op == "read":
        N, K = case["N"], case["K"]
        return {"bytes": float(N * (4 * K + 8 + 8 + 8 * K + 1)), "flops": 2.0 * N * K}
    if op == "ckpt":
        n = case["N"] * case["D"]
        # hidden read, codes and scales written; both read, hidden written
        return {"bytes": n * (2 * eb + 2 * (1 + 1 / 32)), "flops": 4.0 * n}
    if op == "train":
        N, D, V, K = case["N"], case["D"], case["V"], min(case["K"], case["V"])
        nv = N * (1.0 - case["ignored"])
        # forward: hidden, W and the teacher's entries; checkpoint written and
        # read; backward: W and entries again; both gradients
        b = nv * D * eb + N * D * 2.0625 + 2 * (V * D * eb + nv * K * 8) + (N + V) * D * eb
        # projection, and the backward's projection and two contractions
        return {"bytes": float(b), "flops": 8.0 * nv * D * V}
    B, T, V, K = case["B"], case["T"], case["V"], min(case["K"], case["V"])
    rows = B * (2 * T + 1 if K == 0 else T + 1)
    b = rows * V * eb + B * T * K * 8 + B * (T + 1) * 4 * 2 + B * T * 8 + 8 * B
    return {"bytes": float(b), "flops": 5.0 * rows * V}


# ------------------------------------------------------------------ exact --
def _exact_rows(logits, K, logprobs):
    z = logits.double().nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    val, idx = z.sort(dim=1, descending=True, stable=True)
    val, idx = val[:, :K], idx[:, :K]
    lse = torch.logsumexp(z, dim=1, keepdim=True)
    out = val - lse if logprobs else val
    return idx, val, out.masked_fill(val == -math.inf, -math.inf)


def _exact_write(logits, K, logprobs):
    idx, val, out = _exact_rows(logits, K, logprobs)
    none = val[:, 0] == -math.inf
    inside = val >= val[:, :1] - REACH
    low = val.masked_fill(~inside, math.inf).amin(dim=1, keepdim=True)
    step = ((val[:, :1] - low) / CODE_MAX).float().double()      # held in fp32
    code = torch.round((val[:, :1] - val) / step.where(step > 0, torch.ones_like(step)))
    value = (out[:, :1] - code.clamp(max=CODE_MAX) * step).masked_fill(~inside, -math.inf)
    return {"teacher_idx": idx.masked_fill(none[:, None], -1).int(),
            "teacher_logit": value.masked_fill(none[:, None], 0.0), "ignore": none.byte()}


def _exact_checkpoint(hidden):
    """Each value to the nearest number of 4 significant bits (ties to even) on
    its block's grid."""
    x = hidden.detach().double().reshape(hidden.shape[0], -1, 32)
    amax = x.abs().amax(dim=2, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(amax.clamp(min=1e-300) / 448.0)).clamp(min=-127.0))
    t = x / scale
    grid = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(t / grid) * grid * scale).reshape(hidden.shape)


def _exact_train(s):
    """The dense loss, and autograd's gradients of it at the checkpoint, in float64."""
    W = s["W"].detach().double()
    idx = s["teacher_idx"].long()
    rows = torch.arange(s["N"], device=W.device)
    if s["ignore"] is not None:
        rows = rows[s["ignore"] == 0]
    logp = torch.log_softmax(s["teacher_logit"][rows].double() / s["tau"], dim=1)

    def loss_and_G(h):
        logq = torch.log_softmax((h @ W.t()) / s["tau"], dim=1)
        loss = (logp.exp() * (logp - logq.gather(1, idx[rows]))).sum(1).mean()
        G = logq.exp_()
        G.scatter_add_(1, idx[rows], -logp.exp())
        return loss, G.div_(s["tau"] * len(rows))

    loss, G = loss_and_G(s["hidden"].detach()[rows].double())
    del G
    hc = _exact_checkpoint(s["hidden"])
    _, G = loss_and_G(hc[rows])
    gh = torch.zeros_like(hc)
    gh[rows] = G @ W
    return {"loss": loss, "grad_hidden": gh, "grad_W": G.t() @ hc[rows]}


def _exact_verify(s):
    """One sequence after the other, in log-probabilities."""
    B, T = s["B"], s["T"]
    out = {"tokens": torch.full((B, T + 1), -1, dtype=torch.int32),
           "accepted": torch.zeros(B, dtype=torch.int32),
           "accept_prob": torch.zeros(B, T, dtype=torch.float64)}
    tok, u = s["tokens"].tolist(), s["uniform"].double().tolist()
    n = [T] * B if s["lengths"] is None else s["lengths"].tolist()
    for b in range(B):
        p = torch.log_softmax(s["target"][b].double() / s["tau"], dim=1).exp()
        if s["draft_logits"] is not None:
            q = torch.log_softmax(s["draft_logits"][b].double() / s["tau"], dim=1).exp()
        else:
            k = torch.log_softmax(s["draft_logit"][b].double() / s["tau"], dim=1).exp()
            q = torch.zeros_like(p[:T]).scatter_(1, s["draft_idx"][b].long(), k)
        at = torch.tensor(tok[b], device=p.device)[:, None]
        pd, qd = p[:T].gather(1, at)[:, 0].tolist(), q.gather(1, at)[:, 0].tolist()
        for t in range(n[b]):
            out["accept_prob"][b, t] = min(1.0, pd[t] / qd[t]) if qd[t] > 0 else float(pd[t] > 0)
        r = 0
        while r < n[b] and u[b][r] * qd[r] < pd[r]:
            out["tokens"][b, r] = tok[b][r]
            r += 1
        out["accepted"][b] = r
        x = p[r]
        if r < n[b]:
            x = (p[r] - q[r]).clamp(min=0.0)
        c = x.cumsum(0)
        place = torch.searchsorted(c, (u[b][T] * c[-1:]), right=True)
        out["tokens"][b, r] = int(place[0])
    return {k: v.to(s["target"].device) for k, v in out.items()}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "topk":
        idx, _, value = _exact_rows(s["logits"], s["K"], s["logprobs"])
        return {"teacher_idx": idx.int(), "teacher_logit": value}
    if op == "write":
        return _exact_write(s["logits"], s["K"], s["logprobs"])
    if op == "read":
        e, sc = s["entries"][s["rows_idx"]], s["scale"][s["rows_idx"]].double()
        empty = sc[:, 0] == -math.inf
        value = (sc[:, :1] - (e % 4096) * sc[:, 1:]).masked_fill(e % 4096 == 4095, -math.inf)
        return {"teacher_idx": (e // 4096).masked_fill(empty[:, None], -1),
                "teacher_logit": value.masked_fill(empty[:, None], 0.0), "ignore": empty.byte()}
    if op == "ckpt":
        return _exact_checkpoint(s["hidden"])
    if op == "train":
        return _exact_train(s)
    return _exact_verify(s)
