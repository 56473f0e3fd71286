"""The loss's backward from 8-bit checkpoints of the hidden states, and a run of the
operators around the loss as a distillation uses them."""
import numpy as np
import pytest
import torch

import kd_inputs as ki
from oracle import kd_topk_kl
from oracle import ops_oracle as oo
from tests.helpers import TOL, rel_max, to64

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _problem(N, D, V, K, dtype, ignored, seed):
    dev, dt = "cuda", DT[dtype]
    h = ki.make_hidden(N, D, dt, dev, seed=seed)
    W = ki.make_weight(V, D, dt, dev, seed=seed + 1, std=0.1)
    idx, tl = ki.make_teacher(N, K, V, dev, seed=seed + 2)
    ign = None
    if ignored > 0:
        g = torch.Generator(device="cpu")
        g.manual_seed(seed)
        ign = (torch.rand(N, generator=g) < ignored).to(torch.uint8).to(dev)
    return h, W, idx, tl, ign


CASES = [(1, 64, 300, 5, 1, 0.0), (300, 128, 2000, 16, 128, 0.0), (300, 128, 2000, 16, 128, 0.3),
         (77, 320, 5003, 200, 4096, 0.0), (700, 64, 1000, 130, 256, 0.5), (513, 256, 1500, 7, 100, 0.0),
         (40, 64, 500, 3, 16, 1.0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V,K,chunk,ignored", CASES)
def test_bwd_checkpoint(gpu_lib, N, D, V, K, chunk, ignored, dtype):
    """Bitwise the fused call on the decoded rows, and the oracle's gradients
    there; with an upstream scalar and with per-token gradients by linearity."""
    kd, tau = gpu_lib, 1.3
    print(f"[ckpt] {N} {D} {V} {K} chunk={chunk} ignored={ignored} {dtype}", flush=True)
    h, W, idx, tl, ign = _problem(N, D, V, K, dtype, ignored, 300)
    c = kd.checkpoint_write(h)
    hd = kd.checkpoint_read(c["codes"], c["scales"], h.dtype)
    assert np.array_equal(to64(hd), oo.checkpoint(to64(h))[0])
    kw = dict(tau=tau, ignore=ign, chunk=chunk)
    fused = kd.fwd_bwd(hd, W, idx, tl, **kw)
    got = kd.bwd_checkpoint(c["codes"], c["scales"], W, idx, tl, **kw)
    for k in got:
        assert torch.equal(got[k], fused[k]), k
    # one gradient at a time, added to what is there
    acc = torch.full_like(got["grad_W"], 0.25)
    kd.bwd_checkpoint(c["codes"], c["scales"], W, idx, tl, grad_hidden=False, grad_W_out=acc,
                      accumulate_grad_W=True, **kw)
    ref = kd_topk_kl(to64(hd), to64(W), to64(idx), to64(tl), tau=tau, ignore=to64(ign))
    tol = TOL[dtype]["grad"]
    assert rel_max(to64(got["grad_hidden"]), ref["grad_hidden"]) <= tol
    assert rel_max(to64(got["grad_W"]), ref["grad_W"]) <= tol
    # (0.25 + x rounds once more in fp32)
    assert np.abs(to64(acc) - 0.25 - ref["grad_W"]).max() <= \
        tol * np.abs(ref["grad_W"]).max() + 2.0 ** -24
    g = torch.tensor(-2.5, device="cuda")
    f = kd.bwd_checkpoint(c["codes"], c["scales"], W, idx, tl, grad_loss=g, grad_hidden_f32=True, **kw)
    assert f["grad_hidden"].dtype == torch.float32
    assert rel_max(to64(f["grad_hidden"]), -2.5 * ref["grad_hidden"]) <= tol
    assert rel_max(to64(f["grad_W"]), -2.5 * ref["grad_W"]) <= tol
    # per token, some of them 0: the gradient of sum_t u_t l_t
    u = torch.randn(N, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")
    u[::3] = 0.0
    f = kd.bwd_checkpoint(c["codes"], c["scales"], W, idx, tl, grad_loss_per_token=u, **kw)
    n = max(1, N if ign is None else int((ign == 0).sum()))
    gh = ref["grad_hidden"] * n * to64(u)[:, None]
    assert rel_max(to64(f["grad_hidden"]), gh) <= tol
    # dW = sum_t u_t dz_t h_t: from the rows' own gradients of the logits
    y = to64(hd) @ to64(W).T / tau
    y -= y.max(1, keepdims=True)
    G = np.exp(y)
    G /= G.sum(1, keepdims=True)
    p = np.exp(to64(tl) / tau - (to64(tl) / tau).max(1, keepdims=True))
    np.subtract.at(G, (np.arange(N)[:, None], to64(idx)), p / p.sum(1, keepdims=True))
    G *= to64(u)[:, None] / tau * (1.0 if ign is None else (to64(ign) == 0)[:, None])
    assert rel_max(to64(f["grad_W"]), G.T @ to64(hd)) <= tol


@pytest.mark.parametrize("N,D,V,chunk", [
    (5000, 64, 8192, 2048),     # rows prepared once for a group of chunks
    (9000, 4096, 2000, 4000),   # and chunk by chunk inside a group
    (20000, 64, 1000, 1024)])   # several groups
@pytest.mark.parametrize("ignored", [0.0, 0.3])
def test_bwd_checkpoint_schedules(gpu_lib, N, D, V, chunk, ignored):
    kd = gpu_lib
    h, W, idx, tl, ign = _problem(N, D, V, 9, "bf16", ignored, 350)
    c = kd.checkpoint_write(h)
    hd = kd.checkpoint_read(c["codes"], c["scales"], h.dtype)
    kw = dict(ignore=ign, chunk=chunk)
    fused = kd.fwd_bwd(hd, W, idx, tl, **kw)
    got = kd.bwd_checkpoint(c["codes"], c["scales"], W, idx, tl, **kw)
    for k in got:
        assert torch.equal(got[k], fused[k]), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ignored", [0.0, 0.4])
def test_loss_with_checkpoint(gpu_lib, dtype, ignored):
    """topk_kl_loss(checkpoint=True): the exact loss, gradients at the checkpoint;
    twice through one graph; the hidden tensor's memory may go in between."""
    kd, tau = gpu_lib, 0.9
    h, W, idx, tl, ign = _problem(200, 192, 3001, 20, dtype, ignored, 400)
    hd = oo.checkpoint(to64(h))[0]
    ref = kd_topk_kl(to64(h), to64(W), to64(idx), to64(tl), tau=tau, ignore=to64(ign))
    refd = kd_topk_kl(hd, to64(W), to64(idx), to64(tl), tau=tau, ignore=to64(ign))
    x = torch.nn.Parameter(h.clone())
    Wp = torch.nn.Parameter(W.clone())
    kw = dict(tau=tau, ignore=ign, chunk=64, schedule="recompute", checkpoint=True)
    loss = kd.topk_kl_loss(x, Wp, idx, tl, **kw)
    tol = TOL[dtype]
    assert abs(float(loss.detach()) - ref["loss"]) <= tol["loss"] * abs(ref["loss"])
    x.data.fill_(float("nan"))                 # what the backward reads is its own
    for scale in (1.0, 3.0):
        gh, gw = torch.autograd.grad(loss * scale, (x, Wp), retain_graph=True)
        assert gh.dtype == h.dtype and gw.dtype == W.dtype
        # bf16: also the rounding of grad_W to its type, half a step of 2^-8
        extra = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        assert rel_max(to64(gh), scale * refd["grad_hidden"]) <= tol["grad"]
        assert rel_max(to64(gw), scale * refd["grad_W"]) <= tol["grad"] + extra
    # one gradient only, and none
    x.data.copy_(h)
    loss = kd.topk_kl_loss(h, Wp, idx, tl, **kw)
    loss.backward()
    assert rel_max(to64(Wp.grad), refd["grad_W"]) <= tol["grad"] + extra
    with torch.no_grad():
        assert torch.equal(kd.topk_kl_loss(x, Wp, idx, tl, **kw), loss)
    assert torch.equal(kd.topk_kl_loss(h, W, idx, tl, **kw), loss)
    with pytest.raises(ValueError):
        kd.topk_kl_loss(x, Wp, idx, tl, checkpoint=True)


def test_gradient_by_differences(gpu_lib):
    """fp32: the checkpoint's gradient against central differences of the loss at
    the decoded rows (in 64 bits, by the oracle)."""
    kd = gpu_lib
    h, W, idx, tl, _ = _problem(3, 64, 200, 5, "f32", 0.0, 500)
    c = kd.checkpoint_write(h)
    got = kd.bwd_checkpoint(c["codes"], c["scales"], W, idx, tl)
    hd, w = to64(kd.checkpoint_read(c["codes"], c["scales"], torch.float32)), to64(W)

    def loss(a, b):
        return kd_topk_kl(a, b, to64(idx), to64(tl))["loss"]
    rng = np.random.default_rng(0)
    for name, base in (("grad_hidden", hd), ("grad_W", w)):
        g = to64(got[name])
        for _ in range(8):
            d = rng.standard_normal(base.shape)
            e = 1e-5
            hi, lo = (loss(base + e * d, w), loss(base - e * d, w)) if name == "grad_hidden" else \
                (loss(hd, base + e * d), loss(hd, base - e * d))
            # error of the difference: e^2 of third derivatives, 1e-16 / e of rounding
            want = (hi - lo) / (2 * e)
            assert abs((g * d).sum() - want) <= 1e-5 * np.abs(g).max() * np.abs(d).sum() + 1e-7


def test_confident_tokens_have_no_gradient(gpu_lib):
    """A student that is sure of the teacher's only token: large logits move by
    several units under the checkpoint's rounding, and the gradient stays 0."""
    kd, N, D, V = gpu_lib, 64, 64, 256
    h = ki.make_hidden(N, D, torch.float32, "cuda", seed=9)
    W = ki.make_weight(V, D, torch.float32, "cuda", seed=10, std=0.01)
    W[5] = 0.0
    W[5, 0] = 50.0
    h[:, 0] = 2.03
    idx = torch.full((N, 1), 5, dtype=torch.int32, device="cuda")
    tl = torch.zeros(N, 1, device="cuda")
    c = kd.checkpoint_write(h)
    hd = kd.checkpoint_read(c["codes"], c["scales"], torch.float32)
    assert bool(((hd - h)[:, 0].abs() * 50 > 1).all())
    got = kd.bwd_checkpoint(c["codes"], c["scales"], W, idx, tl)
    # every other token has e^-90; q = 2^(y - log2 Z) with both near 146, where half
    # a step of fp32 is 2^-17: up to four such roundings in the exponent
    assert float(got["grad_hidden"].abs().max()) <= 50 * 4 * 2.0 ** -17 / N


@pytest.mark.parametrize("masked", [False, True])
def test_captured_step(gpu_lib, masked):
    """Checkpoint, loss and gradients captured and replayed between eager calls."""
    kd = gpu_lib
    h, W, idx, tl, ign = _problem(300, 128, 2000, 16, "bf16", 0.2 if masked else 0.0, 600)
    ws = kd.alloc_workspace(300, 128, 2000, 16, 128, 1.0, kd.KD_BF16, "cuda")

    def step():
        c = kd.checkpoint_write(h)
        return dict(c, **kd.bwd_checkpoint(c["codes"], c["scales"], W, idx, tl, ignore=ign,
                                           chunk=128, workspace=ws))
    eager = step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for rep in range(3):
        for t in got.values():
            t.zero_()
        kd.fwd_bwd(h, W, idx, tl, ignore=ign, chunk=64)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for k in eager:
            assert torch.equal(got[k], eager[k]), (rep, k)


def test_captured_autograd_step(gpu_lib):
    """Loss and gradients through autograd, captured on leaves of their own."""
    kd = gpu_lib
    h, W, idx, tl, ign = _problem(300, 128, 2000, 16, "bf16", 0.2, 650)
    ws = kd.alloc_workspace(300, 128, 2000, 16, 128, 1.0, kd.KD_BF16, "cuda")

    def step(x, w):
        loss = kd.topk_kl_loss(x, w, idx, tl, ignore=ign, chunk=128, schedule="recompute",
                               checkpoint=True, workspace=ws)
        return (loss.detach(),) + torch.autograd.grad(loss, (x, w))
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):      # (autograd's first call on the capturing stream)
        eager = step(h.clone().requires_grad_(), W.clone().requires_grad_())
    s.synchronize()
    x, w = h.clone().requires_grad_(), W.clone().requires_grad_()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        got = step(x, w)
    for rep in range(3):
        for t in got:
            t.zero_()
        kd.fwd_bwd(h, W, idx, tl, ignore=ign, chunk=64)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            assert torch.equal(a, b), rep


def test_distillation_run(gpu_lib):
    """The operators together: teacher logits to the cache, a shuffled batch read
    from it, a training step with 8-bit hidden states, and the student's drafts
    verified against the teacher."""
    kd, N, D, V, K = gpu_lib, 96, 128, 2003, 20
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(N, V, generator=g, device="cuda") * 4
    z[5] = float("-inf")                       # a position without a target
    cache = kd.teacher_cache_write(z, K, logprobs=True)
    rows = torch.randperm(N, generator=g, device="cuda")
    t = kd.teacher_cache_read(cache["entries"], cache["scale"], rows=rows)
    assert int(t["ignore"].sum()) == 1 and int(t["ignore"][rows == 5]) == 1
    assert kd.check_indices(t["teacher_idx"][t["ignore"] == 0].contiguous(), V)
    h, W, _, _, _ = _problem(N, D, V, K, "f32", 0.0, 700)
    hp, Wp = torch.nn.Parameter(h), torch.nn.Parameter(W)
    loss = kd.topk_kl_loss(hp, Wp, **t, teacher_logprobs=True, schedule="recompute", checkpoint=True)
    loss.backward()
    keep = to64(t["ignore"]) == 0
    ref = kd_topk_kl(to64(h)[keep], to64(W), to64(t["teacher_idx"])[keep],
                     to64(t["teacher_logit"])[keep], teacher_mode="logprobs")
    refd = kd_topk_kl(oo.checkpoint(to64(h))[0][keep], to64(W), to64(t["teacher_idx"])[keep],
                      to64(t["teacher_logit"])[keep], teacher_mode="logprobs")
    assert abs(float(loss.detach()) - ref["loss"]) <= 1e-5 * abs(ref["loss"])
    assert rel_max(to64(hp.grad)[keep], refd["grad_hidden"]) <= 1e-5
    assert not bool(hp.grad[t["ignore"] == 1].any())
    assert rel_max(to64(Wp.grad), refd["grad_W"]) <= 1e-5
    # 32 sequences of 2 drafted tokens: the student proposes from its top K
    B, T = 32, 2
    target = z.view(B, T + 1, V)
    student = (h @ W.t()).view(B, T + 1, V)[:, :T]
    d = kd.topk_entries(student.reshape(B * T, V), K)
    di, dl = d["teacher_idx"].view(B, T, K), d["teacher_logit"].view(B, T, K)
    pick = torch.multinomial(torch.softmax(dl, 2).view(-1, K), 1, generator=g).view(B, T, 1)
    tokens = di.gather(2, pick)[..., 0].contiguous()
    u = torch.rand(B, T + 1, generator=g, device="cuda")
    out = kd.verify_draft(target, tokens, u, draft_idx=di, draft_logit=dl, accept_prob=True)
    q = np.stack([[oo.draft_distribution(to64(di)[b, s], to64(dl)[b, s], V, 1.0) for s in range(T)]
                  for b in range(B)])
    want = oo.verify_draft(to64(target), to64(tokens), to64(u), q)
    assert np.array_equal(to64(out["tokens"]), want[0])
    assert np.array_equal(to64(out["accepted"]), want[1])
