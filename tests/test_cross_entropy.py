"""Cross entropy against labels on the GPU against the fp64 oracle, and the output
head's operators in a row."""
import numpy as np
import pytest
import torch

import kd_inputs as ki
from oracle import head_oracle as ho
from oracle import ops_oracle as oo
from tests.helpers import TOL, rel_max, to64

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _inputs(N, D, V, dtype, labels="some", seed=0):
    h = torch.randn(N, D, generator=_gen(seed), device="cuda").to(DT[dtype])
    W = (torch.randn(V, D, generator=_gen(seed + 1), device="cuda") * 0.05).to(DT[dtype])
    lab = torch.randint(0, V, (N,), generator=_gen(seed + 2), device="cuda")
    if labels == "none":
        lab.fill_(-100)
    elif labels == "some":
        odd = torch.tensor([-100, -1, V, 2 ** 40, -2 ** 63, 2 ** 32, V + 7], device="cuda")
        out = torch.rand(N, generator=_gen(seed + 3), device="cuda") < 0.4
        out[0] = False
        lab = torch.where(out, odd[torch.arange(N, device="cuda") % 7], lab)
    elif labels == "one":
        lab.fill_(V // 2)
    return h, W, lab


def _ref(h, W, lab, **kw):
    return ho.cross_entropy(to64(h), to64(W), lab.cpu().numpy(), **kw)


def _check(got, ref, dtype, h=None, W=None, lab=None):
    """The contract's tolerances, and what the difference of nearly equal numbers adds.
    ln Z and z[label] are sums of numbers of their own size and of the fused call's
    reference, 24 in base 2 above a logit: each comes out of at most 8 roundings (2^-24)
    at size + 24 ln 2. The loss is their difference; q[label] is its exponential, off by
    that much of itself, from which the gradient takes 1 (h, W and lab given: for tokens
    nearly certain of their label, with next to no gradient)."""
    t = TOL[dtype]
    noise = 16 * 2.0 ** -24 * (ref["size"] + 24 * np.log(2.0))
    diff = noise.max(initial=0.0)
    if "loss" in got:
        assert abs(float(got["loss"].detach()) - ref["loss"]) <= t["loss"] * abs(ref["loss"]) + diff
    if "loss_per_token" in got:
        err = np.abs(to64(got["loss_per_token"]) - ref["loss_per_token"]).max(initial=0.0)
        assert err <= t["loss"] * np.abs(ref["loss_per_token"]).max(initial=0.0) + diff
    more = {"grad_hidden": 0.0, "grad_W": 0.0}
    if h is not None:
        n = np.abs(ref["weight"]) * ref["q_label"] * noise
        more["grad_hidden"] = (n * np.abs(to64(W)).max()).max(initial=0.0)
        per = np.zeros(W.shape[0])
        ok = n > 0
        np.add.at(per, lab.cpu().numpy()[ok], n[ok])
        more["grad_W"] = per.max() * np.abs(to64(h)).max()
    for k in ("grad_hidden", "grad_W"):
        if k in got:
            err = np.abs(to64(got[k]) - ref[k]).max(initial=0.0)
            assert err <= t["grad"] * np.abs(ref[k]).max(initial=0.0) + more[k], k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V,chunk,labels,z", [
    (1, 64, 1, 16, "all", 1e-2), (1, 64, 5, 4096, "all", 0.0), (3, 64, 100, 2, "some", 1e-3),
    (64, 512, 8192, 4096, "all", 0.0), (257, 128, 257, 100, "some", 1e-4),
    (300, 256, 3000, 128, "some", 1e-2), (300, 256, 3000, 128, "none", 1e-2),
    (500, 192, 1031, 4096, "one", 1e-4), (1000, 768, 5003, 300, "some", 1e-4),
    (2500, 64, 300, 512, "all", 1e-4)])
def test_fwd_bwd(gpu_lib, dtype, N, D, V, chunk, labels, z):
    kd = gpu_lib
    h, W, lab = _inputs(N, D, V, dtype, labels, seed=N + V)
    ref = _ref(h, W, lab, z_loss=z)
    got = kd.ce_fwd_bwd(h, W, lab, z_loss=z, chunk=chunk, loss_per_token=True)
    _check(got, ref, dtype, h, W, lab)
    ignored = (lab < 0) | (lab >= V)
    assert not got["grad_hidden"][ignored].any() and not got["loss_per_token"][ignored].any()
    # the same bits again, and the loss alone
    again = kd.ce_fwd_bwd(h, W, lab, z_loss=z, chunk=chunk, loss_per_token=True)
    for k in got:
        assert torch.equal(got[k], again[k]), k
    alone = kd.ce_fwd_bwd(h, W, lab, z_loss=z, chunk=chunk, grad_hidden=False, grad_W=False)
    _check(alone, ref, dtype)
    # the split calls: log Z off by its rounding and the projection's, which the
    # contract's tolerance of the loss bounds
    f = kd.ce_fwd(h, W, lab, z_loss=z, chunk=chunk, loss_per_token=True)
    _check({k: f[k] for k in ("loss", "loss_per_token")}, ref, dtype)
    assert rel_max(to64(f["saved_logz"]), ref["logz"]) <= TOL[dtype]["loss"]
    _check(kd.ce_bwd(h, W, lab, f["saved_logz"], z_loss=z, chunk=chunk), ref, dtype, h, W,
           lab)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_is_the_loss_of_one_entry(gpu_lib, dtype):
    """Without the z-loss: bitwise the distillation loss of a teacher that holds the
    label alone, which shares every kernel."""
    kd = gpu_lib
    N, D, V = 700, 256, 5000
    h, W, lab = _inputs(N, D, V, dtype, "some", 4)
    bad = (lab < 0) | (lab >= V)
    idx = torch.where(bad, 0, lab).to(torch.int32)[:, None].contiguous()
    want = kd.fwd_bwd(h, W, idx, torch.zeros(N, 1, device="cuda"), ignore=bad.to(torch.uint8),
                      chunk=256, loss_per_token=True)
    got = kd.ce_fwd_bwd(h, W, lab, chunk=256, loss_per_token=True)
    for k in want:
        assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_upstream_gradients(gpu_lib, dtype):
    kd = gpu_lib
    N, D, V, z = 300, 128, 999, 1e-3
    h, W, lab = _inputs(N, D, V, dtype, "some", 5)
    f = kd.ce_fwd(h, W, lab, z_loss=z)
    up = torch.randn(N, generator=_gen(9), device="cuda")
    got = kd.ce_bwd(h, W, lab, f["saved_logz"], z_loss=z, grad_loss_per_token=up)
    _check(got, _ref(h, W, lab, z_loss=z, g_token=to64(up)), dtype)
    g = torch.tensor(-3.0, device="cuda")
    acc = torch.ones(V, D, device="cuda")
    got = kd.ce_bwd(h, W, lab, f["saved_logz"], z_loss=z, grad_loss=g, grad_W_out=acc,
                    accumulate_grad_W=True, grad_hidden_f32=True)
    ref = _ref(h, W, lab, z_loss=z, g=-3.0)
    assert got["grad_W"] is acc and got["grad_hidden"].dtype == torch.float32
    # (the sum with 1 rounds to a step of fp32 at 2 at most)
    assert np.abs(to64(acc) - 1 - ref["grad_W"]).max() <= \
        TOL[dtype]["grad"] * np.abs(ref["grad_W"]).max() + 2.0 ** -23
    only = kd.ce_bwd(h, W, lab, f["saved_logz"], z_loss=z, grad_hidden=False)
    assert set(only) == {"grad_W"}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("schedule", ["fused", "recompute"])
def test_autograd(gpu_lib, dtype, schedule):
    kd = gpu_lib
    h, W, lab = _inputs(400, 128, 1500, dtype, "some", 6)
    ref = _ref(h, W, lab, z_loss=1e-3, g=2.5)
    h.requires_grad_(True)
    W.requires_grad_(True)
    loss = kd.cross_entropy(h, W, lab, z_loss=1e-3, chunk=128, schedule=schedule)
    (2.5 * loss).backward(retain_graph=True)
    _check({"loss": loss, "grad_hidden": h.grad, "grad_W": W.grad}, ref, dtype)
    assert h.grad.dtype == h.dtype and W.grad.dtype == W.dtype
    if schedule == "fused":
        with pytest.raises(RuntimeError):
            loss.backward()
    else:
        first = h.grad.clone()
        (2.5 * loss).backward()
        assert torch.equal(h.grad, first + first)
    # one of the two alone, and none
    h2 = h.detach()
    gw, = torch.autograd.grad(kd.cross_entropy(h2, W, lab, z_loss=1e-3, schedule=schedule), [W])
    _check({"grad_W": gw}, _ref(h, W, lab, z_loss=1e-3), dtype)
    with torch.no_grad():
        assert not kd.cross_entropy(h, W, lab, schedule=schedule).requires_grad


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("far", [-2000.0, -60.0, 60.0, 2000.0])
def test_far_labels(gpu_lib, dtype, far):
    """Tokens whose label lies far from the other logits: nearly certain ones, whose
    gradient is nearly 0, and ones with next to no probability."""
    kd = gpu_lib
    N, D, V = 130, 64, 700
    h = torch.zeros(N, D, device="cuda")
    h[:, 0] = 1.0
    h[:, 1:] = torch.randn(N, D - 1, generator=_gen(1), device="cuda")
    W = torch.randn(V, D, generator=_gen(2), device="cuda") * 0.1
    W[:, 0] = 0.0
    W[7, 0] = far
    h, W = h.to(DT[dtype]), W.to(DT[dtype])
    lab = torch.full((N,), 7, device="cuda")
    lab[1::3] = 9
    ref = _ref(h, W, lab, z_loss=1e-4)
    got = kd.ce_fwd_bwd(h, W, lab, z_loss=1e-4, loss_per_token=True)
    _check({k: got[k] for k in ("loss", "grad_hidden", "grad_W")}, ref, dtype, h, W, lab)
    f = kd.ce_fwd(h, W, lab, z_loss=1e-4)
    _check(kd.ce_bwd(h, W, lab, f["saved_logz"], z_loss=1e-4), ref, dtype, h, W, lab)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("factor", [0.5, 1.0, 1.0 + 2.0 ** -20, 3.0])
def test_z_loss_that_cancels(gpu_lib, dtype, factor):
    """ln Z below 0 and a z-loss whose weight 1 + 2 z_loss ln Z is 0, near it, or
    below: the gradient is what is left, the label's column."""
    kd = gpu_lib
    N, D, V = 64, 64, 512
    h = torch.ones(N, D, device="cuda")
    W = torch.full((V, D), -0.25, device="cuda")
    h, W = h.to(DT[dtype]), W.to(DT[dtype])
    lab = torch.arange(N, device="cuda") * 3
    lnz = np.log(V) - 16.0
    z = float(np.float32(factor * -0.5 / lnz))
    ref = _ref(h, W, lab, z_loss=z)
    got = kd.ce_fwd_bwd(h, W, lab, z_loss=z)
    _check(got, ref, dtype, h, W, lab)
    f = kd.ce_fwd(h, W, lab, z_loss=z)
    _check(kd.ce_bwd(h, W, lab, f["saved_logz"], z_loss=z), ref, dtype, h, W, lab)


def test_gradient_against_differences(gpu_lib):
    """The loss along a direction. fp32: each loss of about 7 is off by at most 1e-5 of
    itself (the contract's tolerance), so a quotient over a step of 2 t by 7e-5 / t;
    the third derivative along a unit direction is below 1 (logits change by at most
    |dh| |W| + |h| |dW|), which leaves t^2 / 6."""
    kd = gpu_lib
    N, D, V, z = 64, 64, 1000, 1e-2
    h, W, lab = _inputs(N, D, V, "f32", "some", 11)
    out = kd.ce_fwd_bwd(h, W, lab, z_loss=z)
    for name, x, grad in (("h", h, out["grad_hidden"]), ("W", W, out["grad_W"])):
        # the steepest direction, where the quotient is largest
        d = grad / grad.norm()
        t = 0.1
        def at(s):
            a, b = (h + s * d, W) if name == "h" else (h, W + s * d)
            return float(kd.ce_fwd_bwd(a, b, lab, z_loss=z, grad_hidden=False,
                                       grad_W=False)["loss"])
        quotient = (at(t) - at(-t)) / (2 * t)
        assert abs(quotient - float(grad.norm())) <= 7e-5 / t + t * t / 6


def test_empty(gpu_lib):
    kd = gpu_lib
    h = torch.empty(0, 64, device="cuda")
    W = torch.ones(10, 64, device="cuda")
    out = kd.ce_fwd_bwd(h, W, torch.empty(0, dtype=torch.int64, device="cuda"))
    assert float(out["loss"]) == 0 and not out["grad_W"].any()
    assert out["grad_hidden"].shape == (0, 64)


@pytest.mark.parametrize("schedule", ["fused", "recompute"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [0, 3])
def test_no_labels_autograd(gpu_lib, N, dtype, schedule):
    """No token, and none with a label: a loss of 0 and gradients of 0."""
    kd = gpu_lib
    h = torch.ones(N, 64, device="cuda", dtype=dtype, requires_grad=True)
    W = torch.ones(10, 64, device="cuda", dtype=dtype, requires_grad=True)
    lab = torch.tensor([-100, 10, 1 << 40][:N], dtype=torch.int64, device="cuda")
    loss = kd.cross_entropy(h, W, lab, z_loss=1e-3, schedule=schedule)
    loss.backward()
    assert float(loss.detach()) == 0 and h.grad.shape == h.shape
    assert not h.grad.any() and not W.grad.any()


def test_ignored_upstream_not_a_number(gpu_lib):
    """An ignored token's upstream gradient, logit row and ln Z reach no result."""
    kd = gpu_lib
    h, W, lab = _inputs(130, 64, 700, "f32", "some", 19)
    keep = (lab >= 0) & (lab < 700)
    assert keep.any() and not keep.all()
    up = torch.ones(130, device="cuda")
    logz = kd.ce_fwd(h, W, lab)["saved_logz"]
    want = kd.ce_bwd(h, W, lab, logz, grad_loss_per_token=up)
    h2, up2, logz2 = h.clone(), up.clone(), logz.clone()
    h2[~keep], up2[~keep], logz2[~keep] = float("nan"), float("nan"), float("nan")
    got = kd.ce_bwd(h2, W, lab, logz2, grad_loss_per_token=up2)
    for k in want:
        assert torch.equal(got[k], want[k]), k
    for k, v in kd.ce_fwd_bwd(h, W, lab).items():
        assert torch.equal(v, kd.ce_fwd_bwd(h2, W, lab)[k]), k


@pytest.mark.parametrize("z", [0.0, 1e-3])
def test_graph(gpu_lib, z):
    """A captured step replays with new inputs, on workspaces full of anything."""
    kd = gpu_lib
    N, D, V = 300, 128, 2000
    h, W, lab = _inputs(N, D, V, "bf16", "some", 13)
    ws = torch.empty(kd.ce_workspace_size(N, D, V, 128), dtype=torch.uint8, device="cuda")
    out = kd.ce_fwd_bwd(h, W, lab, z_loss=z, chunk=128, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kd.ce_fwd_bwd(h, W, lab, z_loss=z, chunk=128, workspace=ws, out=out)
    for seed in (20, 30, 40):
        h2, _, lab2 = _inputs(N, D, V, "bf16", "some", seed)
        h.copy_(h2)
        lab.copy_(lab2)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        want = kd.ce_fwd_bwd(h, W, lab, z_loss=z, chunk=128)
        for k in want:
            assert torch.equal(out[k], want[k]), k


def test_two_at_a_time(gpu_lib):
    """Calls that overlap on streams of their own, and graphs that share a workspace."""
    kd = gpu_lib
    N, D, V = 500, 256, 3000
    sets = []
    for seed in (1, 2):
        h, W, lab = _inputs(N, D, V, "bf16", "some", seed)
        sets.append((h, W, lab, kd.ce_fwd_bwd(h, W, lab, z_loss=1e-3), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for h, W, lab, want, s in sets:
            with torch.cuda.stream(s):
                got.append((kd.ce_fwd_bwd(h, W, lab, z_loss=1e-3), want))
    torch.cuda.synchronize()
    for a, b in got:
        assert all(torch.equal(a[k], b[k]) for k in b)
    ws = torch.empty(kd.ce_workspace_size(N, D, V), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for h, W, lab, want, s in sets:
        out = {k: torch.zeros_like(v) for k, v in want.items()}
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kd.ce_fwd_bwd(h, W, lab, z_loss=1e-3, workspace=ws, out=out)
        graphs.append(g)
        outs.append(out)
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for out, s in zip(outs, sets):
            assert all(torch.equal(out[k], s[3][k]) for k in out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_groups(gpu_lib, dtype):
    """More tokens than a contraction gathers and than the scan takes labels for, most of
    them ignored in stretches."""
    kd = gpu_lib
    N, D, V = 20000, 64, 257
    h, W, lab = _inputs(N, D, V, dtype, "some", 23)
    lab[3000:17000] = -100
    ref = _ref(h, W, lab, z_loss=1e-3)
    got = kd.ce_fwd_bwd(h, W, lab, z_loss=1e-3, chunk=1000, loss_per_token=True)
    _check(got, ref, dtype, h, W, lab)
    f = kd.ce_fwd(h, W, lab, z_loss=1e-3, chunk=1000)
    _check(kd.ce_bwd(h, W, lab, f["saved_logz"], z_loss=1e-3, chunk=1000), ref, dtype, h, W, lab)


def test_captured_autograd_step(gpu_lib):
    kd = gpu_lib
    h, W, lab = _inputs(200, 128, 1500, "bf16", "some", 17)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        hg, Wg = h.clone().requires_grad_(True), W.clone().requires_grad_(True)
        for _ in range(2):
            torch.autograd.grad(kd.cross_entropy(hg, Wg, lab, z_loss=1e-3), [hg, Wg])
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = kd.cross_entropy(hg, Wg, lab, z_loss=1e-3)
        gh, gw = torch.autograd.grad(loss, [hg, Wg])
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        ref = _ref(h, W, lab, z_loss=1e-3)
        _check({"loss": loss, "grad_hidden": gh, "grad_W": gw}, ref, "bf16")


def test_refusals(gpu_lib):
    kd = gpu_lib
    h, W, lab = _inputs(20, 64, 100, "f32", "all", 1)
    for bad in (lambda: kd.cross_entropy(h, W, lab[:19]), lambda: kd.cross_entropy(h[:, :32], W, lab),
                lambda: kd.cross_entropy(h, W, lab[:, None]),
                lambda: kd.cross_entropy(h.t().contiguous().t(), W, lab),
                lambda: kd.cross_entropy(h, W, lab.cpu()), lambda: kd.cross_entropy(h.cpu(), W, lab),
                lambda: kd.cross_entropy(h, W, lab, schedule="other"),
                lambda: kd.cross_entropy(h, W, torch.stack([lab, lab], 1)[:, 0]),
                lambda: kd.ce_bwd(h, W, lab, torch.zeros(19, device="cuda")),
                lambda: kd.ce_bwd(h, W, lab, torch.zeros(20, device="cuda"),
                                  grad_loss=torch.ones(2, device="cuda")),
                lambda: kd.ce_fwd_bwd(h, W, lab, grad_W_out=torch.zeros(100, 32, device="cuda")),
                lambda: kd.ce_fwd_bwd(h, W, lab, accumulate_grad_W=True),
                lambda: kd.ce_bwd(h, W, lab, torch.zeros(20, device="cuda"), accumulate_grad_W=True),
                lambda: kd.ce_fwd_bwd(h, W, lab, workspace=torch.empty(9, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: kd.cross_entropy(h, W.bfloat16(), lab), lambda: kd.cross_entropy(h, W, lab.int()),
                lambda: kd.cross_entropy(h.half(), W.half(), lab)):
        with pytest.raises(TypeError):
            bad()
    for kw in (dict(z_loss=-1.0), dict(z_loss=float("nan")), dict(chunk=0),
               dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(kd.KdError):
            kd.cross_entropy(h, W, lab, **kw)


def test_head_in_a_row(gpu_lib):
    """A training step through a head rounded to 4 bits (labels and a teacher), then the
    head held so, drafted from and verified."""
    kd = gpu_lib
    N, D, V, K = 96, 256, 1200, 16
    h, W, lab = _inputs(N, D, V, "bf16", "some", 21)
    idx, tl = ki.make_teacher(N, K, V, "cuda", seed=5)
    h.requires_grad_(True)
    W.requires_grad_(True)
    Wq = kd.mx4_round(W)
    loss = kd.cross_entropy(h, Wq, lab, z_loss=1e-3) + 0.5 * kd.topk_kl_loss(h, Wq, idx, tl)
    gh, gw = torch.autograd.grad(loss, [h, W])
    from oracle import kd_topk_kl
    ref = _ref(h, Wq, lab, z_loss=1e-3)
    kl = kd_topk_kl(to64(h), to64(Wq), to64(idx), to64(tl), tau=1.0, chunk=64)
    assert abs(float(loss.detach()) - ref["loss"] - 0.5 * kl["loss"]) <= TOL["bf16"]["loss"] * float(loss.detach())
    for g, k in ((gh, "grad_hidden"), (gw, "grad_W")):
        assert rel_max(to64(g), ref[k] + 0.5 * kl[k]) <= TOL["bf16"]["grad"]
    # the head in 4 bits gives the loss's own logits
    q = kd.mx4_write(W.detach())
    z = kd.mx4_logits(h.detach(), q["codes"], q["scales"], dtype=torch.float32)
    want, mag = ho.mx4_logits(to64(h), q["codes"].cpu().numpy(), q["scales"].cpu().numpy())
    assert (np.abs(to64(z) - want) <= (D + 64) * 2.0 ** -23 * mag + 2.0 ** -24 * np.abs(want)).all()
    f = kd.ce_fwd(h.detach(), kd.mx4_read(q["codes"], q["scales"], torch.bfloat16), lab)
    ok = ((lab >= 0) & (lab < V)).cpu().numpy()
    lse = np.log(np.exp(to64(z)).sum(axis=1))
    assert (np.abs(to64(f["saved_logz"]) - lse)[ok] <= 1e-4).all()
    # 16 sequences of 5 drafted tokens and the target's 6 rows
    B, T = 16, 5
    draft = z[:B * T].view(B, T, V)
    e = kd.topk_entries(z[:B * T], K)
    oi, ov = oo.topk_entries(to64(z[:B * T]), K)
    assert np.array_equal(e["teacher_idx"].cpu().numpy(), oi)
    tokens = e["teacher_idx"][:, 0].view(B, T).contiguous()
    target = z.view(B, T + 1, V)
    u = torch.rand(B, T + 1, generator=_gen(3), device="cuda")
    got = kd.verify_draft(target, tokens, u, draft_logits=draft.contiguous())
    p = torch.softmax(target.double(), -1).cpu().numpy()
    d = torch.softmax(draft.double(), -1).cpu().numpy()
    t, uu = tokens.cpu().numpy(), u.double().cpu().numpy()
    for b in range(B):
        r = 0
        while r < T and uu[b, r] * d[b, r, t[b, r]] < p[b, r, t[b, r]]:
            r += 1
        assert int(got["accepted"][b]) == r
