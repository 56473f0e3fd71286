"""Gradients of the bf16 cross entropy of one projection, whose label's part is formed
in fp32 where the gradients are: entry by entry against fp64."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as ho
from tests.helpers import to64

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -8  # half a step of bf16, relative to the value


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _inputs(N, D, V, labels, seed, far=0.0):
    h = torch.randn(N, D, generator=_gen(seed), device="cuda")
    W = torch.randn(V, D, generator=_gen(seed + 1), device="cuda") * 0.05
    lab = torch.randint(0, V, (N,), generator=_gen(seed + 2), device="cuda")
    if labels == "one":
        lab.fill_(V // 2)
    elif labels == "few":
        lab = lab % 5
    if labels != "all":
        odd = torch.tensor([-100, V, 2 ** 32, -2 ** 63], device="cuda")
        out = torch.rand(N, generator=_gen(seed + 3), device="cuda") < 0.3
        out[0] = False
        lab = torch.where(out, odd[torch.arange(N, device="cuda") % 4], lab)
    if far:
        # the labels' logits far above the others: tokens nearly certain of them
        h[:, 0] = 1.0
        W[:, 0] = 0.0
        W[lab.clamp(0, V - 1).unique(), 0] = far
    return h.bfloat16(), W.bfloat16(), lab


def _bounds(h, W, lab, z):
    """fp64 gradients, and what a call may be off by before its results are rounded.
    Every entry of dL/dz but the label's is rounded to bf16 once (a row that fell back
    to its own reference: twice) and, for grad_W, met by a hidden row times its factor,
    rounded once: less than 2.05 half steps of the product either way, of the sum of
    magnitudes without the label's. Probabilities are off by `noise` of themselves (16
    roundings of fp32 of the logits' and the reference's size), sums of n terms by
    n 2^-24 of their magnitudes. The label's part is fp32: its weight, coef ((1 + 2 z
    ln Z) q - 1), is off by that of q and by 8 roundings."""
    h, W, lab = to64(h), to64(W), lab.cpu().numpy()
    N, V = h.shape[0], W.shape[0]
    ref = ho.cross_entropy(h, W, lab, z_loss=z)
    ok = (lab >= 0) & (lab < V)
    at, rows = np.where(ok, lab, 0), np.arange(N)
    x = h @ W.T
    lz = np.log(np.exp(x - x.max(1, keepdims=True)).sum(1)) + x.max(1)
    coef = ref["weight"]
    size = np.maximum(np.abs(lz), np.abs(x).max(1)) + 24 * np.log(2.0)
    noise = 16 * 2.0 ** -24 * size
    # (the z-loss's weight has ln Z in it)
    m = np.abs(1 + 2 * z * lz) + 2 * z * noise
    G = np.exp(x - lz[:, None]) * (coef * m)[:, None]
    q = ref["q_label"] * coef * m
    w = np.abs((1 + 2 * z * lz) * ref["q_label"] - 1) * coef
    w_off = np.where(ok, q * (noise + 2 * z * noise / m) + 8 * 2.0 ** -24 * (w + q), 0.0)
    G[rows, at] = np.where(ok, 0.0, G[rows, at])
    each = 2.05 * STEP + noise + 2 * z * noise / m
    aH, aW = np.abs(h), np.abs(W)
    eH = (G * (each + V * 2.0 ** -24)[:, None]) @ aW + (w_off + 4 * 2.0 ** -24 * w)[:, None] * aW[at]
    eW = (G * (each + N * 2.0 ** -24)[:, None]).T @ aH
    np.add.at(eW, at[ok], ((w_off + N * 2.0 ** -24 * w)[:, None] * aH)[ok])
    return ref, {"grad_hidden": eH + 2.0 ** -24 * np.abs(ref["grad_hidden"]),
                 "grad_W": eW + 2.0 ** -24 * np.abs(ref["grad_W"])}


CASES = [(1, 64, 5, 4096, "all", 0.0), (300, 128, 1500, 128, "some", 1e-3),
         (500, 192, 1031, 4096, "one", 0.0), (70, 2112, 515, 4096, "few", 1e-2),
         (9000, 64, 300, 1000, "some", 1e-4), (4097, 128, 257, 4096, "all", 0.0),
         (1000, 1024, 3001, 300, "few", 0.0), (5000, 64, 999, 5000, "one", 1e-3)]


@pytest.mark.parametrize("N,D,V,chunk,labels,z", CASES)
def test_fp32_gradients(gpu_lib, N, D, V, chunk, labels, z):
    kd = gpu_lib
    h, W, lab = _inputs(N, D, V, labels, N + V)
    ref, bound = _bounds(h, W, lab, z)
    got = kd.ce_fwd_bwd(h, W, lab, z_loss=z, chunk=chunk, grad_hidden_f32=True)
    for k in bound:
        err = np.abs(to64(got[k]) - ref[k])
        assert (err <= bound[k]).all(), (k, (err / np.maximum(bound[k], 1e-300)).max())
    ignored = (lab < 0) | (lab >= V)
    assert not got["grad_hidden"][ignored].any()
    again = kd.ce_fwd_bwd(h, W, lab, z_loss=z, chunk=chunk, grad_hidden_f32=True)
    for k in got:
        assert torch.equal(got[k], again[k]), k
    # either gradient alone, and one added to what is there (a sum with 1 rounds once more)
    one = kd.ce_fwd_bwd(h, W, lab, z_loss=z, chunk=chunk, grad_hidden_f32=True, grad_W=False)
    assert torch.equal(one["grad_hidden"], got["grad_hidden"])
    one = kd.ce_fwd_bwd(h, W, lab, z_loss=z, chunk=chunk, grad_hidden_f32=True, grad_hidden=False)
    assert torch.equal(one["grad_W"], got["grad_W"])
    acc = torch.ones(V, D, device="cuda")
    kd.ce_fwd_bwd(h, W, lab, z_loss=z, chunk=chunk, grad_hidden_f32=True, grad_W_out=acc,
                  accumulate_grad_W=True)
    # (each group of tokens and each 4096 of them adds once)
    adds = 2 * (N // 4096 + N // chunk + 2)
    err = np.abs(to64(acc) - 1 - ref["grad_W"])
    assert (err <= bound["grad_W"] + adds * 2.0 ** -24 * (1 + np.abs(ref["grad_W"]))).all()


@pytest.mark.parametrize("far", [2.0, 8.0, 20.0, 60.0])
def test_certain_tokens(gpu_lib, far):
    kd = gpu_lib
    h, W, lab = _inputs(400, 128, 700, "few", 3, far)
    ref, bound = _bounds(h, W, lab, 1e-4)
    got = kd.ce_fwd_bwd(h, W, lab, z_loss=1e-4, grad_hidden_f32=True)
    for k in bound:
        assert (np.abs(to64(got[k]) - ref[k]) <= bound[k]).all(), k


@pytest.mark.parametrize("N,D,V,chunk,labels,z", CASES)
def test_autograd(gpu_lib, N, D, V, chunk, labels, z):
    """The default schedule's gradients: those, rounded once."""
    kd = gpu_lib
    h, W, lab = _inputs(N, D, V, labels, N + V)
    ref, bound = _bounds(h, W, lab, z)
    h.requires_grad_(True)
    W.requires_grad_(True)
    loss = kd.cross_entropy(h, W, lab, z_loss=z, chunk=chunk)
    got = dict(zip(("grad_hidden", "grad_W"), torch.autograd.grad(loss, [h, W])))
    for k in bound:
        err = np.abs(to64(got[k]) - ref[k])
        b = bound[k] + STEP * (np.abs(ref[k]) + bound[k])
        assert (err <= b).all(), (k, (err / np.maximum(b, 1e-300)).max())


def test_graph(gpu_lib):
    """A captured step replays with new inputs, on workspaces full of anything."""
    kd = gpu_lib
    N, D, V = 300, 128, 2000
    h, W, lab = _inputs(N, D, V, "few", 13)
    ws = torch.empty(kd.ce_workspace_size(N, D, V, 128), dtype=torch.uint8, device="cuda")
    out = kd.ce_fwd_bwd(h, W, lab, chunk=128, workspace=ws, grad_hidden_f32=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kd.ce_fwd_bwd(h, W, lab, chunk=128, workspace=ws, out=out, grad_hidden_f32=True)
    for seed in (20, 30, 40):
        h2, _, lab2 = _inputs(N, D, V, "some", seed)
        h.copy_(h2)
        lab.copy_(lab2)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        want = kd.ce_fwd_bwd(h, W, lab, chunk=128, grad_hidden_f32=True)
        for k in want:
            assert torch.equal(out[k], want[k]), k


def test_rows_not_a_number(gpu_lib):
    """An ignored token's hidden row reaches no label's part, whatever its label."""
    kd = gpu_lib
    h, W, lab = _inputs(200, 64, 100, "few", 7)
    want = kd.ce_fwd_bwd(h, W, lab, grad_hidden_f32=True)
    h2 = h.clone()
    h2[(lab < 0) | (lab >= 100)] = float("nan")
    got = kd.ce_fwd_bwd(h2, W, lab, grad_hidden_f32=True)
    for k in want:
        assert torch.equal(got[k], want[k]), k
