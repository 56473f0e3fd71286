"""What cross entropy does under autograd's other modes: forward mode, which it has
no rule for, and second derivatives, which it does not have."""
import pytest
import torch
import torch.autograd.forward_ad as fw

pytestmark = pytest.mark.gpu

SCHEDULES = ["fused", "recompute"]


def _inputs(dtype=torch.float32):
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    h = torch.randn(40, 64, generator=g, device="cuda").to(dtype)
    W = torch.randn(90, 64, generator=g, device="cuda").to(dtype)
    return h, W, torch.randint(0, 90, (40,), generator=g, device="cuda")


@pytest.mark.parametrize("schedule", SCHEDULES)
@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("which", [0, 1])
def test_forward_mode_is_refused(gpu_lib, schedule, grad, which):
    """A tensor that carries a tangent: an error, never a loss without one (no_grad leaves
    forward mode on)."""
    x = list(_inputs())
    with fw.dual_level():
        x[which] = fw.make_dual(x[which], torch.ones_like(x[which]))
        with torch.set_grad_enabled(grad), pytest.raises(NotImplementedError):
            gpu_lib.cross_entropy(*x, schedule=schedule)


@pytest.mark.parametrize("schedule", SCHEDULES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_second_derivative_is_refused(gpu_lib, schedule, dtype):
    """With create_graph the gradients are the same ones, and a derivative of them raises
    instead of being taken for 0."""
    h, W, lab = _inputs(dtype)
    h.requires_grad_(True)
    W.requires_grad_(True)
    want = torch.autograd.grad(gpu_lib.cross_entropy(h, W, lab, schedule=schedule), [h, W])
    loss = gpu_lib.cross_entropy(h, W, lab, schedule=schedule)
    got = torch.autograd.grad(loss, [h, W], create_graph=True)
    for a, b in zip(got, want):
        assert a.dtype == dtype and torch.equal(a.detach(), b) and not b.requires_grad
    for a in got:
        with pytest.raises(RuntimeError, match="second derivative"):
            ((h.float() ** 2).sum() + (a.float() ** 2).sum()).backward()
    # one of the two alone
    g, = torch.autograd.grad(gpu_lib.cross_entropy(h.detach(), W, lab, schedule=schedule), [W],
                             create_graph=True)
    assert torch.equal(g.detach(), want[1])
    with pytest.raises(RuntimeError, match="second derivative"):
        g.sum().backward()


@pytest.mark.parametrize("schedule", SCHEDULES)
def test_loss_alone(gpu_lib, schedule):
    """No gradient wanted: the loss, by the same bits, with grad mode on or off."""
    h, W, lab = _inputs()
    want = gpu_lib.ce_fwd_bwd(h, W, lab, grad_hidden=False, grad_W=False)["loss"]
    assert torch.equal(gpu_lib.cross_entropy(h, W, lab, schedule=schedule), want)
    h.requires_grad_(True)
    with torch.no_grad():
        got = gpu_lib.cross_entropy(h, W, lab, schedule=schedule)
    assert torch.equal(got, want) and not got.requires_grad
