"""The operators around the loss at values next to a border: finite masks and
extreme temperatures, every kind of NaN, draws from a mass far below the rounding
of 1, cache entries next to the reach, long streamed rows."""
import pytest
import torch

from tests.test_ops import DT, _check_verify, _gen


@pytest.mark.gpu
@pytest.mark.parametrize("K", [0, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask,tau,V,columns", [
    (-1e7, 0.35, 4096, {100: 0.0, 3000: 5.0}), (-65504.0, 0.002, 4096, {100: 0.0, 3000: 5.0}),
    (-1e4, 5e-4, 4096, {100: 0.0, 3000: 5.0}), (-1e4, 5e-4, 6000, {3: 0.0, 1600: 4.0, 5999: 4.5})])
def test_verify_finite_mask(gpu_lib, mask, tau, V, columns, dtype, K):
    """Constrained decoding: a few columns in stretches of 2048 that are masked by a
    finite number, beginning with masked ones or not. The largest logit, hundreds of
    powers of two above its stretch's first ones, has the row's probability."""
    print(f"[mask] {mask} {tau} {V} {dtype} K={K}", flush=True)
    B, T = 4, 2
    z = torch.full((B, T + 1, V), mask, device="cuda")
    d = torch.full((B, T, V), mask, device="cuda")
    for v, x in columns.items():
        z[:, :, v] = x
        d[:, :, v] = 1.0
    z, d = z.to(DT[dtype]), d.to(DT[dtype])
    tokens = torch.tensor([list(columns)[:2], list(columns)[1::-1]] * 2, dtype=torch.int32,
                          device="cuda")
    u = torch.rand(B, T + 1, generator=_gen(5), device="cuda")
    draft = dict(draft_logits=d)
    if K:
        e = d.float().topk(K, dim=2)
        draft = dict(draft_idx=e.indices.int().contiguous(), draft_logit=e.values.contiguous())
    _check_verify(gpu_lib, z, tokens, u, draft, tau)


@pytest.mark.gpu
@pytest.mark.parametrize("K", [0, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", [-1e4, -65504.0, -1e6, -1e7])
def test_verify_finite_mask_sweep(gpu_lib, mask, dtype, K):
    """Finite masks and temperatures from 1e-4 to 1, up to four columns left of each row
    at any place."""
    B, T, V = 12, 2, 9001
    for i, tau in enumerate((1e-4, 5e-4, 2e-3, 0.01, 0.05, 0.35, 1.0)):
        g = _gen(1000 + i)
        at = torch.randint(0, V, (B, T + 1, 4), generator=g, device="cuda")
        x = 4.0 * torch.randn(B, T + 1, 4, generator=g, device="cuda")
        x += tau * torch.randn(B, T + 1, 4, generator=g, device="cuda")
        z = torch.full((B, T + 1, V), mask, device="cuda").scatter_(2, at, x)
        near = x[:, :T] + tau * torch.randn(B, T, 4, generator=g, device="cuda")
        d = torch.full((B, T, V), mask, device="cuda").scatter_(2, at[:, :T], near).to(DT[dtype])
        tokens = at[:, :T, 0].int().contiguous()
        u = torch.rand(B, T + 1, generator=g, device="cuda")
        draft = dict(draft_logits=d)
        if K:
            e = d.float().topk(K, dim=2)
            draft = dict(draft_idx=e.indices.int().contiguous(), draft_logit=e.values.contiguous())
        print(f"[mask sweep] {mask} tau={tau} {dtype} K={K}", flush=True)
        _check_verify(gpu_lib, z.to(DT[dtype]), tokens, u, draft, tau)
