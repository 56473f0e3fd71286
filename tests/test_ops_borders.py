"""The operators around the loss at values next to a border: finite masks and
extreme temperatures, every kind of NaN, draws from a mass far below the rounding
of 1, cache entries next to the reach, long streamed rows."""
import numpy as np
import pytest
import torch

from oracle import ops_oracle as oo
from tests.helpers import to64
from tests.test_ops import DT, E32, _check_topk, _check_verify, _draft, _gen, _logits


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


@pytest.mark.gpu
@pytest.mark.filterwarnings("ignore:invalid value encountered in cast")
@pytest.mark.parametrize("share", [0.0, 0.5, 0.95])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V", [(3, 3000), (3, 60000), (300, 101000), (1600, 17000), (300, 3000),
                                 (300, 60000)])
def test_every_kind_of_nan_in_every_pass(gpu_lib, N, V, dtype, share):
    """Rows that one workgroup streams (512 and 256 threads), holds, or selects behind a
    first pass, with every kind of NaN in four of five columns or in a share of them at
    any place: the oracle's entries, and its log-probabilities."""
    kd, K = gpu_lib, 40
    x = _logits(N, V, dtype, 15)
    bits = x.view(torch.int16 if dtype == "bf16" else torch.int32)
    kinds = (0x7f81, -0x7f, 0x7fc0, -1) if dtype == "bf16" else (0x7f800001, -0x7fffff, 0x7fc00000, -1)
    for i, b in enumerate(kinds):
        if share:
            bits[torch.rand(N, V, generator=_gen(20 + i), device="cuda") < 1 - (1 - share) ** 0.25] = b
        else:
            bits[:, i::5] = b
    got, plain = kd.topk_entries(x, K, logprobs=True), kd.topk_entries(x, K)
    assert torch.equal(got["teacher_idx"], plain["teacher_idx"])
    some = torch.tensor(sorted({0, 1, 2, N // 3, N // 2, N - 2, N - 1}), device="cuda")
    a = x[some].float().cpu().numpy()
    idx, val = oo.topk_entries(a, K)
    assert np.array_equal(to64(plain["teacher_idx"][some]), idx)
    assert np.array_equal(to64(plain["teacher_logit"][some]), val)
    _, val = oo.topk_entries(a, K, True)
    # (as in _check_topk)
    assert np.all(np.abs(to64(got["teacher_logit"][some]) - val)
                  <= 64 * E32 + 3 * E32 * np.abs(val))
    # all rows: what is no number nowhere, each row largest first
    v = plain["teacher_logit"]
    assert bool(torch.isfinite(v).all()) and bool((v[:, 1:] <= v[:, :-1]).all())


@pytest.mark.gpu
@pytest.mark.filterwarnings("ignore:invalid value encountered in cast")
@pytest.mark.parametrize("tau", [1.0, 1e-30])
@pytest.mark.parametrize("K", [0, 20])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_verify_every_kind_of_nan(gpu_lib, dtype, K, tau):
    """The same for both distributions of a verification, also where no stretch is fast."""
    B, T, V = 6, 3, 9001
    target, tokens, u, draft = _draft(B, T, V, K, dtype, 16, ld=5)
    for j, t in enumerate((target, draft.get("draft_logits", draft.get("draft_logit")))):
        f32 = t.dtype == torch.float32
        bits = t.view(torch.int32 if f32 else torch.int16)
        kinds = (0x7f800001, -0x7fffff, 0x7fc00000, -1) if f32 else (0x7f81, -0x7f, 0x7fc0, -1)
        for i, b in enumerate(kinds):
            bits[torch.rand(t.shape, generator=_gen(30 + 4 * j + i), device="cuda") < 0.2] = b
    _check_verify(gpu_lib, target, tokens, u, draft, tau)
