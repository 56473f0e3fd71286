"""The operators around the loss on the GPU against the fp64 oracle: top-K
entries, the teacher cache, 8-bit checkpoints, draft verification."""
import numpy as np
import pytest
import torch

import kd_inputs as ki
from oracle import ops_oracle as oo
from tests.helpers import to64

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
E32 = 2.0 ** -24  # half a step of fp32, relative


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _logits(N, V, dtype, seed, ld=None, offset=0, std=5.0):
    """[N, V] view with rows `ld` apart that starts `offset` elements into its storage."""
    ld = V if ld is None else ld
    flat = torch.full((offset + N * ld,), float("nan"), dtype=DT[dtype], device="cuda")
    x = flat[offset:].view(N, ld)[:, :V]
    x.copy_(torch.randn(N, V, generator=_gen(seed), device="cuda") * std)
    return x


SPECIALS = ("plain", "ties", "constant", "masked", "lowest", "nan", "inf", "ascending", "wide",
            "logprobs", "two", "halves")


def _special(x, kind):
    """Rows with the values that a selection can go wrong at, in place."""
    N, V = x.shape
    low = torch.finfo(x.dtype).min
    if kind == "ties":
        x.copy_((x / 4).round() * 4)
    elif kind == "constant":
        x.fill_(-1.5)
    elif kind == "masked":           # three columns left, in the last row none
        keep = x[:, [0, V // 2, V - 1]].clone()
        x.fill_(float("-inf"))
        x[:, [0, V // 2, V - 1]] = keep
        x[-1] = float("-inf")
    elif kind == "lowest":           # the same by the type's lowest value
        keep = x[:, [0, V // 2, V - 1]].clone()
        x.fill_(low)
        x[:, [0, V // 2, V - 1]] = keep
        x[-1] = low
    elif kind == "nan":
        x[:, ::3] = float("nan")
        x[-1] = float("nan")
    elif kind == "inf":
        x[0, V // 3] = float("inf")
        x[-1, [0, V - 1]] = float("inf")
        x[:, 1] = float("-inf")
    elif kind == "wide":             # magnitudes over the whole range, either sign
        e = torch.randint(-120, 121, (N, V), generator=_gen(3), device=x.device).float()
        x.copy_(x.sign() * torch.exp2(e))
    elif kind == "logprobs":         # one column near 0, the others far below
        x.copy_(torch.log_softmax(x.float() * 3, 1) - 1e-5)
    elif kind == "two":              # more equal ones than wanted below a few larger
        big = x > 6
        x.fill_(-2.0)
        x[big] = 3.0
    elif kind == "halves":           # the same at the end of the row only, -inf before
        x[:, V // 2:] = 1.25
        x[:, :V // 2] = float("-inf")
    elif kind == "ascending":
        x.copy_(torch.arange(V, device=x.device).to(x.dtype) * 0.5)
    return x


def _check_topk(kd, x, K):
    a = x.float().cpu().numpy().astype(np.float64)
    got = kd.topk_entries(x, K)
    lp = kd.topk_entries(x, K, logprobs=True)
    torch.cuda.synchronize()
    idx, val = oo.topk_entries(a, K)
    assert np.array_equal(to64(got["teacher_idx"]), idx)
    assert np.array_equal(to64(got["teacher_logit"]), val)
    idx, val = oo.topk_entries(a, K, True)
    assert np.array_equal(to64(lp["teacher_idx"]), idx)
    g = to64(lp["teacher_logit"])
    fin = np.isfinite(val)
    assert np.array_equal(fin, np.isfinite(g)) and np.array_equal(g[~fin], val[~fin])
    # log of the sum: each exp off by up to 4 half steps (difference, product and
    # 2^x), the sum of positive terms by one for each of the additions on its
    # longest path (32 in a lane, 6 in a wave, 9 + 6 over the segments); then the
    # logarithm, the difference and the value's own roundings
    assert np.all(np.abs(g[fin] - val[fin]) <= 64 * E32 + 3 * E32 * np.abs(val[fin]))


@pytest.mark.parametrize("kind", SPECIALS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,K,ld,offset", [
    (3, 1, 1, None, 0), (4, 7, 7, 9, 1), (5, 64, 3, None, 3), (3, 300, 300, 301, 5),
    (2, 2049, 100, 2051, 7), (3, 6500, 100, None, 0), (2, 32003, 257, 32005, 2),
    (2, 70001, 300, 70003, 1), (3, 132000, 100, None, 0), (520, 20000, 64, None, 0),
    (515, 3000, 200, 3001, 0)])
def test_topk_entries(gpu_lib, N, V, K, ld, offset, dtype, kind):
    print(f"[topk] {N} {V} {K} ld={ld} +{offset} {dtype} {kind}", flush=True)
    x = _logits(N, V, dtype, 11, ld, offset)
    if V >= 3:
        _special(x, kind)
    _check_topk(gpu_lib, x, K)


@pytest.mark.parametrize("dtype,N,V,K", [
    ("bf16", 2, 131072, 100), ("f32", 1, 131072, 100), ("bf16", 2, 1 << 20, 4096),
    ("f32", 1, (1 << 20) - 3, 1000), ("bf16", 2, 50257, 4096), ("f32", 2, 5000, 4096)])
def test_topk_entries_large(gpu_lib, dtype, N, V, K):
    print(f"[topk] {dtype} {N} {V} {K}", flush=True)
    _check_topk(gpu_lib, _logits(N, V, dtype, 12), K)


@pytest.mark.parametrize("kind", ["plain", "masked", "two", "nan"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,K,ld,offset", [(300, 101000, 60, 101001, 3), (1540, 17000, 20, None, 0),
                                             (260, 131072, 512, None, 0)])
def test_topk_entries_streamed(gpu_lib, N, V, K, ld, offset, dtype, kind):
    """Rows that their own workgroups stream: the selection of the whole against
    the oracle's on some rows, and every row against a call for it alone."""
    kd = gpu_lib
    x = _special(_logits(N, V, dtype, 14, ld, offset), kind)
    for logprobs in (False, True):
        got = kd.topk_entries(x, K, logprobs=logprobs)
        for r0 in range(0, N, 200):   # few rows take another way
            part = kd.topk_entries(x[r0:r0 + 200], K, logprobs=logprobs)
            assert torch.equal(got["teacher_idx"][r0:r0 + 200], part["teacher_idx"])
            a, b = to64(got["teacher_logit"][r0:r0 + 200]), to64(part["teacher_logit"])
            f = np.isfinite(a)
            assert np.array_equal(f, np.isfinite(b))
            # (each within 64 E32 of the sum's logarithm, see _check_topk)
            tol = 128 * E32 + 6 * E32 * np.abs(b[f]) if logprobs else 0.0
            assert np.all(np.abs(a[f] - b[f]) <= tol)
    some = torch.tensor([0, 1, N // 2, N - 1], device="cuda")
    idx, val = oo.topk_entries(x[some].float().cpu().numpy(), K)
    got = kd.topk_entries(x, K)
    assert np.array_equal(to64(got["teacher_idx"][some]), idx)
    assert np.array_equal(to64(got["teacher_logit"][some]), val)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_topk_entries_largest(gpu_lib, dtype):
    """More rows than have a workgroup of 1024 threads each, at the largest V and K."""
    kd, N, V, K = gpu_lib, 260, 1 << 20, 4096
    x = _logits(N, V, dtype, 15)
    for logprobs in (False, True):
        got = kd.topk_entries(x, K, logprobs=logprobs)
        for r in (0, N - 4):
            part = kd.topk_entries(x[r:r + 4], K, logprobs=logprobs)
            assert torch.equal(got["teacher_idx"][r:r + 4], part["teacher_idx"])
            assert torch.equal(got["teacher_logit"][r:r + 4], part["teacher_logit"])
    idx, val = oo.topk_entries(x[N - 1:].float().cpu().numpy(), K)
    got = kd.topk_entries(x, K)
    assert np.array_equal(to64(got["teacher_idx"][N - 1:]), idx)
    assert np.array_equal(to64(got["teacher_logit"][N - 1:]), val)


def test_topk_many_rows_in_batches(gpu_lib):
    """More rows than the workspace holds at a time."""
    kd, N, V, K = gpu_lib, 500000, 9, 2
    assert kd.topk_workspace_size(N, V, K) < 70 << 20
    x = _logits(N, V, "bf16", 13)
    got = kd.topk_entries(x, K)
    idx, val = oo.topk_entries(x.float().cpu().numpy(), K)
    assert np.array_equal(to64(got["teacher_idx"]), idx)
    assert np.array_equal(to64(got["teacher_logit"]), val)


@pytest.mark.parametrize("kind", SPECIALS)
@pytest.mark.parametrize("logprobs", [False, True])
@pytest.mark.parametrize("dtype,N,V,K", [("bf16", 3, 300, 8), ("f32", 4, 5003, 100),
                                          ("bf16", 3, 40000, 129), ("f32", 2, 70, 70)])
def test_teacher_cache(gpu_lib, dtype, N, V, K, logprobs, kind):
    kd = gpu_lib
    print(f"[cache] {dtype} {N} {V} {K} {logprobs} {kind}", flush=True)
    x = _special(_logits(N, V, dtype, 21), kind)
    # written into the middle of a larger cache
    entries = torch.full((N + 2, K), 7, dtype=torch.int32, device="cuda")
    scale = torch.full((N + 2, 2), 7.0, device="cuda")
    kd.teacher_cache_write(x, K, logprobs=logprobs,
                           out={"entries": entries[1:-1], "scale": scale[1:-1]})
    e, top, step = oo.cache_write(x.float().cpu().numpy(), K, logprobs)
    got_e = to64(entries).astype(np.int64) & 0xffffffff
    assert np.array_equal(got_e[1:-1], e)
    assert (got_e[[0, -1]] == 7).all() and bool((scale[[0, -1]] == 7.0).all())
    sc = to64(scale[1:-1])
    assert np.array_equal(sc[:, 1], step.astype(np.float64))
    fin = np.isfinite(top)
    assert np.array_equal(fin, np.isfinite(sc[:, 0]))
    # top as in _check_topk; exact without log-probabilities
    tol = 64 * E32 + 3 * E32 * np.abs(top[fin]) if logprobs else 0.0
    assert np.all(np.abs(sc[fin, 0] - top[fin]) <= tol)
    # read back: all rows, and rows by number (twice the same, outside the cache)
    for rows in (None, [N, 0, N + 1, -1, 1, 1, N + 2, 1 << 40, -(1 << 40)]):
        r = None if rows is None else torch.tensor(rows, device="cuda")
        t = kd.teacher_cache_read(entries, scale, rows=r)
        idx, logit, ignore = oo.cache_read(to64(entries), to64(scale), rows)
        assert np.array_equal(to64(t["teacher_idx"]), idx)
        assert np.array_equal(to64(t["ignore"]), ignore)
        g = to64(t["teacher_logit"])
        assert np.array_equal(np.isfinite(g), np.isfinite(logit))
        f = np.isfinite(logit)
        assert np.array_equal(g[f], logit[f].astype(np.float32).astype(np.float64))


def test_teacher_cache_far_rows(gpu_lib):
    """Entries past 2^32 elements of a cache (17 GB)."""
    kd, K = gpu_lib, 4096
    N = (1 << 20) + 5
    entries = torch.empty(N, K, dtype=torch.int32, device="cuda")
    scale = torch.empty(N, 2, device="cuda")
    rows = torch.tensor([N - 1, 0, 1 << 19, N - 3], device="cuda")
    for i, r in enumerate(rows.tolist()):
        entries[r] = torch.arange(K, device="cuda", dtype=torch.int32) * 4096 + i
        scale[r] = torch.tensor([10.0 * i, 0.5], device="cuda")
    t = kd.teacher_cache_read(entries, scale, rows=rows)
    for i in range(4):
        assert torch.equal(t["teacher_idx"][i], torch.arange(K, device="cuda", dtype=torch.int32))
        assert bool((t["teacher_logit"][i] == 10.0 * i - 0.5 * i).all())
    assert not bool(t["ignore"].any())


def test_large_results(gpu_lib):
    """Results beyond the caches, which are stored another way: against the rows and
    blocks one by one."""
    kd = gpu_lib
    g = _gen(25)
    N, K = 1000, 52
    e = torch.randint(0, 1 << 31, (N, K), generator=g, device="cuda").int()
    sc = torch.rand(N, 2, generator=g, device="cuda")
    sc[7, 0] = float("-inf")
    rows = torch.randint(-2, N + 2, (300001,), generator=g, device="cuda")
    t = kd.teacher_cache_read(e, sc, rows=rows)
    every = kd.teacher_cache_read(e, sc, rows=torch.arange(-2, N + 2, device="cuda"))
    for k in t:
        assert torch.equal(t[k], every[k][rows + 2]), k
    for dt in (torch.bfloat16, torch.float32):
        x = (torch.randn(50001, 1184, generator=g, device="cuda") * 7).to(dt)
        c = kd.checkpoint_write(x)
        back = kd.checkpoint_read(c["codes"], c["scales"], dt)
        for s0 in range(0, 50001, 10000):
            p = kd.checkpoint_write(x[s0:s0 + 10000])
            assert torch.equal(p["codes"], c["codes"][s0:s0 + 10000])
            assert torch.equal(p["scales"], c["scales"][s0:s0 + 10000])
            assert torch.equal(kd.checkpoint_read(p["codes"], p["scales"], dt),
                               back[s0:s0 + 10000])


# -------------------------------------------------------------- checkpoints --
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D", [(1, 32), (3, 64), (77, 768), (5, 96)])
def test_checkpoint_round_trip(gpu_lib, N, D, dtype):
    kd = gpu_lib
    x = torch.randn(N, D, generator=_gen(31), device="cuda")
    # magnitudes from far below to far above 1, block by block and inside blocks
    x *= torch.exp2(torch.randint(-40, 41, (N, D // 32, 1), generator=_gen(32), device="cuda")
                    .expand(N, D // 32, 32).reshape(N, D).float())
    x *= torch.exp2(-torch.randint(0, 24, (N, D), generator=_gen(33), device="cuda").float())
    x = x.to(DT[dtype])
    if N > 2:
        x[0, :32] = 0.0
        x[1, 3] = float("inf")
        x[2, 40] = float("nan")
        x[2, :32] = torch.finfo(DT[dtype]).max * (1 - 2 * (torch.arange(32, device="cuda") % 2))
    c = kd.checkpoint_write(x)
    want, s = oo.checkpoint(to64(x))
    assert np.array_equal(to64(c["scales"]), s)
    for out in (torch.bfloat16, torch.float32):
        got = to64(kd.checkpoint_read(c["codes"], c["scales"], out))
        assert np.array_equal(got, want, equal_nan=True)


def test_checkpoint_every_code(gpu_lib):
    """Every e4m3 code at several scales, and every bf16 magnitude's rounding."""
    kd = gpu_lib
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(1, 256).repeat(5, 1)
    scales = torch.tensor([0, 1, 127, 200, 240], dtype=torch.uint8, device="cuda")
    got = kd.checkpoint_read(codes, scales[:, None].repeat(1, 8).contiguous(), torch.float32)
    one = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        one[c] = np.nan if c & 127 == 127 else -v if c & 128 else v
    for i, s in enumerate(scales.tolist()):
        assert np.array_equal(to64(got[i]), one * 2.0 ** (s - 127), equal_nan=True)
    bits = torch.arange(0, 0x7f80, device="cuda").to(torch.int16)
    bits = torch.cat([bits, bits[:0x80]])  # (a whole number of blocks)
    x = bits.view(torch.bfloat16).view(-1, 32)
    for top in (0, 1):  # alone, and below a large value of the block
        y = x.clone()
        if top:
            y[:, 0] = 2.0 ** 14
        c = kd.checkpoint_write(y)
        want, s = oo.checkpoint(to64(y))
        assert np.array_equal(to64(c["scales"]), s)
        assert np.array_equal(to64(kd.checkpoint_read(c["codes"], c["scales"], torch.float32)), want)


# ------------------------------------------------------------- verification --
def _draft(B, T, V, K, dtype, seed, ld=0, masked=0.0, err=0.7):
    g = _gen(seed)
    target = _logits(B * (T + 1), V, dtype, seed, V + ld)
    if masked:
        target[:, torch.rand(V, generator=g, device="cuda") < masked] = float("-inf")
    target = target.unflatten(0, (B, T + 1))
    t = target[:, :T].float()
    d = (t + err * torch.randn(B, T, V, generator=g, device="cuda")).to(DT[dtype])
    # (a tenth of the tokens are any: unlikely ones are rejected)
    tokens = d.float().add(-torch.log(-torch.log(
        torch.rand(B, T, V, generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)))).argmax(2)
    tokens = torch.where(torch.rand(B, T, generator=g, device="cuda") < 0.1,
                         torch.randint(0, V, (B, T), generator=g, device="cuda"), tokens).int()
    u = torch.rand(B, T + 1, generator=g, device="cuda")
    if K:
        e = d.float().topk(K, dim=2)
        return target, tokens, u, dict(draft_idx=e.indices.int().contiguous(),
                                       draft_logit=e.values.contiguous())
    return target, tokens, u, dict(draft_logits=d)


def _dense_q(draft, V, tau):
    if "draft_logits" in draft:
        d = to64(draft["draft_logits"])
        return np.stack([[oo.softmax(r, tau) for r in s] for s in d]).reshape(*d.shape)
    i, l = to64(draft["draft_idx"]), to64(draft["draft_logit"])
    return np.stack([[oo.draft_distribution(i[b, t], l[b, t], V, tau) for t in range(i.shape[1])]
                     for b in range(i.shape[0])]).reshape(i.shape[0], i.shape[1], V)


def _check_verify(kd, target, tokens, u, draft, tau=1.0, lengths=None):
    V = target.shape[2]
    out = kd.verify_draft(target, tokens, u, lengths=lengths, tau=tau, accept_prob=True, **draft)
    torch.cuda.synchronize()
    q = _dense_q(draft, V, tau) if tokens.shape[1] else np.zeros((target.shape[0], 0, V))
    want = oo.verify_draft(to64(target), to64(tokens), to64(u), q,
                           None if lengths is None else to64(lengths), tau)
    assert np.array_equal(to64(out["accepted"]), want[1])
    assert np.array_equal(to64(out["tokens"]), want[0])
    # computed in 64 bits, rounded once: half a step of fp32, which below 2^-126 is the
    # half of 2^-149 (subnormal numbers), and 1e-12 of the 64-bit weights
    assert np.all(np.abs(to64(out["accept_prob"]) - want[2])
                  <= (E32 + 1e-12) * want[2] + 2.0 ** -150)
    return want


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,V,K,ld,tau,masked", [
    (1, 1, 2, 1, 0, 1.0, 0.0), (5, 3, 50, 50, 3, 1.0, 0.0), (7, 4, 2049, 20, 1, 0.7, 0.3),
    (3, 5, 30011, 100, 5, 1.3, 0.0), (9, 2, 5000, 513, 0, 2.0, 0.9), (2, 2, 9000, 4096, 0, 1.0, 0.0),
    (5, 3, 50, 0, 3, 1.0, 0.0), (7, 4, 2049, 0, 1, 0.7, 0.3), (3, 5, 30011, 0, 5, 1.3, 0.0),
    (4, 20, 700, 0, 0, 1.0, 0.5)])
def test_verify_draft(gpu_lib, B, T, V, K, ld, tau, masked, dtype):
    print(f"[verify] {B} {T} {V} {K} ld+{ld} tau={tau} {masked} {dtype}", flush=True)
    accepted = set()
    for seed in (41, 42):
        target, tokens, u, draft = _draft(B, T, V, K, dtype, seed, ld, masked)
        accepted |= set(_check_verify(gpu_lib, target, tokens, u, draft, tau)[1].tolist())
        n = torch.randint(-1, T + 3, (B,), generator=_gen(seed), device="cuda", dtype=torch.int32)
        _check_verify(gpu_lib, target, tokens, u, draft, tau, n)
    if B * T > 8:
        assert len(accepted) > 1


@pytest.mark.parametrize("K", [0, 30])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_verify_draft_edges(gpu_lib, dtype, K):
    """Equal distributions, all or nothing masked, infinities and what is not a
    number, tokens and indices outside the vocabulary, repeated indices, uniform
    numbers at the ends."""
    B, T, V = 8, 3, 3001
    target, tokens, u, draft = _draft(B, T, V, K, dtype, 51, ld=7)
    z = target.clone()
    z[0] = float("-inf")                       # nothing left
    z[1, 1] = torch.finfo(DT[dtype]).min       # all at the type's lowest value: uniform
    z[2, 0, 5] = float("inf")
    z[2, 1, [3, 9]] = float("inf")
    z[3, :, ::2] = float("nan")
    u[4] = 0.0
    u[5] = 1.0 - 2.0 ** -24
    tokens[6, 0] = V
    tokens[7, 1] = -5
    if K:
        draft["draft_idx"][3, :, 4] = V + 3
        draft["draft_idx"][4, :, 7] = draft["draft_idx"][4, :, 2]
        draft["draft_idx"][5, :, :] = draft["draft_idx"][5, :, :1]
        draft["draft_idx"][6, 1, 1] = -1
        draft["draft_logit"][7] = float("-inf")
        draft["draft_logit"][1, 2, 3] = float("nan")
        draft["draft_logit"][1, 1, 3] = float("inf")
    else:
        draft["draft_logits"][7] = float("-inf")
        draft["draft_logits"][5, 1] = z[5, 1]   # the draft is the target there
        draft["draft_logits"][3, :, ::3] = float("nan")
        draft["draft_logits"][1, 1, 3] = float("inf")
    _check_verify(gpu_lib, z, tokens, u, draft)
    _check_verify(gpu_lib, z, tokens, u, draft, tau=1e-30)  # greedy
    # rejected although p = q everywhere (a uniform number of 1): from p
    u[:] = 1.0
    u[:, T] = 0.5
    if not K:
        draft["draft_logits"] = z[:, :T].contiguous()
    out = gpu_lib.verify_draft(z, tokens, u, **draft)
    assert int(out["accepted"][3]) == 0
    assert 0 <= int(out["tokens"][3, 0]) < V


@pytest.mark.parametrize("K", [0, 12])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_verify_far_logits(gpu_lib, dtype, K):
    """Logits hundreds of powers of two apart inside a row's stretches of 2048
    columns, stretches that begin or end in -inf, extreme tau."""
    B, T, V = 6, 2, 9001
    target, tokens, u, draft = _draft(B, T, V, K, dtype, 55, ld=3)
    z = target.clone()
    z[0, :, 2500:2600] += 700.0               # most of a stretch far below the rest of it
    z[1, :, 4000:4010] += 3000.0
    z[2, :, :6000] = float("-inf")
    z[3, :, 2048:3500] = float("-inf")
    z[3, :, 7000:] -= 900.0
    z[4] *= 40.0
    for s in range(0, V, 2048):
        z[5, :, s:s + 1024] = float("-inf")
    tokens[0] = 2550
    tokens[1, 0] = 4003
    for tau in (1.0, 0.05, 30.0, 1e30, 1e-20):
        _check_verify(gpu_lib, z, tokens, u, draft, tau)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_verify_little_left(gpu_lib, dtype):
    """A draft that is the target but for a mass far below the rounding of 1, rejected
    for a token that neither of them has: the next one comes from that mass."""
    B, V = 16, 70001
    z = _logits(B * 2, V, dtype, 57, V + 1, std=1.0).unflatten(0, (B, 2))
    z -= 60.0
    z[:, 0, 25] = float("-inf")
    z[:, 0, 64] = 3.0
    z[:, 0, [3000, 65000]] = -45.0
    draft = dict(draft_idx=torch.full((B, 1, 1), 64, dtype=torch.int32, device="cuda"),
                 draft_logit=torch.zeros(B, 1, 1, device="cuda"))
    tokens = torch.full((B, 1), 25, dtype=torch.int32, device="cuda")
    u = torch.rand(B, 2, generator=_gen(58), device="cuda")
    _, accepted, _ = _check_verify(gpu_lib, z, tokens, u, draft)
    assert not accepted.any()
    # and with a mass of 2^-12, near where the way changes
    z[:, 0, 40000] = 3.0 - 12 * np.log(2.0)
    _check_verify(gpu_lib, z, tokens, u, draft)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_verify_without_draft(gpu_lib, dtype):
    """T = 0: a draw from the target alone; and B = 0."""
    target, tokens, u, _ = _draft(6, 0, 4099, 0, dtype, 61, ld=1)
    _check_verify(gpu_lib, target, tokens, u, {})
    out = gpu_lib.verify_draft(target[:0], tokens[:0], u[:0])
    assert out["tokens"].shape == (0, 1)


def test_verify_draft_large_vocabulary(gpu_lib):
    for K in (0, 100):
        target, tokens, u, draft = _draft(2, 2, 1 << 20, K, "bf16", 71)
        _check_verify(gpu_lib, target, tokens, u, draft)


@pytest.mark.parametrize("V,K", [(5000, 4096), (1 << 20, 4096), (300, 0)])
def test_verify_longest_draft(gpu_lib, V, K):
    """T = 1024 places, the most entries: any, all, half of them, all but the last kept."""
    B, T = 1, 1024 if V < 1 << 20 else 20
    target, tokens, u, draft = _draft(B, T, V, K, "bf16", 72, err=0.1)
    _check_verify(gpu_lib, target, tokens, u, draft)
    u[:, :T] = 0.0   # kept wherever the target has the token
    for lengths in (None, torch.tensor([T // 2], dtype=torch.int32, device="cuda")):
        want = _check_verify(gpu_lib, target, tokens, u, draft, lengths=lengths)
        assert want[1][0] == (T if lengths is None else T // 2)
    tokens[0, T - 1] = -1
    assert _check_verify(gpu_lib, target, tokens, u, draft)[1][0] == T - 1


def test_verify_draft_follows_the_target(gpu_lib):
    """Over many uniform numbers the token that comes out has the target's
    probabilities, whatever the draft: counts within 6 standard deviations."""
    kd, V, B = gpu_lib, 12, 200000
    g = _gen(81)
    z = torch.randn(1, 2, V, generator=g, device="cuda")
    d = torch.randn(1, 1, V, generator=g, device="cuda")
    p, q = torch.softmax(z[0, 0].double(), 0), torch.softmax(d[0, 0].double(), 0)
    tokens = torch.multinomial(q.expand(1, V), B, replacement=True, generator=g).view(B, 1).int()
    u = torch.rand(B, 2, generator=g, device="cuda")
    for draft in (dict(draft_logits=d.expand(B, 1, V).contiguous()),
                  dict(draft_idx=torch.arange(V, device="cuda").int().expand(B, 1, V).contiguous(),
                       draft_logit=d.expand(B, 1, V).contiguous())):
        out = kd.verify_draft(z.expand(B, 2, V).contiguous(), tokens, u, **draft)
        n = torch.bincount(out["tokens"][:, 0].long(), minlength=V).double()
        assert bool(((n - B * p).abs() <= 6 * (B * p * (1 - p)).sqrt()).all())


@pytest.mark.filterwarnings("ignore:invalid value encountered in cast")
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [2, 300])
def test_every_kind_of_nan(gpu_lib, N, dtype):
    """Quiet and signalling, of either sign, first in a vector or not: all count as -inf."""
    kd, V, K = gpu_lib, 101000, 40
    x = _logits(N, V, dtype, 15)
    bits = x.view(torch.int16 if dtype == "bf16" else torch.int32)
    kinds = (0x7f81, -0x7f, 0x7fc0, -1) if dtype == "bf16" else (0x7f800001, -0x7fffff, 0x7fc00000, -1)
    for i, b in enumerate(kinds):
        bits[:, i::5] = b
    _check_topk(kd, x[:2], K)
    got = kd.topk_entries(x, K, logprobs=True)
    want = kd.topk_entries(x[:200], K, logprobs=True)   # (few rows take another way)
    assert torch.equal(got["teacher_idx"][:200], want["teacher_idx"])
    assert bool(torch.isfinite(got["teacher_logit"]).all())
    target, tokens, u, draft = _draft(2, 2, 9001, 0, dtype, 16)
    for t in (target, draft["draft_logits"]):
        b = t.view(torch.int16 if dtype == "bf16" else torch.int32)
        for i, k in enumerate(kinds):
            b[:, :, i::7] = k
    _check_verify(kd, target, tokens, u, draft)


# ------------------------------------------------------- streams and graphs --
def test_graph_replays_and_streams(gpu_lib):
    """Captured calls replay to the eager results between eager work, and a call on
    another stream gives the same bits."""
    kd, B, T, V, K = gpu_lib, 6, 3, 9001, 40
    target, tokens, u, draft = _draft(B, T, V, K, "bf16", 91)
    dense = _draft(B, T, V, 0, "bf16", 91)[3]
    rows = target[:, 0].contiguous()
    h = ki.make_hidden(33, 128, torch.bfloat16, "cuda", seed=5)

    def calls():
        c = kd.teacher_cache_write(rows, K, logprobs=True)
        k = kd.checkpoint_write(h)
        res = dict(kd.topk_entries(rows, K), **c)
        res.update({"r_" + n: t for n, t in kd.teacher_cache_read(c["entries"], c["scale"]).items()})
        res.update(k, back=kd.checkpoint_read(k["codes"], k["scales"], h.dtype))
        res.update(kd.verify_draft(target, tokens, u, accept_prob=True, **draft))
        res.update({"d_" + n: t for n, t in
                    kd.verify_draft(target, tokens, u, accept_prob=True, **dense).items()})
        return res
    eager = calls()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = calls()
    s.synchronize()
    for n in eager:
        assert torch.equal(other[n], eager[n]), n
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = calls()
    for rep in range(3):
        for t in captured.values():
            t.zero_()
        kd.topk_entries(rows * 0.5, K)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for n in eager:
            assert torch.equal(captured[n], eager[n]), (rep, n)


def test_bindings_refuse(gpu_lib):
    """Shapes, dtypes, layouts and devices that the library could not check."""
    kd = gpu_lib
    x = _logits(4, 100, "bf16", 1)
    bad = [lambda: kd.topk_entries(x.cpu(), 3), lambda: kd.topk_entries(x[0], 3),
           lambda: kd.topk_entries(x.t(), 3), lambda: kd.topk_entries(x[:, ::2], 3),
           lambda: kd.topk_entries(x[:1].expand(4, 100), 3),
           lambda: kd.topk_entries(x, 3, out={"teacher_idx": torch.empty(4, 4, dtype=torch.int32,
                                                                         device="cuda")}),
           lambda: kd.topk_entries(x, 3, workspace=torch.empty(10, device="cuda")),
           lambda: kd.teacher_cache_write(x, 3, out={"scale": torch.empty(4, 1, device="cuda")})]
    c = kd.teacher_cache_write(x, 3)
    bad += [lambda: kd.teacher_cache_read(c["entries"], c["scale"][:3]),
            lambda: kd.teacher_cache_read(c["entries"].long(), c["scale"]),
            lambda: kd.teacher_cache_read(c["entries"], c["scale"],
                                          rows=torch.zeros(2, dtype=torch.int32, device="cuda")),
            lambda: kd.teacher_cache_read(c["entries"], c["scale"], rows=torch.zeros(2, dtype=torch.int64)),
            lambda: kd.teacher_cache_read(c["entries"][:, :2], c["scale"])]
    h = torch.zeros(4, 64, device="cuda")
    k = kd.checkpoint_write(h)
    bad += [lambda: kd.checkpoint_write(h.t()), lambda: kd.checkpoint_write(h.cpu()),
            lambda: kd.checkpoint_read(k["codes"], k["scales"][:, :1], torch.float32),
            lambda: kd.checkpoint_read(k["codes"], k["scales"], torch.float32, out=h.bfloat16())]
    target, tokens, u, draft = _draft(2, 3, 50, 5, "bf16", 2)
    dense = _draft(2, 3, 50, 0, "bf16", 2)[3]
    bad += [lambda: kd.verify_draft(target, tokens, u),
            lambda: kd.verify_draft(target, tokens, u, **draft, **dense),
            lambda: kd.verify_draft(target, tokens, u, draft_idx=draft["draft_idx"]),
            lambda: kd.verify_draft(target, tokens, u[:, :3], **draft),
            lambda: kd.verify_draft(target[:, :0], tokens[:, :0], u[:, :0], **draft),
            lambda: kd.verify_draft(target[0], tokens, u, **draft),
            lambda: kd.verify_draft(target.transpose(0, 1), tokens, u, **draft),
            lambda: kd.verify_draft(target, tokens.long(), u, **draft),
            lambda: kd.verify_draft(target, tokens, u, draft_logits=dense["draft_logits"].float()),
            lambda: kd.verify_draft(target, tokens, u, lengths=torch.zeros(2, device="cuda"), **draft)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was not refused")
    with pytest.raises(TypeError):
        kd.topk_entries(x.half(), 3)
    with pytest.raises(kd.KdError):
        kd.topk_entries(x, 101)
    with pytest.raises(kd.KdError):
        kd.verify_draft(target, tokens, u, tau=0.0, **draft)


def test_calls_on_two_streams_at_once(gpu_lib):
    """Calls in flight together on two streams, each with its own workspace, and two
    captured graphs that share one workspace replayed one after the other."""
    kd, B, T, V, K = gpu_lib, 40, 3, 50001, 60
    cases = [_draft(B, T, V, K, "bf16", seed) for seed in (101, 102)]
    rows = [c[0][:, 0].contiguous() for c in cases]
    wants = [(kd.topk_entries(r, K, logprobs=True), kd.verify_draft(*c[:3], accept_prob=True, **c[3]))
             for r, c in zip(rows, cases)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append((kd.topk_entries(rows[i], K, logprobs=True),
                               kd.verify_draft(*cases[i][:3], accept_prob=True, **cases[i][3])))
    torch.cuda.synchronize()
    for i in range(2):
        for pair in got[i]:
            for a, b in zip(pair, wants[i]):
                assert all(torch.equal(a[k], b[k]) for k in b)
    ws = torch.empty(max(kd.topk_workspace_size(B, V, K), kd.verify_workspace_size(B, T, V, K)),
                     dtype=torch.uint8, device="cuda")
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = (kd.topk_entries(rows[i], K, logprobs=True, workspace=ws),
                   kd.verify_draft(*cases[i][:3], accept_prob=True, workspace=ws, **cases[i][3]))
        graphs.append((g, out))
    for _ in range(3):
        for i, (g, out) in enumerate(graphs):
            for o in out:
                for t in o.values():
                    t.zero_()
            g.replay()
        torch.cuda.synchronize()
        for (_, out), want in zip(graphs, wants):
            for a, b in zip(out, want):
                assert all(torch.equal(a[k], b[k]) for k in b)


@pytest.mark.parametrize("seed", range(12))
def test_sweep(gpu_lib, seed):
    """Seeded problems of any size: selections and verifications against the oracle."""
    import random
    kd, rng = gpu_lib, random.Random(seed)
    for _ in range(4):
        V = int(round(2 ** rng.uniform(0, 16.2)))
        N = rng.choice([1, 2, 5, 270]) if V < 3000 else rng.choice([1, 3])
        K = rng.randint(1, min(V, rng.choice([3, 40, 700])))
        dtype, pad, offset = rng.choice(["bf16", "f32"]), rng.randint(0, 9), rng.randint(0, 7)
        kind = rng.choice(SPECIALS if V >= 3 else ("plain",))
        print(f"[sweep] topk {N} {V} {K} +{pad} +{offset} {dtype} {kind}", flush=True)
        _check_topk(kd, _special(_logits(N, V, dtype, seed, V + pad, offset), kind)
                    if kind != "plain" else _logits(N, V, dtype, seed, V + pad, offset), K)
    for _ in range(4):
        V = int(round(2 ** rng.uniform(1, 15)))
        B, T = rng.randint(1, 9), rng.randint(1, 6)
        K = rng.choice([0, rng.randint(1, min(V, rng.choice([1, 30, 600])))])
        dtype, ld = rng.choice(["bf16", "f32"]), rng.randint(0, 9)
        tau, masked = rng.choice([0.3, 0.9, 1.0, 2.5]), rng.choice([0.0, 0.4, 0.95])
        print(f"[sweep] verify {B} {T} {V} {K} +{ld} {dtype} {tau} {masked}", flush=True)
        target, tokens, u, draft = _draft(B, T, V, K, dtype, seed + 200, ld, masked)
        n = torch.randint(0, T + 1, (B,), generator=_gen(seed), device="cuda", dtype=torch.int32)
        _check_verify(kd, target, tokens, u, draft, tau, rng.choice([None, n]))
