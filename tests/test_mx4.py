"""4-bit microscaled matrices and logits with a head of them on the GPU against
the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as ho
from tests.helpers import to64

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step, relative to the value


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _edges(dtype):
    """Blocks at the borders of scales and codes."""
    f = torch.finfo(DT[dtype])
    rows = []
    up = 1.0 + f.eps
    for e in (-149, -133, -130, -127, -126, -125, -124, -100, -1, 0, 3, 60, 124, 125):
        for top in (6.0, 6.0 * up, 3.0, 3.0 * up, 4.0, 7.0, 1.0):
            b = torch.linspace(-1.0, 1.0, 32, dtype=torch.float64) * top
            b[:8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.0]) * top / 6.0
            b[8] = top
            b[9] = -0.0
            x = b * 2.0 ** e
            rows.append(x.clamp(-f.max, f.max).to(DT[dtype]))
    rows.append(torch.zeros(32, dtype=DT[dtype]))
    rows.append(torch.full((32,), f.max, dtype=DT[dtype]))
    rows.append(torch.full((32,), -f.max, dtype=DT[dtype]))
    rows.append(torch.full((32,), f.smallest_normal, dtype=DT[dtype]))
    for bad in (float("inf"), float("-inf"), float("nan")):
        x = torch.ones(32, dtype=DT[dtype])
        x[31] = bad
        rows.append(x)
    n = len(rows) // 4 * 4
    return torch.stack(rows[-n:]).reshape(-1, 128).cuda()


def _same(got, want):
    g, w = to64(got), want
    assert g.shape == w.shape
    assert np.array_equal(np.isnan(g), np.isnan(w))
    ok = ~np.isnan(w)
    assert np.array_equal(g[ok], w[ok])


def _check_write(x):
    kd = pytest.importorskip("paper_2608_03796_amd")
    q = kd.mx4_write(x)
    codes, scales = ho.mx4_write(to64(x))
    assert np.array_equal(q["scales"].cpu().numpy(), scales)
    nan = np.repeat(scales == 255, 16, axis=1)
    assert np.array_equal(np.where(nan, 0, q["codes"].cpu().numpy()), np.where(nan, 0, codes))
    for t in DT.values():
        _same(kd.mx4_read(q["codes"], q["scales"], t), ho.mx4_read(codes, scales))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_write_read_edges(gpu_lib, dtype):
    _check_write(_edges(dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D", [(1, 32), (3, 96), (77, 800), (2, 65536), (130, 1024)])
def test_write_read(gpu_lib, dtype, N, D):
    g = _gen(N + D)
    x = torch.randn(N, D, generator=g, device="cuda")
    x *= torch.exp2(torch.randint(-20, 20, (N, 1), generator=g, device="cuda").float())
    _check_write(x.to(DT[dtype]))


def test_write_read_large(gpu_lib):
    """Over the size from which results pass by the caches, some blocks against the
    oracle and all against their own rounding."""
    kd = gpu_lib
    x = torch.randn(12000, 4096, generator=_gen(5), device="cuda").to(torch.bfloat16)
    q = kd.mx4_write(x)
    back = kd.mx4_read(q["codes"], q["scales"], torch.bfloat16)
    part = [0, 6000, 11999]
    codes, scales = ho.mx4_write(to64(x[part]))
    _same(back[part], ho.mx4_read(codes, scales))
    # rounding what is already rounded changes nothing
    again = kd.mx4_write(back)
    assert torch.equal(kd.mx4_read(again["codes"], again["scales"], torch.bfloat16), back)
    scale = torch.exp2(q["scales"].float() - 127).repeat_interleave(32, dim=1)
    err = (back.float() - x.float()).abs()
    assert bool((err <= torch.maximum(0.2 * x.float().abs(), 0.25 * scale) * (1 + 2 ** -20)).all())


def test_write_empty(gpu_lib):
    kd = gpu_lib
    q = kd.mx4_write(torch.empty(0, 64, device="cuda"))
    assert q["codes"].shape == (0, 32) and q["scales"].shape == (0, 2)
    assert kd.mx4_read(q["codes"], q["scales"], torch.float32).shape == (0, 64)


def test_read_every_code_and_scale(gpu_lib):
    kd = gpu_lib
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).reshape(1, 16, 16)
    codes = codes.expand(256, 16, 16).reshape(256, 256).contiguous()
    scales = torch.arange(256, dtype=torch.int32).to(torch.uint8)[:, None].expand(256, 16).contiguous()
    want = ho.mx4_read(codes.numpy(), scales.numpy())
    for t in DT.values():
        got = to64(kd.mx4_read(codes.cuda(), scales.cuda(), t))
        w = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
        ok = ~np.isnan(w)
        assert np.array_equal(np.isnan(got), ~ok)
        assert np.array_equal(got[ok], w[ok])


def _head(V, D, seed, spread=3):
    """Random codes and scales of a head (every code, scales of a few powers of two)."""
    g = _gen(seed)
    codes = torch.randint(0, 256, (V, D // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(120 - spread, 121 + spread, (V, D // 32), generator=g, device="cuda",
                           dtype=torch.uint8)
    return codes, scales


def _hidden(N, D, kind, seed):
    """(arguments of mx4_logits, the values they stand for)."""
    g = _gen(seed + 1)
    if kind == "mx4":
        codes, scales = _head(N, D, seed + 2)
        return (codes, scales), ho.mx4_read(codes.cpu().numpy(), scales.cpu().numpy())
    x = torch.randn(N, D, generator=g, device="cuda").to(DT[kind])
    return (x, None), to64(x)


def _tol(hidden_kind, D, mag, ref, out):
    """Products are exact. Of the additions (one per column and term, and those of the
    parts of a row) each is off by at most a step of fp32, 2^-23 of a partial sum that
    the magnitudes' sum bounds; then one rounding to the output's type."""
    terms = 3 if hidden_kind == "f32" else 1
    return (terms * D + 64) * 2.0 ** -23 * mag + HALF[out] * np.abs(ref)


def _check_logits(kd, N, D, V, kind, out, seed=0):
    codes, scales = _head(V, D, seed)
    (h, hs), hv = _hidden(N, D, kind, seed)
    got = kd.mx4_logits(h, codes, scales, hidden_scales=hs, dtype=DT[out])
    assert got.dtype == DT[out] and got.shape == (N, V)
    ref, mag = ho.mx4_logits(hv, codes.cpu().numpy(), scales.cpu().numpy())
    err = np.abs(to64(got) - ref)
    tol = _tol(kind, D, mag, ref, out)
    assert (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("kind", ["bf16", "f32", "mx4"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", [
    (1, 32, 1), (1, 64, 1000), (1, 4096, 2053), (3, 96, 17), (5, 800, 30011), (16, 2048, 515),
    (17, 160, 1023), (32, 1024, 4000), (33, 288, 999), (64, 512, 3001), (65, 320, 257),
    (100, 1632, 777), (127, 256, 256), (129, 416, 1300), (300, 768, 513), (513, 224, 300)])
def test_logits(gpu_lib, kind, out, N, D, V):
    _check_logits(gpu_lib, N, D, V, kind, out, seed=N + D + V)


@pytest.mark.parametrize("kind", ["bf16", "f32", "mx4"])
@pytest.mark.parametrize("N,D,V", [(2, 65536, 40), (70, 16384, 300), (1, 128, 200003)])
def test_logits_long(gpu_lib, kind, N, D, V):
    _check_logits(gpu_lib, N, D, V, kind, "f32", seed=D)


# Products of enough work for tiles (bf16 and fp32, 4 bits): widths of one to many steps,
# with and without a last half step; tiles of 128 and 256 hidden rows; ranges of
# columns that are joined; fewer and more items than compute units
TILES = [
    (300, 768, 20011), (300, 800, 40009), (600, 1632, 20003), (2000, 64, 9001), (3000, 96, 17001),
    (3100, 32, 16411), (700, 288, 65537), (70, 8192, 5003), (129, 16384, 5500), (257, 4096, 9003),
    (1025, 544, 24577), (90, 2080, 30001)]


def _tiled(kd, N, D, V, kind):
    code = {"mx4": kd.KD_MX4, "bf16": kd.KD_BF16, "f32": kd.KD_F32}[kind]
    return kd.mx4_workspace_size(N, D, V, code) >= (V + 255) // 256 * 4 * ((D + 255) // 256 * 512)


@pytest.mark.parametrize("kind,out", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"),
                                      ("mx4", "f32"), ("mx4", "bf16")])
@pytest.mark.parametrize("N,D,V", TILES)
def test_logits_tiles(gpu_lib, kind, out, N, D, V):
    _check_logits(gpu_lib, N, D, V, kind, out, seed=N + D + V)


def test_tiles_are_reached(gpu_lib):
    """Each kind of hidden rows takes the tiles' workspace for most of them."""
    for kind in ("bf16", "f32", "mx4"):
        assert sum(_tiled(gpu_lib, N, D, V, kind) for N, D, V in TILES) >= 8, kind


def test_logits_many_passes(gpu_lib):
    """More fp32 hidden rows than a pass's terms hold, and more rows than a pass takes."""
    _check_logits(gpu_lib, 600, 65536, 130, "f32", "f32", seed=3)
    kd = gpu_lib
    N, D, V = 2 ** 18 + 5, 64, 130
    codes, scales = _head(V, D, 5)
    (h, _), hv = _hidden(N, D, "bf16", 5)
    got = kd.mx4_logits(h, codes, scales, dtype=torch.float32)
    for rows in (slice(0, 40), slice(2 ** 18 - 40, N)):
        ref, mag = ho.mx4_logits(hv[rows], codes.cpu().numpy(), scales.cpu().numpy())
        assert (np.abs(to64(got[rows]) - ref) <= _tol("bf16", D, mag, ref, "f32")).all()


@pytest.mark.parametrize("N,D,V", [(3, 96, 1003), (40, 288, 1003), (100, 768, 40001)])
def test_logits_far_apart(gpu_lib, N, D, V):
    """Rows of hidden states and of logits so far apart that offsets pass 32 bits."""
    kd = gpu_lib
    codes, scales = _head(V, D, 6)
    ldh, ldo = 2 ** 23 + 8 * 61, 2 ** 26 + 3
    (x, _), hv = _hidden(N, D, "bf16", 6)
    h = torch.empty(N, ldh, dtype=torch.bfloat16, device="cuda")[:, :D]
    h.copy_(x)
    z = torch.empty(N, ldo, dtype=torch.bfloat16, device="cuda")[:, :V]
    z.fill_(7.0)
    kd.mx4_logits(h, codes, scales, out=z)
    ref, mag = ho.mx4_logits(hv, codes.cpu().numpy(), scales.cpu().numpy())
    assert (np.abs(to64(z) - ref) <= _tol("bf16", D, mag, ref, "bf16")).all()
    # hidden rows close together: by tiles where there is the work
    z.fill_(7.0)
    kd.mx4_logits(x, codes, scales, out=z)
    assert (np.abs(to64(z) - ref) <= _tol("bf16", D, mag, ref, "bf16")).all()


@pytest.mark.parametrize("kind", ["bf16", "f32", "mx4"])
def test_logits_sweep(gpu_lib, kind):
    """Seeded sizes over the ranges of every kernel's choice."""
    rng = np.random.default_rng({"bf16": 1, "f32": 2, "mx4": 3}[kind])
    for i in range(24):
        N = int(round(2 ** rng.uniform(0, 10.5)))
        D = 32 * int(round(2 ** rng.uniform(0, 7)))
        V = int(round(2 ** rng.uniform(0, 16)))
        while N * D * V > 2 ** 34:
            V = V // 2 + 1
        print(kind, N, D, V, flush=True)
        _check_logits(gpu_lib, N, D, V, kind, ("bf16", "f32")[i % 2], seed=100 + i)


@pytest.mark.parametrize("kind", ["bf16", "f32", "mx4"])
@pytest.mark.parametrize("N,D,V", [(1, 288, 1003), (40, 288, 1003), (260, 288, 1003),
                                   (260, 288, 60003)])
def test_logits_strides(gpu_lib, kind, N, D, V):
    """Hidden rows out of a larger tensor, logits into a padded one at an odd element:
    what lies around them is neither read nor written."""
    kd = gpu_lib
    codes, scales = _head(V, D, 3)
    (h, hs), hv = _hidden(N, D, kind, 3)
    if kind != "mx4":
        wide = torch.full((N, D + 32), float("nan"), dtype=h.dtype, device="cuda")
        wide[:, :D] = h
        h = wide[:, :D]
    for out in ("bf16", "f32"):
        buf = torch.full((3 + N * (V + 6),), 7.0, dtype=DT[out], device="cuda")
        view = buf[3:].view(N, V + 6)[:, :V]
        res = kd.mx4_logits(h, codes, scales, hidden_scales=hs, out=view)
        assert res is view
        ref, mag = ho.mx4_logits(hv, codes.cpu().numpy(), scales.cpu().numpy())
        assert (np.abs(to64(view) - ref) <= _tol(kind, D, mag, ref, out)).all()
        assert bool((buf[:3] == 7).all()) and bool((buf[3:].view(N, V + 6)[:, V:] == 7).all())


@pytest.mark.parametrize("N,V", [(1, 600), (40, 600), (300, 600), (300, 130003)])
def test_logits_special_values(gpu_lib, N, V):
    """Blocks that are not numbers stay with their row; infinite and huge hidden values."""
    kd = gpu_lib
    D = 160
    codes, scales = _head(V, D, 8)
    scales[5, 2] = 255
    scales[599, 4] = 255
    scales[7] = 0
    for kind in ("bf16", "f32", "mx4"):
        (h, hs), hv = _hidden(N, D, kind, 9)
        got = to64(kd.mx4_logits(h, codes, scales, hidden_scales=hs, dtype=torch.float32))
        bad = np.isnan(got)
        assert bad[:, [5, 599]].all() and bad.sum() == 2 * N
    # a code of every element that is not 0, positive: infinities keep their sign
    codes.fill_(0x33)
    scales.fill_(127)
    for kind in ("bf16", "f32"):
        h = torch.ones(N, D, dtype=DT[kind], device="cuda")
        h[0, 33] = float("-inf")
        h[N - 1, 7] = float("nan") if N > 1 else 1.0
        got = to64(kd.mx4_logits(h, codes, scales, dtype=torch.float32))
        assert (got[0] == -np.inf).all()
        if N > 1:
            assert np.isnan(got[N - 1]).all()
            assert (got[1:N - 1] == 1.5 * D).all()
    # the largest fp32 number times 1.5 is infinite, times 0.5 it is itself halved
    codes.fill_(0)
    codes[:, 0] = 0x01
    codes[3, 0] = 0x03
    h = torch.zeros(N, D, device="cuda")
    h[:, 0] = torch.finfo(torch.float32).max
    got = to64(kd.mx4_logits(h, codes, scales))
    assert (got[:, 3] == np.inf).all()
    ref = 0.5 * float(torch.finfo(torch.float32).max)
    assert (np.abs(np.delete(got, 3, axis=1) - ref) <= ref * 2.0 ** -22).all()


@pytest.mark.parametrize("N,V", [(3, 600), (40, 600), (300, 130003)])
def test_hidden_block_not_a_number(gpu_lib, N, V):
    """A 4-bit hidden row with such a block has no number in its logits, the others do."""
    kd = gpu_lib
    D = 416
    codes, scales = _head(V, D, 8)
    (h, hs), hv = _hidden(N, D, "mx4", 9)
    hs[N - 1, 12] = 255
    got = kd.mx4_logits(h, codes, scales, hidden_scales=hs, dtype=torch.float32)
    assert bool(got[N - 1].isnan().all()) and bool(got[:N - 1].isfinite().all())


@pytest.mark.parametrize("kind", ["bf16", "f32", "mx4"])
@pytest.mark.parametrize("N,D,V", [(40, 4096, 1500), (300, 512, 70001)])
def test_logits_two_at_a_time(gpu_lib, kind, N, D, V):
    """Two calls that overlap on streams of their own, and two captured graphs that
    share a workspace one after the other."""
    kd = gpu_lib
    code = {"mx4": kd.KD_MX4, "bf16": kd.KD_BF16, "f32": kd.KD_F32}[kind]
    n = kd.mx4_workspace_size(N, D, V, code)
    sets = []
    for seed in (1, 2):
        codes, scales = _head(V, D, seed)
        (h, hs), _ = _hidden(N, D, kind, seed)
        want = kd.mx4_logits(h, codes, scales, hidden_scales=hs, dtype=torch.float32)
        sets.append((h, hs, codes, scales, want, torch.zeros_like(want), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for h, hs, codes, scales, want, out, s in sets:
            with torch.cuda.stream(s):
                kd.mx4_logits(h, codes, scales, hidden_scales=hs, out=out)
    torch.cuda.synchronize()
    for *_, want, out, _ in sets:
        assert torch.equal(out, want)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    graphs = []
    for h, hs, codes, scales, want, out, s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kd.mx4_logits(h, codes, scales, hidden_scales=hs, out=out, workspace=ws)
        graphs.append(g)
    for _ in range(3):
        for s in sets:
            s[5].zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for *_, want, out, _ in sets:
            assert torch.equal(out, want)


def test_write_read_graph(gpu_lib):
    kd = gpu_lib
    x = torch.randn(100, 256, generator=_gen(1), device="cuda")
    q = kd.mx4_write(x)
    back = kd.mx4_read(q["codes"], q["scales"], torch.bfloat16)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kd.mx4_write(x, out=q)
        kd.mx4_read(q["codes"], q["scales"], torch.bfloat16, out=back)
    for seed in (2, 3, 4):
        x.copy_(torch.randn(100, 256, generator=_gen(seed), device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        _same(back, ho.mx4_read(*ho.mx4_write(to64(x))))


@pytest.mark.parametrize("N", [0, 1])
def test_logits_few(gpu_lib, N):
    kd = gpu_lib
    codes, scales = _head(10, 64, 1)
    got = kd.mx4_logits(torch.ones(N, 64, device="cuda"), codes, scales)
    assert got.shape == (N, 10) and got.dtype == torch.float32


@pytest.mark.parametrize("kind", ["bf16", "f32", "mx4"])
@pytest.mark.parametrize("N,D,V", [(4, 512, 2500), (300, 512, 2500), (40, 4096, 1500),
                                   (300, 512, 70001), (80, 8192, 9001)])
def test_logits_graph_and_streams(gpu_lib, kind, N, D, V):
    """The same bits from a replayed graph, from another stream, and twice in a row."""
    kd = gpu_lib
    codes, scales = _head(V, D, 4)
    (h, hs), _ = _hidden(N, D, kind, 4)
    want = kd.mx4_logits(h, codes, scales, hidden_scales=hs, dtype=torch.float32)
    code = kd.KD_MX4 if kind == "mx4" else kd.KD_BF16 if kind == "bf16" else kd.KD_F32
    ws = torch.empty(kd.mx4_workspace_size(N, D, V, code), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        kd.mx4_logits(h, codes, scales, hidden_scales=hs, out=out, workspace=ws)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kd.mx4_logits(h, codes, scales, hidden_scales=hs, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_round_straight_through(gpu_lib):
    kd = gpu_lib
    W = torch.randn(50, 96, generator=_gen(2), device="cuda").requires_grad_(True)
    r = kd.mx4_round(W)
    q = kd.mx4_write(W.detach())
    assert torch.equal(r.detach(), kd.mx4_read(q["codes"], q["scales"], torch.float32))
    up = torch.randn(50, 96, generator=_gen(3), device="cuda")
    (r * up).sum().backward()
    assert torch.equal(W.grad, up)


def test_refusals(gpu_lib):
    kd = gpu_lib
    codes, scales = _head(20, 64, 1)
    h = torch.ones(4, 64, device="cuda")
    good = kd.mx4_logits(h, codes, scales)
    for bad in (lambda: kd.mx4_logits(h[:, :32].contiguous(), codes, scales),
                lambda: kd.mx4_logits(h.cpu(), codes, scales),
                lambda: kd.mx4_logits(h, codes, scales[:, :1]),
                lambda: kd.mx4_logits(h, codes.int(), scales),
                lambda: kd.mx4_logits(h[0], codes, scales),
                lambda: kd.mx4_logits(h.t().contiguous().t(), codes, scales),
                lambda: kd.mx4_logits(codes, codes, scales, hidden_scales=scales[:3]),
                lambda: kd.mx4_logits(h, codes, scales, out=good[:, :19]),
                lambda: kd.mx4_logits(h, codes, scales, out=good, dtype=torch.bfloat16),
                lambda: kd.mx4_logits(h, codes, scales, workspace=torch.empty(256, device="cuda")),
                lambda: kd.mx4_write(h.t()), lambda: kd.mx4_write(h[0]),
                lambda: kd.mx4_write(h, out={"codes": codes, "scales": scales}),
                lambda: kd.mx4_read(codes, scales[:, :1], torch.float32),
                lambda: kd.mx4_read(codes, scales, torch.float32, out=h)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: kd.mx4_logits(h.half(), codes, scales),
                lambda: kd.mx4_logits(h, codes, scales, dtype=torch.float16),
                lambda: kd.mx4_write(h.half()), lambda: kd.mx4_read(codes, scales, torch.float16)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(kd.KdError):    # rows that are not 16-byte aligned
        kd.mx4_logits(torch.ones(4, 67, device="cuda")[:, :64], codes, scales)
    with pytest.raises(kd.KdError):    # a width that is not a multiple of 32
        kd.mx4_write(torch.ones(4, 48, device="cuda"))
    with pytest.raises(kd.KdError):
        kd.mx4_logits(h, codes, scales, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert torch.equal(kd.mx4_logits(h, codes, scales), good)
