"""Logits with a 4-bit head, bit by bit: values whose sums are exact in fp32 whatever
their order, for every kernel, tile and split that the plan chooses (test_mx4_plan.py
checks that these sizes take them all)."""
import pytest
import torch

from tests.mx4_shapes import CASES, FAR

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _power(e):
    """2^e in fp64, exactly (e in [-127, 127]; torch's own powers are not always)."""
    return torch.tensor([2.0 ** k for k in range(-127, 128)], dtype=torch.float64,
                        device="cuda")[e.long() + 127]


def _values(codes, scales):
    """What codes and scales stand for, in fp64."""
    table = torch.tensor(E2M1 + [-x for x in E2M1], dtype=torch.float64, device="cuda")
    c = torch.stack([codes & 15, codes >> 4], dim=2).flatten(1)
    s = _power(scales.int() - 127)
    return table[c.long()] * s.repeat_interleave(32, dim=1)


def _ints(lo, hi, shape, g, dtype=torch.uint8):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=dtype)


def _whole(kind, N, D, V, seed):
    """Numbers that are multiples of a small unit: (hidden, its scales, codes, scales, the
    logits in fp64, which are exact in fp32: the products' magnitudes sum to less than
    2^24 units)."""
    g = _gen(seed)
    codes = _ints(0, 256, (V, D // 2), g)
    scales = _ints(126, 129, (V, D // 32), g)
    w = _values(codes, scales)
    if kind == "mx4":
        h, hs = _ints(0, 256, (N, D // 2), g), torch.full((N, D // 32), 127, dtype=torch.uint8,
                                                          device="cuda")
        hv, unit = _values(h, hs), 0.125
    else:
        # 48 units a product of 1 at most; in bf16 whole numbers are exact up to 256
        most = min(100 if kind == "bf16" else 4000, 2 ** 24 // 48 // D)
        h, hs = _ints(-most, most + 1, (N, D), g, torch.int32).to(DT[kind]), None
        hv, unit = h.double(), 0.25
    assert float((hv.abs() @ w.abs().t()).max()) < 2.0 ** 24 * unit
    return h, hs, codes, scales, hv @ w.t()


@pytest.mark.parametrize("kind,N,D,V", CASES)
def test_sums(gpu_lib, kind, N, D, V):
    h, hs, codes, scales, ref = _whole(kind, N, D, V, N + D + V)
    got = gpu_lib.mx4_logits(h, codes, scales, hidden_scales=hs, dtype=torch.float32)
    assert torch.equal(got.double(), ref)
    got = gpu_lib.mx4_logits(h, codes, scales, hidden_scales=hs, dtype=torch.bfloat16)
    assert torch.equal(got, ref.float().bfloat16())


@pytest.mark.parametrize("kind,N,D,V", CASES)
def test_one_column(gpu_lib, kind, N, D, V):
    """One column of a hidden row that is not 0, of every block in turn: the product of two
    numbers with all their bits, and of the blocks' scales."""
    g = _gen(N + D + V + 1)
    codes = _ints(0, 256, (V, D // 2), g)
    if kind == "f32":
        # (powers of two, with which 24 bits stay 24)
        place = torch.tensor([1, 2, 4, 6, 9, 10, 12, 14], dtype=torch.uint8, device="cuda")
        c = place[_ints(0, 8, (V, D), g).long()]
        codes = c[:, 0::2] | (c[:, 1::2] << 4)
    scales = _ints(117, 138, (V, D // 32), g)
    w = _values(codes, scales)
    B = D // 32
    calls = min(8, -(-B // N))
    # blocks of all calls' rows, spread over the width, the last one among them
    blocks = torch.linspace(0, B - 1, calls * N, dtype=torch.float64).round().long().flip(0)
    for k in range(calls):
        b = blocks[k::calls].cuda()
        col = 32 * b + _ints(0, 32, (N,), g, torch.int64)
        rows = torch.arange(N, device="cuda")
        if kind == "mx4":
            h = torch.zeros(N, D // 2, dtype=torch.uint8, device="cuda")
            code = _ints(1, 16, (N,), g)
            h[rows, col // 2] = torch.where(col % 2 == 1, code << 4, code)
            hs = _ints(117, 138, (N, B), g)
            x = _values(h, hs)[rows, col]
        else:
            # an odd significand of as many bits as the type's, at any of 40 sizes
            bits = 8 if kind == "bf16" else 24
            m = _ints(2 ** (bits - 2), 2 ** (bits - 1), (N,), g, torch.int64) * 2 + 1
            x = m.double() * _power(_ints(-40, 0, (N,), g, torch.int64))
            x = torch.where(_ints(0, 2, (N,), g) == 1, -x, x)
            h, hs = torch.zeros(N, D, dtype=DT[kind], device="cuda"), None
            h[rows, col] = x.to(DT[kind])
            assert torch.equal(h[rows, col].double(), x)
        got = gpu_lib.mx4_logits(h, codes, scales, hidden_scales=hs, dtype=torch.float32)
        ref = x[:, None] * w[:, col].t()
        assert torch.equal(ref.float().double(), ref)
        assert torch.equal(got.double(), ref), k


def test_many_rows(gpu_lib):
    """More rows than a pass takes."""
    h, hs, codes, scales, ref = _whole("bf16", 2 ** 18 + 5, 64, 130, 1)
    got = gpu_lib.mx4_logits(h, codes, scales, dtype=torch.float32)
    assert torch.equal(got.double(), ref)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("kind,N,D,V", FAR)
def test_far_apart(gpu_lib, kind, N, D, V, out):
    """Rows of logits that a tile's 32-bit offsets do not reach."""
    h, hs, codes, scales, ref = _whole(kind, N, D, V, 2)
    z = torch.empty(N, 2 ** 26 + 3, dtype=DT[out], device="cuda")
    z[:, V:V + 70].fill_(7.0)
    gpu_lib.mx4_logits(h, codes, scales, hidden_scales=hs, out=z[:, :V])
    assert torch.equal(z[:, :V], ref.float().to(DT[out]))
    assert bool((z[:, V:V + 70] == 7).all())


@pytest.mark.parametrize("kind,D,V", [("bf16", 8192, 5003), ("f32", 4096, 8001), ("mx4", 8192, 5003)])
def test_one_workspace(gpu_lib, kind, D, V):
    """One workspace, of the size for the largest batch, serves every smaller one."""
    kd = gpu_lib
    code = {"f32": kd.KD_F32, "bf16": kd.KD_BF16, "mx4": kd.KD_MX4}[kind]
    ws = torch.empty(kd.mx4_workspace_size(600, D, V, code), dtype=torch.uint8, device="cuda")
    for N in (600, 300, 257, 128, 65, 64, 20, 1):
        h, hs, codes, scales, ref = _whole(kind, N, D, V, N)
        ws.fill_(255)
        got = kd.mx4_logits(h, codes, scales, hidden_scales=hs, dtype=torch.float32, workspace=ws)
        assert torch.equal(got.double(), ref), N
