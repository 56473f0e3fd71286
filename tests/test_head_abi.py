"""Host-side checks of the output head's operators (no GPU needed): every argument
error is found before anything is enqueued, so fake pointers serve. A call that
would pass its checks is never made here. And pins of their oracle."""
import ctypes

import numpy as np
import pytest

import paper_2608_03796_amd as kd
from oracle import head_oracle as ho

FAKE = 0x10000
ODD = 0x10001
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return kd.load_library()


def _v(x):
    return None if x is None else ctypes.c_void_p(x)


@pytest.mark.parametrize("name", ["kd_mx4_write", "kd_mx4_read"])
def test_mx4_rejected(lib, name):
    def call(N=4, D=64, dtype=kd.KD_BF16, x=FAKE, c=FAKE, s=FAKE):
        p = (x, c, s) if name.endswith("write") else (c, s, x)
        return getattr(lib, name)(N, D, dtype, *[_v(q) for q in p], None)
    for kw in (dict(N=-1), dict(N=2 ** 31), dict(D=0), dict(D=16), dict(D=65568)):
        assert call(**kw) == 2
    for kw in (dict(x=None), dict(c=None), dict(s=None)):
        assert call(**kw) == 1
    for kw in (dict(D=48), dict(dtype=2), dict(dtype=-1), dict(x=FAKE + 8), dict(c=FAKE + 8)):
        assert call(**kw) == 4
    assert call(N=0, x=None, c=None, s=None) == 0


def _head(N=4, D=64, V=1000, ld_hidden=64, ld_out=1000, dtype=kd.KD_BF16, out_dtype=kd.KD_F32,
          flags=0):
    return kd.KdMx4Head(N, D, V, ld_hidden, ld_out, dtype, out_dtype, flags)


def _logits(lib, pr, n=BIG, **kw):
    names = ("hidden", "hidden_scales", "codes", "scales", "out", "ws")
    return lib.kd_mx4_logits(None if pr is None else ctypes.byref(pr),
                             *[_v(kw.get(k, FAKE)) for k in names], ctypes.c_size_t(n), None)


@pytest.mark.parametrize("kw,code", [
    (dict(N=-1), 2), (dict(N=2 ** 31), 2), (dict(D=0), 2), (dict(D=65568, ld_hidden=65568), 2),
    (dict(D=48), 4), (dict(V=0), 2), (dict(V=2 ** 20 + 1, ld_out=2 ** 21), 2),
    (dict(ld_out=999), 2), (dict(ld_out=2 ** 31 + 1), 2), (dict(ld_hidden=63), 2),
    (dict(ld_hidden=2 ** 31 + 16), 2), (dict(ld_hidden=68), 4), (dict(dtype=3), 4),
    (dict(dtype=-1), 4), (dict(out_dtype=2), 4), (dict(flags=1), 3)])
def test_head_rejected(lib, kw, code):
    pr = _head(**kw)
    n = ctypes.c_size_t(0)
    assert lib.kd_mx4_logits_workspace_size(ctypes.byref(pr), ctypes.byref(n)) == code
    assert _logits(lib, pr) == code


def test_head_pointers_rejected(lib):
    assert _logits(lib, None) == 1
    n = ctypes.c_size_t(0)
    assert lib.kd_mx4_logits_workspace_size(None, ctypes.byref(n)) == 1
    assert lib.kd_mx4_logits_workspace_size(ctypes.byref(_head()), None) == 1
    for name in ("hidden", "codes", "scales", "out", "ws"):
        assert _logits(lib, _head(), **{name: None}) == 1, name
    assert _logits(lib, _head(dtype=kd.KD_MX4), hidden_scales=None) == 1
    for name in ("hidden", "codes", "ws"):
        assert _logits(lib, _head(), **{name: FAKE + 8}) == 4, name
    assert _logits(lib, _head(), out=FAKE + 2) == 4
    assert _logits(lib, _head(out_dtype=kd.KD_BF16), out=ODD) == 4
    for dtype in (kd.KD_F32, kd.KD_BF16, kd.KD_MX4):
        for N in (1, 64, 4096):
            pr = _head(N=N, dtype=dtype)
            assert lib.kd_mx4_logits_workspace_size(ctypes.byref(pr), ctypes.byref(n)) == 0
            assert _logits(lib, pr, n=n.value - 1) == 5
    # no rows: nothing launched
    assert _logits(lib, _head(N=0), hidden=None, codes=None, scales=None, out=None) == 0


def test_oracle_mx4_by_hand():
    x = np.zeros((1, 64))
    x[0, :8] = [6.0, 0.25, 0.75, -1.25, 2.5, -5.0, 3.5, 0.26]
    x[0, 32:35] = [0.7, -0.1, 0.05]     # scale 2^-3: 5.6, -0.8, 0.4
    codes, scales = ho.mx4_write(x)
    assert list(scales[0]) == [127, 124]
    v = ho.mx4_read(codes, scales)[0]
    assert list(v[:8]) == [6.0, 0.0, 1.0, -1.0, 2.0, -4.0, 4.0, 0.5]
    assert list(v[32:35]) == [0.75, -0.125, 0.0625]
    assert codes[0, 0] == 7 | 0 << 4 and codes[0, 1] == 2 | (2 + 8) << 4


def test_oracle_mx4_is_nearest():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((20, 96)) * np.exp2(rng.integers(-30, 30, (20, 1)))
    codes, scales = ho.mx4_write(x)
    v = ho.mx4_read(codes, scales)
    s = np.repeat(np.exp2(scales.astype(float) - 127), 32, axis=1)
    top = np.abs(x).reshape(20, 3, 32).max(axis=2)
    p = np.exp2(scales.astype(float) - 127)
    assert (top <= 6 * p).all() and (top > 3 * p).all()
    grid = np.concatenate([-ho.VALUES[::-1], ho.VALUES])
    best = np.abs(x[..., None] / s[..., None] - grid).min(axis=-1)
    assert np.array_equal(np.abs(x - v) / s, best)
    assert np.array_equal(ho.mx4_read(*ho.mx4_write(v)), v)


def _labels(N=256, D=256, V=4096, chunk=64, dtype=kd.KD_BF16, z=0.0, flags=0):
    return kd.KdLabelProblem(N, D, V, chunk, dtype, z, flags)


def _ce(lib, name, pr, n=BIG, acc=0, **kw):
    p = {k: _v(kw.get(k, FAKE)) for k in ("hidden", "W", "labels", "loss", "lpt", "logz", "gl", "glt",
                                          "gh", "gw", "ws")}
    ptr = None if pr is None else ctypes.byref(pr)
    tail = (p["ws"], ctypes.c_size_t(n), None)
    if name == "kd_cross_entropy_fwd_bwd":
        return lib.kd_cross_entropy_fwd_bwd(ptr, p["hidden"], p["W"], p["labels"], p["loss"],
                                            p["lpt"], p["gh"], p["gw"], acc, *tail)
    if name == "kd_cross_entropy_fwd":
        return lib.kd_cross_entropy_fwd(ptr, p["hidden"], p["W"], p["labels"], p["loss"], p["lpt"],
                                        p["logz"], *tail)
    return lib.kd_cross_entropy_bwd(ptr, p["hidden"], p["W"], p["labels"], p["logz"], p["gl"],
                                    p["glt"], p["gh"], p["gw"], acc, *tail)


CE = ("kd_cross_entropy_fwd_bwd", "kd_cross_entropy_fwd", "kd_cross_entropy_bwd")


@pytest.mark.parametrize("kw,code", [
    (dict(N=-1), 2), (dict(N=2 ** 31), 2), (dict(D=0), 2), (dict(D=96), 4), (dict(V=0), 2),
    (dict(V=2 ** 20 + 1), 2), (dict(chunk=0), 3), (dict(dtype=2), 4), (dict(dtype=-1), 4),
    (dict(z=-1e-3), 3), (dict(z=float("inf")), 3), (dict(z=float("nan")), 3), (dict(flags=1), 3),
    (dict(flags=4), 3)])
def test_labels_rejected(lib, kw, code):
    pr = _labels(**kw)
    n = ctypes.c_size_t(0)
    assert lib.kd_cross_entropy_workspace_size(ctypes.byref(pr), ctypes.byref(n)) == code
    for name in CE:
        assert _ce(lib, name, pr) == code


@pytest.mark.parametrize("name", CE)
def test_labels_pointers_rejected(lib, name):
    pr = _labels()
    assert _ce(lib, name, None) == 1
    need = ["hidden", "W", "labels", "ws"]
    need += ["logz"] if name != CE[0] else []
    need += ["loss"] if name != CE[2] else []
    for k in need:
        assert _ce(lib, name, pr, **{k: None}) == 1, k
    for k in ("hidden", "W", "ws", "labels") + (() if name == CE[1] else ("gh", "gw")):
        assert _ce(lib, name, pr, **{k: FAKE + (4 if k == "labels" else 8)}) == 4, k
    n = ctypes.c_size_t(0)
    assert lib.kd_cross_entropy_workspace_size(ctypes.byref(pr), ctypes.byref(n)) == 0
    assert _ce(lib, name, pr, n=n.value - 1) == 5
    if name != CE[1]:
        assert _ce(lib, name, pr, acc=2) == 3
    # the teacher's arrays stand behind the loss's own workspace
    m = ctypes.c_size_t(0)
    q = kd.problem(256, 256, 4096, 1, 64, 1.0, kd.KD_BF16)
    assert lib.kd_topk_kl_workspace_size(ctypes.byref(q), ctypes.byref(m)) == 0
    assert m.value + 9 * 256 <= n.value <= m.value + 9 * 256 + 1024


def test_oracle_cross_entropy():
    """Against torch's autograd in fp64, and central differences."""
    import torch
    rng = np.random.default_rng(1)
    N, D, V, z = 7, 5, 11, 0.03
    h, W = rng.standard_normal((N, D)), rng.standard_normal((V, D))
    lab = np.array([0, 10, -100, 3, 11, 3, 5])
    g = rng.standard_normal(N)
    for kw in (dict(g=1.7), dict(g_token=g)):
        got = ho.cross_entropy(h, W, lab, z_loss=z, **kw)
        th, tW = (torch.tensor(x, requires_grad=True) for x in (h, W))
        x = th @ tW.T
        ok = torch.tensor((lab >= 0) & (lab < V))
        lz = torch.logsumexp(x, 1)
        l = lz - x[torch.arange(N), torch.tensor(np.where(ok, lab, 0))] + z * lz ** 2
        l = torch.where(ok, l, 0.0)
        mean = l.sum() / ok.sum()
        total = 1.7 * mean if "g" in kw else (l * torch.tensor(g)).sum()
        total.backward()
        assert abs(got["loss"] - float(mean.detach())) < 1e-14
        assert np.allclose(got["loss_per_token"], l.detach().numpy(), atol=1e-13)
        assert np.allclose(got["grad_hidden"], th.grad.numpy(), atol=1e-14)
        assert np.allclose(got["grad_W"], tW.grad.numpy(), atol=1e-14)
    got = ho.cross_entropy(h, W, lab, z_loss=z)
    for name, x, grad in (("h", h, got["grad_hidden"]), ("W", W, got["grad_W"])):
        for at in ((0, 0), (3, 2), (5, 4)):
            d = np.zeros_like(x)
            d[at] = 1e-5
            a = ho.cross_entropy(*((h + d, W) if name == "h" else (h, W + d)), lab, z_loss=z)
            b = ho.cross_entropy(*((h - d, W) if name == "h" else (h, W - d)), lab, z_loss=z)
            assert abs((a["loss"] - b["loss"]) / 2e-5 - grad[at]) < 1e-8
    assert ho.cross_entropy(h, W, np.full(N, -1))["loss"] == 0.0
