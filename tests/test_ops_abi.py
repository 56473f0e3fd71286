"""Host-side checks of the operators around the loss (no GPU needed): every
argument error is found before anything is enqueued, so fake pointers serve. A
call that would pass its checks is never made here."""
import ctypes

import pytest

import paper_2608_03796_amd as kd

FAKE = 0x10000
ODD = 0x10001
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return kd.load_library()


def _v(x):
    return None if x is None else ctypes.c_void_p(x)


def _rows(N=4, V=1000, ld=1000, K=8, dtype=kd.KD_BF16, flags=0):
    return kd.KdRows(N, V, ld, K, dtype, flags)


def _topk(lib, pr, name, logits=FAKE, a=FAKE, b=FAKE, ws=FAKE, n=BIG):
    return getattr(lib, name)(None if pr is None else ctypes.byref(pr), _v(logits), _v(a), _v(b),
                              _v(ws), ctypes.c_size_t(n), None)


@pytest.mark.parametrize("kw,code", [
    (dict(N=-1), 2), (dict(N=2 ** 31), 2), (dict(V=0, ld=0), 2), (dict(V=2 ** 20 + 1, ld=2 ** 21), 2),
    (dict(ld=999), 2), (dict(ld=2 ** 31 + 1), 2), (dict(K=0), 2), (dict(K=1001), 2),
    (dict(V=5000, ld=5000, K=4097), 2), (dict(dtype=2), 4), (dict(dtype=-1), 4),
    (dict(flags=2), 3), (dict(flags=-1), 3)])
def test_rows_rejected(lib, kw, code):
    pr = _rows(**kw)
    n = ctypes.c_size_t(0)
    assert lib.kd_topk_entries_workspace_size(ctypes.byref(pr), ctypes.byref(n)) == code
    for name in ("kd_topk_entries", "kd_teacher_cache_write"):
        assert _topk(lib, pr, name) == code


def test_rows_workspace(lib):
    n = ctypes.c_size_t(0)
    assert lib.kd_topk_entries_workspace_size(None, ctypes.byref(n)) == 1
    assert lib.kd_topk_entries_workspace_size(ctypes.byref(_rows()), None) == 1
    # bounded in N: group maxima of a batch of rows
    for N in (0, 1, 1000, 1 << 30):
        for V in (1, 131072, 1 << 20):
            pr = _rows(N=N, V=V, ld=V, K=1)
            assert lib.kd_topk_entries_workspace_size(ctypes.byref(pr), ctypes.byref(n)) == 0
            assert 0 < n.value <= (64 << 20) + 4096


@pytest.mark.parametrize("name", ["kd_topk_entries", "kd_teacher_cache_write"])
def test_topk_pointers_rejected(lib, name):
    pr = _rows()
    assert _topk(lib, None, name) == 1
    for kw in (dict(logits=None), dict(a=None), dict(b=None), dict(ws=None)):
        assert _topk(lib, pr, name, **kw) == 1
    for kw in (dict(logits=ODD), dict(a=FAKE + 2), dict(b=FAKE + 2), dict(ws=FAKE + 8)):
        assert _topk(lib, pr, name, **kw) == 4
    assert _topk(lib, _rows(dtype=kd.KD_F32), name, logits=FAKE + 2) == 4
    n = ctypes.c_size_t(0)
    assert lib.kd_topk_entries_workspace_size(ctypes.byref(pr), ctypes.byref(n)) == 0
    assert _topk(lib, pr, name, n=n.value - 1) == 5
    # nothing to do: nothing launched
    assert _topk(lib, _rows(N=0), name, logits=None, a=None, b=None) == 0


def test_cache_read_rejected(lib):
    def call(N=10, K=4, e=FAKE, s=FAKE, rows=FAKE, M=5, idx=FAKE, logit=FAKE, ign=FAKE):
        return lib.kd_teacher_cache_read(N, K, _v(e), _v(s), _v(rows), M, _v(idx), _v(logit),
                                         _v(ign), None)
    for kw in (dict(N=-1), dict(M=-1), dict(M=2 ** 31), dict(K=0), dict(K=4097),
               dict(rows=None, M=11)):
        assert call(**kw) == 2
    for kw in (dict(e=None), dict(s=None), dict(idx=None), dict(logit=None)):
        assert call(**kw) == 1
    for kw in (dict(e=FAKE + 2), dict(s=FAKE + 2), dict(rows=FAKE + 4), dict(idx=ODD),
               dict(logit=FAKE + 1)):
        assert call(**kw) == 4
    assert call(M=0, idx=None, logit=None) == 0


@pytest.mark.parametrize("name", ["kd_checkpoint_write", "kd_checkpoint_read"])
def test_checkpoint_rejected(lib, name):
    def call(N=4, D=64, dtype=kd.KD_BF16, h=FAKE, c=FAKE, s=FAKE):
        p = (h, c, s) if name.endswith("write") else (c, s, h)
        return getattr(lib, name)(N, D, dtype, *[_v(x) for x in p], None)
    for kw in (dict(N=-1), dict(N=2 ** 31), dict(D=0), dict(D=16), dict(D=65568)):
        assert call(**kw) == 2
    for kw in (dict(h=None), dict(c=None), dict(s=None)):
        assert call(**kw) == 1
    for kw in (dict(D=48), dict(dtype=2), dict(h=FAKE + 8), dict(c=FAKE + 8)):
        assert call(**kw) == 4
    assert call(N=0, h=None, c=None, s=None) == 0


def _draft(B=4, T=3, V=1000, ld_target=1000, ld_draft=1000, K=8, dtype=kd.KD_BF16, tau=1.0, flags=0):
    return kd.KdDraft(B, T, V, ld_target, ld_draft, K, dtype, tau, flags)


def _verify(lib, pr, n=BIG, **kw):
    names = ("target", "tokens", "idx", "logit", "logits", "uniform", "lengths", "out", "accepted",
             "prob", "ws")
    return lib.kd_verify_draft(None if pr is None else ctypes.byref(pr),
                               *[_v(kw.get(k, FAKE)) for k in names], ctypes.c_size_t(n), None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), 2), (dict(B=2 ** 20 + 1), 2), (dict(T=-1), 2), (dict(T=1025), 2), (dict(V=0), 2),
    (dict(V=2 ** 20 + 1, ld_target=2 ** 21), 2), (dict(ld_target=999), 2),
    (dict(ld_target=2 ** 31 + 1), 2), (dict(K=-1), 2), (dict(K=1001), 2),
    (dict(V=9000, ld_target=9000, K=4097), 2), (dict(K=0, ld_draft=999), 2), (dict(dtype=2), 4),
    (dict(tau=0.0), 3), (dict(tau=-1.0), 3), (dict(tau=float("nan")), 3),
    (dict(tau=float("inf")), 3), (dict(flags=1), 3),
    (dict(B=2 ** 20, T=16), 2), (dict(B=65536, V=2 ** 20, ld_target=2 ** 20), 2)])
def test_draft_rejected(lib, kw, code):
    pr = _draft(**kw)
    n = ctypes.c_size_t(0)
    assert lib.kd_verify_draft_workspace_size(ctypes.byref(pr), ctypes.byref(n)) == code
    assert _verify(lib, pr) == code


def test_verify_pointers_rejected(lib):
    assert _verify(lib, None) == 1
    n = ctypes.c_size_t(0)
    assert lib.kd_verify_draft_workspace_size(None, ctypes.byref(n)) == 1
    assert lib.kd_verify_draft_workspace_size(ctypes.byref(_draft()), None) == 1
    for name in ("target", "tokens", "idx", "logit", "uniform", "out", "accepted", "ws"):
        assert _verify(lib, _draft(), **{name: None}) == 1, name
    assert _verify(lib, _draft(K=0), logits=None) == 1
    for name in ("target", "tokens", "idx", "logit", "logits", "uniform", "lengths", "out",
                 "accepted", "prob", "ws"):
        assert _verify(lib, _draft(), **{name: ODD}) == 4, name
    for K in (0, 8):
        pr = _draft(K=K)
        assert lib.kd_verify_draft_workspace_size(ctypes.byref(pr), ctypes.byref(n)) == 0
        assert _verify(lib, pr, n=n.value - 1) == 5
    # no sequences: nothing launched
    assert _verify(lib, _draft(B=0), target=None, tokens=None, uniform=None, out=None,
                   accepted=None) == 0


def test_bwd_checkpoint_rejected(lib):
    def call(pr, codes=FAKE, scales=FAKE, W=FAKE, idx=FAKE, tl=FAKE, gh=FAKE, gw=FAKE, acc=0,
             ws=FAKE, n=BIG):
        return lib.kd_topk_kl_bwd_checkpoint(
            None if pr is None else ctypes.byref(pr), _v(codes), _v(scales), _v(W), _v(idx), _v(tl),
            None, None, None, _v(gh), _v(gw), acc, _v(ws), ctypes.c_size_t(n), None)
    pr = kd.problem(256, 256, 4096, 16, 64, 1.0, kd.KD_BF16)
    assert call(None) == 1
    for kw in (dict(codes=None), dict(scales=None), dict(W=None), dict(idx=None), dict(tl=None),
               dict(ws=None)):
        assert call(pr, **kw) == 1
    for kw in (dict(codes=FAKE + 8), dict(W=FAKE + 8), dict(gh=FAKE + 8), dict(gw=FAKE + 8),
               dict(ws=FAKE + 8)):
        assert call(pr, **kw) == 4
    assert call(pr, acc=2) == 3
    need = ctypes.c_size_t(0)
    assert lib.kd_topk_kl_workspace_size(ctypes.byref(pr), ctypes.byref(need)) == 0
    assert call(pr, n=need.value - 1) == 5
    for kw, code in ((dict(tau=0.0), 3), (dict(chunk=0), 3), (dict(D=96), 4), (dict(K=0), 2)):
        a = dict(N=256, D=256, V=4096, K=16, chunk=64, tau=1.0, dtype=kd.KD_BF16)
        a.update(kw)
        assert call(kd.problem(**a)) == code
    # no gradient asked for: nothing launched
    assert call(pr, gh=None, gw=None) == 0
