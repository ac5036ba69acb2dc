"""Arguments of the full-rank and AdamW calls that the host refuses, on the CPU: nothing here reaches a GPU."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2605_16341_b200 import binding
    if not os.path.exists(binding.LIB_PATH):
        binding.build_library()
    return binding.lib()


def muon(L, m=64, n=48, mu=0.95, eta=0.02, wd=0.1, nesterov=1):
    h = ctypes.c_void_p()
    return L.orthdion_muon_create(ctypes.byref(h), m, n, mu, eta, wd, nesterov), h


def test_muon_create_refuses(L):
    nan = float("nan")
    for kw in (dict(m=0), dict(n=0), dict(m=-1), dict(m=(1 << 18) + 1), dict(m=40000, n=40000), dict(mu=1.0), dict(mu=-0.1), dict(mu=nan), dict(eta=nan),
               dict(wd=float("inf")), dict(nesterov=2)):
        rc, h = muon(L, **kw)
        assert rc == -1 and not h.value, kw
    assert L.orthdion_muon_create(None, 4, 4, 0.9, 0.1, 0.0, 1) == -3
    rc, h = muon(L, m=1, n=1 << 18)
    assert rc == 0 and L.orthdion_muon_destroy(h) == 0 and L.orthdion_muon_destroy(h) == -1
    assert L.orthdion_muon_destroy(None) == -1


def test_muon_setters_refuse(L):
    _, h = muon(L)
    nan = float("nan")
    assert L.orthdion_muon_set_dtypes(h, 2, 0) == -1 and L.orthdion_muon_set_dtypes(h, 0, -1) == -1 and L.orthdion_muon_set_dtypes(h, 0, 1) == 0
    assert L.orthdion_muon_set_lr(h, nan) == -1 and L.orthdion_muon_set_lr(h, 0.0) == 0
    assert L.orthdion_muon_set_scale(h, nan) == -1 and L.orthdion_muon_set_scale(h, 2.0) == 0
    assert L.orthdion_muon_set_ld(h, 47, 48, 48) == -1 and L.orthdion_muon_set_ld(h, 48, 48, 1 << 32) == -1 and L.orthdion_muon_set_ld(h, 50, 49, 48) == 0
    assert L.orthdion_muon_set_passes(h, 2) == -1 and L.orthdion_muon_set_passes(h, 3) == 0 and L.orthdion_muon_set_passes(h, 0) == 0

    def schedule(rows, eps=1e-7):
        flat = [v for r in rows for v in r]
        return L.orthdion_muon_set_schedule(h, len(rows), (ctypes.c_float * max(1, len(flat)))(*flat), eps)

    fast = (3.4445, -4.7750, 2.0315)
    assert schedule([fast] * 5) == 0 and schedule([fast] * 32) == 0
    assert schedule([]) == -1 and schedule([fast] * 33) == -1
    assert schedule([fast], -1.0) == -1 and schedule([fast], nan) == -1 and schedule([fast], 0.0) == 0
    assert schedule([(nan, 0, 0)]) == -1
    assert schedule([(9.0, 0.0, 0.0)]) == -1                         # a singular value of 9
    assert schedule([(3.0, 0.0, 0.0)] * 2) == -1 and schedule([(2.8, 0.0, 0.0)] * 2) == 0
    assert schedule([(100.0, -200.0, 101.0)]) == -1                  # factors beyond what the images hold
    assert L.orthdion_muon_set_schedule(h, 1, None, 0.0) == -3
    assert L.orthdion_muon_destroy(h) == 0
    for f in ("set_dtypes", "set_ld"):
        assert getattr(L, "orthdion_muon_" + f)(None, *([48] * (2 if f == "set_dtypes" else 3))) == -1


def test_muon_calls_refuse_on_the_host(L):
    rc, h = muon(L)
    p = ctypes.c_void_p
    arr = lambda *v: (p * len(v))(*v)  # noqa: E731
    big = 1 << 40
    step = lambda *a: L.orthdion_muon_step(h, *a)  # noqa: E731
    assert step(None, p(256), p(256), p(256), big, None) == -3
    assert step(p(256), None, p(256), p(256), big, None) == -3
    assert step(p(256), p(256), None, p(256), big, None) == -3
    assert step(p(256), p(256), p(256), None, big, None) == -3
    assert step(p(264), p(256), p(256), p(256), big, None) == -6
    assert step(p(256), p(256), p(512), p(128), big, None) == -4       # workspace off its 256 bytes
    assert step(p(256), p(256), p(512), p(256), 100, None) == -4       # ... too small
    grouped = lambda hs, X, M, n=2: L.orthdion_muon_step_grouped(arr(*hs), n, arr(*X), arr(*M), arr(256, 256), p(256), big, None)  # noqa: E731
    assert grouped([h.value, h.value], [512, 512], [256, 1024]) == -1  # a matrix twice
    assert grouped([h.value, h.value], [512, 1024], [256, 256]) == -1
    assert grouped([h.value, h.value], [512, 1024], [256, 2048], 0) == -1
    assert L.orthdion_orthogonalize_grouped(None, 1, arr(256), arr(256), p(256), big, None) == -3
    assert L.orthdion_orthogonalize(h, p(256), p(264), p(256), big, None) == -6
    assert L.orthdion_muon_last_status(0, p(256), None, (ctypes.c_int32 * 1)()) == -1
    assert L.orthdion_muon_last_status(1, None, None, (ctypes.c_int32 * 1)()) == -3
    # a handle of another kind, and one that was given back
    other = p()
    assert L.orthdion_create(ctypes.byref(other), 64, 48, 16, 0.9, 0.1, 0.0, 0) == 0
    assert L.orthdion_muon_step(other, p(256), p(256), p(256), p(256), big, None) == -1
    assert L.orthdion_workspace_bytes(h) == 0 and L.orthdion_muon_workspace_bytes(other) == 0
    assert L.orthdion_destroy(other) == 0 and L.orthdion_muon_destroy(h) == 0


def test_workspace_holds_the_largest_batch_not_all_of_them(L):
    from paper_2605_16341_b200 import binding as od
    hs = [od.orthdion_muon_create(4096, 4096, 0.95, 0.02, 0.0) for _ in range(40)]
    one = od.orthdion_muon_workspace_bytes(hs[0])
    assert 2 * 2 * 4096 * 4096 <= one <= od.orthdion_muon_workspace_bytes_grouped(hs) <= (4 << 30) + (1 << 20)
    for h in hs:
        od.orthdion_muon_destroy(h)


def test_adamw_refuses(L):
    def create(numel=64, b1=0.9, b2=0.95, eps=1e-8, eta=1e-3, wd=0.1):
        h = ctypes.c_void_p()
        return L.orthdion_adamw_create(ctypes.byref(h), numel, b1, b2, eps, eta, wd), h
    nan = float("nan")
    for kw in (dict(numel=0), dict(numel=-5), dict(numel=(1 << 40) + 1), dict(b1=1.0), dict(b2=1.0), dict(b1=-0.1), dict(b2=nan), dict(eps=-1.0), dict(eps=nan),
               dict(eta=nan), dict(wd=nan)):
        rc, h = create(**kw)
        assert rc == -1 and not h.value, kw
    assert L.orthdion_adamw_create(None, 1, 0.9, 0.9, 0.0, 0.1, 0.0) == -3
    rc, h = create()
    assert rc == 0
    assert L.orthdion_adamw_set_dtypes(h, 3, 0) == -1 and L.orthdion_adamw_set_lr(h, nan) == -1
    p = ctypes.c_void_p
    step = lambda *a: L.orthdion_adamw_step(h, *a, None)  # noqa: E731
    ok = [p(256), p(512), p(1024), p(2048), p(4096)]
    for i in range(5):
        assert step(*[None if k == i else v for k, v in enumerate(ok)]) == -3
        assert step(*[p(v.value + 8) if k == i else v for k, v in enumerate(ok)]) == -6
    arr = lambda *v: (p * len(v))(*v)  # noqa: E731
    two = arr(h.value, h.value)
    assert L.orthdion_adamw_step_grouped(two, 2, arr(256, 256), arr(512, 1024), arr(2048, 4096), arr(256, 256), p(256), None) == -1
    assert L.orthdion_adamw_step_grouped(two, 0, arr(256), arr(512), arr(2048), arr(256), p(256), None) == -1
    assert L.orthdion_adamw_step_grouped(None, 1, arr(256), arr(512), arr(2048), arr(256), p(256), None) == -3
    assert L.orthdion_adamw_destroy(h) == 0 and L.orthdion_adamw_destroy(h) == -1
    assert step(*ok) == -1


def test_binding_checks_tensors_before_pointers():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the CPU tensors below are refused by another check there")
    from paper_2605_16341_b200 import binding as od
    with pytest.raises(ValueError):
        od.orthdion_muon_set_schedule(od.orthdion_muon_create(8, 8, 0.9, 0.1, 0.0), [(1.0, 2.0)])
    with pytest.raises(ValueError):
        od.MuonTable([], [], [], [])
