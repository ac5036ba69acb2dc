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


class Fake:
    """A CUDA tensor as far as the binding looks at one."""

    def __init__(self, ptr, shape, dtype, device=0):
        import torch
        self.ptr, self.shape, self.dtype, self.device, self.is_cuda = ptr, tuple(shape), dtype, torch.device("cuda", device), True

    def stride(self, k):
        return (self.shape[1], 1)[k]

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.ptr


def test_tables_are_checked_again_before_a_call(L, monkeypatch):
    """Plans that changed or went, and tensors of another device than the current one, are refused before a pointer is handed on."""
    import torch
    from paper_2605_16341_b200 import binding as od
    current = [0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(od, "_stream_ptr", lambda stream: 0)
    bf, f32 = torch.bfloat16, torch.float32
    h = od.orthdion_muon_create(64, 48, 0.9, 0.1, 0.0)
    a = od.orthdion_adamw_create(100, 0.9, 0.95, 1e-8, 0.1, 0.0)
    X, M, G = Fake(256, (64, 48), bf), Fake(1 << 20, (64, 48), f32), Fake(2 << 20, (64, 48), bf)
    ws, off = Fake(3 << 20, (64,), torch.uint8), Fake(3 << 20, (64,), torch.uint8, 1)
    table = od.MuonTable([h], [X], [M], [G])
    with pytest.raises(od.OrthDionError) as e:          # as far as the library: the workspace is too small
        od.orthdion_muon_step_grouped(table, ws)
    assert e.value.code == -4
    with pytest.raises(ValueError):
        od.orthdion_muon_step_grouped(table, off)
    v = [Fake(k << 20, (100,), d) for k, d in ((5, bf), (6, f32), (7, f32), (8, bf))]
    step, far = Fake(9 << 20, (2,), torch.int64), Fake(9 << 20, (2,), torch.int64, 1)
    adamw = od.AdamWTable([a], *[[t] for t in v])
    with pytest.raises(ValueError):
        od.orthdion_adamw_step_grouped(adamw, far)
    current[0] = 1
    for call in (lambda: od.orthdion_muon_step_grouped(table, off), lambda: od.orthdion_orthogonalize_grouped(table, off),
                 lambda: od.orthdion_adamw_step_grouped(adamw, far), lambda: od.orthdion_muon_step(h, X, M, G, off)):
        with pytest.raises(ValueError):
            call()
    current[0] = 0
    for bad in (lambda: od.MuonTable([a], [X], [M], [G]), lambda: od.AdamWTable([h], *[[t] for t in v])):
        with pytest.raises(od.OrthDionError):
            bad()
    od.orthdion_muon_set_dtypes(h, bf, f32)
    od.orthdion_adamw_set_dtypes(a, f32, bf)
    with pytest.raises(ValueError):
        od.orthdion_muon_step_grouped(table, ws)
    with pytest.raises(ValueError):
        od.orthdion_adamw_step_grouped(adamw, step)
    od.orthdion_muon_set_dtypes(h, bf, bf)
    od.orthdion_muon_set_ld(h, 56, 48, 48)
    with pytest.raises(ValueError):
        od.orthdion_muon_step_grouped(table, ws)
    od.orthdion_muon_destroy(h)
    od.orthdion_adamw_destroy(a)
    for call in (lambda: od.orthdion_muon_step_grouped(table, ws), lambda: od.orthdion_adamw_step_grouped(adamw, step)):
        with pytest.raises(od.OrthDionError) as e:
            call()
        assert e.value.code == -1
