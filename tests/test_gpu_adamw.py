"""The AdamW step against its definition in 64 bits, and a step of all kinds of parameters in one captured sequence."""
import pytest
import torch

from muon_util import FAST, HALF_STEP, adamw, gradient, muon, rel
from paper_2605_16341_b200 import binding as od

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def plan(numel, x=BF16, g=BF16, beta1=0.9, beta2=0.95, eps=1e-8, eta=3e-4, wd=0.1):
    h = od.orthdion_adamw_create(numel, beta1, beta2, eps, eta, wd)
    od.orthdion_adamw_set_dtypes(h, x, g)
    return h


def tensors(numel, x, g, first, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda: torch.randn(numel, generator=gen, device="cuda")  # noqa: E731
    X, G = (0.02 * new()).to(x), (1e-3 * new()).to(g)
    M, V = (torch.zeros(numel, device="cuda"), torch.zeros(numel, device="cuda")) if first else (3e-4 * new(), 1e-6 * new() ** 2 + 1e-10)
    return X, M, V, G


def counter(taken):
    return torch.tensor([taken, 0], dtype=torch.int64, device="cuda")


def check(X, M, V, want, before):
    """Entry by entry.  m and v: three roundings and the constants'.  X: the update passes about ten roundings, the weight four and
    the one of its type."""
    wx, wm, wv = want
    size = lambda a, b: a.double().abs().maximum(b.double().abs())  # noqa: E731
    assert bool(((V - wv).abs() <= 6 * 2.0 ** -24 * wv + 1e-44).all())
    assert bool(((M - wm).abs() <= 6 * 2.0 ** -24 * (size(before[1], before[3]) + wm.abs()) + 1e-44).all())
    # what a rounding of m (relative to its larger summand) does to the update
    step = (wx - before[0].double()).abs()
    lost = 6 * 2.0 ** -24 * size(before[1], before[3]) / (wm.abs() + 1e-300)
    tol = HALF_STEP[X.dtype] * wx.abs() + 4 * 2.0 ** -24 * before[0].double().abs() + (16 * 2.0 ** -24 + lost) * step
    off = (X.double() - wx).abs()
    assert bool((off <= 1.001 * tol + 1e-44).all()), (off - tol).max().item()


@pytest.mark.parametrize("taken", [0, 1, 1000, 10 ** 6])
@pytest.mark.parametrize("x,g", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("numel", [1, 7, 8, 4096, 4097, 100_003])
def test_one_tensor(numel, x, g, taken):
    for kw in ({}, dict(beta1=0.0, beta2=0.999, wd=0.0), dict(beta1=0.95, beta2=0.9999, eps=1e-6, eta=0.01)):
        X, M, V, G = tensors(numel, x, g, taken == 0)
        before = [t.clone() for t in (X, M, V, G)]
        p = dict(beta1=0.9, beta2=0.95, eps=1e-8, eta=3e-4, wd=0.1) | kw
        f = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731  (eps, eta, wd travel in 32 bits)
        want = adamw(*before, taken + 1, p["beta1"], p["beta2"], f(p["eps"]), f(p["eta"]), f(p["wd"]))
        step = counter(taken)
        od.orthdion_adamw_step(plan(numel, x, g, **p), X, M, V, G, step)
        assert step.tolist() == [taken + 1, 0]
        check(X, M, V, want, before)
        assert torch.equal(G, before[3])


def test_many_tensors_of_all_types_in_one_call():
    """More tensors, and more different constants, than one launch holds; against single calls, bit for bit."""
    cases = [(1 + 37 * i % 5000, (BF16, F32)[i % 2], (BF16, F32)[i // 2 % 2], 1e-4 * (1 + i % 11)) for i in range(150)]
    hs = [plan(n, x, g, eta=eta) for n, x, g, eta in cases]
    state = [tensors(n, x, g, False, i) for i, (n, x, g, _) in enumerate(cases)]
    alone = [[t.clone() for t in s] for s in state]
    step = counter(5)
    table = od.AdamWTable(hs, *[list(v) for v in zip(*state)])
    for _ in range(3):
        od.orthdion_adamw_step_grouped(table, step)
    assert step.tolist() == [8, 0]
    for h, s, a in zip(hs, state, alone):
        one = counter(5)
        for _ in range(3):
            od.orthdion_adamw_step(h, *a, one)
        assert all(torch.equal(p, q) for p, q in zip(s, a))


def test_entries_behind_the_end_are_left():
    for x in (BF16, F32):
        full = [torch.full((4120,), 9.0, device="cuda", dtype=t) for t in (x, F32, F32, x)]
        step = counter(0)
        od.orthdion_adamw_step(plan(4101, x, x), *[t[:4101] for t in full], step)
        # (inside, v becomes 0.95 * 9 + 0.05 * 81)
        assert all(bool((t[4101:] == 9).all()) for t in full) and not bool((full[2][:4101] == 9).any())


def test_zero_gradients_and_non_finite_ones():
    X, M, V, G = tensors(1000, F32, F32, True)
    G.zero_()
    before = X.clone()
    od.orthdion_adamw_step(plan(1000, F32, F32, wd=0.0), X, M, V, G, counter(0))
    assert torch.equal(X, before) and M.abs().max().item() == 0 and V.abs().max().item() == 0
    G[5], G[6] = float("nan"), float("inf")      # no entry reaches another one
    od.orthdion_adamw_step(plan(1000, F32, F32, wd=0.0), X, M, V, G, counter(1))
    keep = torch.ones(1000, dtype=torch.bool, device="cuda")
    keep[5:7] = False
    assert torch.equal(X[keep], before[keep]) and not bool(torch.isfinite(X[5:7]).any())


def test_refusals():
    h = plan(64)
    X, M, V, G = tensors(64, BF16, BF16, True)
    step = counter(0)
    for bad in ((X.float(), M, V, G), (X, M.to(BF16), V, G), (X, M, V, G.float()), (X[:63], M, V, G), (X.cpu(), M, V, G)):
        with pytest.raises(ValueError):
            od.orthdion_adamw_step(h, *bad, step)
    with pytest.raises(ValueError):
        od.orthdion_adamw_step(h, X, M, V, G, torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(od.OrthDionError) as e:
        od.orthdion_adamw_step_grouped(od.AdamWTable([h, h], [X, X], [M, M.clone()], [V, V.clone()], [G, G]), step)
    assert e.value.code == -1
    with pytest.raises(od.OrthDionError) as e:
        od.orthdion_adamw_step(plan(56), X[8:].clone(), M[8:].clone(), torch.zeros(64, device="cuda")[1:57], G[8:].clone(), step)
    assert e.value.code == -6
    torch.cuda.synchronize()
    assert step.tolist() == [0, 0]


def test_a_model_of_all_three_kinds_captured_and_replayed():
    """A low-rank step for the MLP matrices, Muon for the attention ones, AdamW for embedding and norms: one captured sequence,
    replayed, against the same calls made eagerly, and the Muon and AdamW parts against their definitions."""
    def build():
        gen = torch.Generator(device="cuda").manual_seed(3)
        new = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        low = [(m, n, (0.02 * new(m, n)).to(BF16), torch.zeros(m, n, device="cuda"), new(m, n).to(BF16),
                torch.linalg.qr(new(n, 32))[0].contiguous()) for m, n in ((512, 256), (256, 512))]
        full = [((0.02 * new(256, 256)).to(BF16), torch.zeros(256, 256, device="cuda"), gradient("spikes", 256, 256, k, BF16)) for k in range(3)]
        rest = [tensors(k, BF16, BF16, True, k) for k in (1000 * 256, 256, 256, 257)]
        return low, full, rest

    hl = [od.orthdion_create(m, n, 32, 0.95, 0.01, 0.0, od.MODE_ORTH) for m, n in ((512, 256), (256, 512))]
    hm = od.orthdion_muon_create(256, 256, 0.95, 0.02, 0.1, True)
    wl = od.alloc_workspace(od.orthdion_workspace_bytes_grouped(hl))
    wm = od.alloc_workspace(od.orthdion_muon_workspace_bytes_grouped([hm] * 3))

    def tables(state):
        low, full, rest = state
        t = od.PointerTable(hl, [v[2] for v in low], [v[3] for v in low], [v[4] for v in low], [v[5] for v in low])
        u = od.MuonTable([hm] * 3, *[list(v) for v in zip(*full)])
        a = od.AdamWTable([plan(v[0].numel()) for v in rest], *[list(v) for v in zip(*rest)])
        return t, u, a, counter(0)

    def steps(t, u, a, step):
        od.orthdion_step_grouped(t, wl)
        od.orthdion_muon_step_grouped(u, wm)
        od.orthdion_adamw_step_grouped(a, step)

    eager, captured = build(), build()
    te, tc = tables(eager), tables(captured)
    first = [(X.clone(), M.clone(), G) for X, M, G in eager[1]], [[t.clone() for t in v] for v in eager[2]]
    steps(*te)
    for (X0, M0, G), (X, M, _) in zip(first[0], eager[1]):
        want, wm_, _, _ = muon(X0, M0, G, 0.95, 0.02, 0.1, 1.0, True, [FAST] * 5)
        assert rel(X, want) <= 5e-3 and rel(M, wm_) <= 2.0 ** -22
    for before, now in zip(first[1], eager[2]):
        f = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
        check(*now[:3], adamw(*before, 1, 0.9, 0.95, f(1e-8), f(3e-4), f(0.1)), before)
    for _ in range(3):
        steps(*te)
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        steps(*tc)
    for _ in range(4):
        g.replay()
    torch.cuda.synchronize()
    assert tc[3].tolist() == te[3].tolist() == [4, 0]
    for a, b in zip(captured, eager):
        for u, v in zip(a, b):
            assert all(torch.equal(p, q) for p, q in zip(u, v) if isinstance(p, torch.Tensor))
