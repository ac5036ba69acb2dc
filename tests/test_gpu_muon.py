"""The Newton-Schulz orthogonalisation and the Muon step against their definitions in 64 bits."""
import pytest
import torch

from muon_util import FAST, SMOOTH, HALF_STEP, STATED, bound, gradient, muon, orthogonalise, rel
from paper_2605_16341_b200 import binding as od

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def plan(m, n, x=BF16, g=BF16, mu=0.95, eta=0.02, wd=0.1, nesterov=True, schedule=None, eps=1e-7, scale=1.0, passes=0, ld=None):
    h = od.orthdion_muon_create(m, n, mu, eta, wd, nesterov)
    od.orthdion_muon_set_dtypes(h, x, g)
    od.orthdion_muon_set_scale(h, scale)
    if schedule is not None:
        od.orthdion_muon_set_schedule(h, schedule, eps)
    od.orthdion_muon_set_passes(h, passes)
    if ld:
        od.orthdion_muon_set_ld(h, *ld)
    return h


def workspace(hs, fill=0x7f):
    ws = od.alloc_workspace(od.orthdion_muon_workspace_bytes_grouped(hs))
    ws.fill_(fill)              # NaN wherever a kernel would read what it has not written
    return ws


def orth(G, x=None, schedule=None, **kw):
    h = plan(*G.shape, x=x or G.dtype, g=G.dtype, schedule=schedule, **kw)
    ws, O = workspace([h]), torch.full(G.shape, float("nan"), dtype=x or G.dtype, device="cuda")
    od.orthdion_orthogonalize(h, G, O, ws)
    assert od.orthdion_muon_last_status(1, ws) == [0]
    od.orthdion_muon_destroy(h)
    return O


SHAPES = [(1, 1), (1, 64), (64, 1), (2, 3), (31, 33), (100, 37), (37, 100), (128, 128), (129, 127), (257, 513), (300, 300),
          (640, 1000), (1000, 129), (520, 2056), (2049, 130), (1151, 1153)]


@pytest.mark.parametrize("x,g", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)], ids=["bf16", "f32", "bf16_of_f32", "f32_of_bf16"])
@pytest.mark.parametrize("m,n", SHAPES)
def test_orthogonalise(m, n, x, g):
    for seed, kind in enumerate(("noise", "spikes", "decay")):
        G = gradient(kind, m, n, seed, g)
        ref = orthogonalise(G, [FAST] * 5)
        passes = 3 if x == F32 else 1
        tol = min(STATED[passes], bound(G, [FAST] * 5, passes, x, exact_input=g == BF16))
        assert rel(orth(G, x), ref) <= tol, (kind, rel(orth(G, x), ref), tol)


@pytest.mark.parametrize("passes", [1, 3])
@pytest.mark.parametrize("schedule", [[FAST], [FAST] * 2, [FAST] * 3, [FAST] * 6, [SMOOTH] * 7, [FAST] * 2 + [SMOOTH] * 2, [SMOOTH] * 32, [(1.0, 0.0, 0.0)],
                                      [(1.5, -0.5, 0.0)] * 4], ids=["1", "2", "3", "6", "smooth7", "mixed", "smooth32", "identity", "cubic4"])
def test_schedules(schedule, passes):
    for m, n in ((200, 333), (333, 200), (260, 260)):
        G = gradient("spikes", m, n, 3, BF16)
        ref = orthogonalise(G, schedule)
        got = orth(G, F32, schedule, passes=passes)
        assert rel(got, ref) <= bound(G, schedule, passes, F32, exact_input=True), (m, n, rel(got, ref))


@pytest.mark.parametrize("factor", [1e-36, 1e-20, 1e-6, 1e6, 1e20, 1e36])
def test_magnitudes(factor):
    # the norm is summed in 64 bits: no square overflows or vanishes.  (eps 0: the result does not depend on the factor)
    G = gradient("spikes", 130, 70, 1, F32) * factor
    ref = orthogonalise(G, [FAST] * 5, 0.0)
    tol = bound(G, [FAST] * 5, 3, F32, 0.0)
    if factor == 1e-36:          # entries are subnormal: 2^-149 apart, which is an error of the input
        tol += 2.0 ** -149 * 70 * 130 / G.double().norm().item() * 500
    assert rel(orth(G, F32, [FAST] * 5, eps=0.0), ref) <= min(tol, STATED[3])


@pytest.mark.parametrize("m,n", [(40, 104), (41, 103)])
def test_one_entry_above_all_others(m, n):
    # its square overflows 32 bits, the others' do not: rank one as far as fp32 can tell
    G = gradient("noise", m, n, 4, F32)
    G[3, 5] = 1e30
    assert rel(orth(G, F32), orthogonalise(G, [FAST] * 5)) <= STATED[3]


def test_zeros_stay_zeros_and_eps_counts():
    for eps in (0.0, 1e-7):
        assert orth(torch.zeros(70, 90, device="cuda"), F32, [FAST] * 5, eps=eps).abs().max().item() == 0.0
    G = gradient("noise", 70, 90, 1, F32)
    G = G / G.norm()
    assert rel(orth(G, F32, [FAST] * 5, eps=0.5), orthogonalise(G, [FAST] * 5, 0.5)) <= min(STATED[3], bound(G, [FAST] * 5, 3, F32, 0.5))
    # one entry; one row; orthonormal rows, whose singular values all take the same way
    G = torch.zeros(65, 65, device="cuda")
    G[7, 60] = -3.0
    assert rel(orth(G, F32), orthogonalise(G, [FAST] * 5)) <= STATED[3]
    Q = torch.linalg.qr(torch.randn(300, 200, device="cuda", dtype=torch.float64))[0].float().contiguous()
    assert rel(orth(Q, F32), orthogonalise(Q, [FAST] * 5)) <= STATED[3]
    assert rel(orth(Q.T.contiguous(), F32), orthogonalise(Q.T, [FAST] * 5)) <= STATED[3]


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_non_finite_matrices_keep_their_state(bad):
    hs = [plan(66, 50), plan(50, 66), plan(66, 50)]
    Gs = [gradient("noise", 66, 50, 1, BF16), gradient("noise", 50, 66, 2, BF16), gradient("noise", 66, 50, 3, BF16)]
    Xs = [torch.randn(g.shape, device="cuda").to(BF16) for g in Gs]
    Ms = [torch.randn(g.shape, device="cuda") for g in Gs]
    Gs[0][65, 49] = bad
    before = [t.clone() for t in (Xs[0], Ms[0])]
    want = [muon(X, M, G, 0.95, 0.02, 0.1, 1.0, True, [FAST] * 5) for X, M, G in zip(Xs, Ms, Gs)]
    ws = workspace(hs)
    od.orthdion_muon_step_grouped(od.MuonTable(hs, Xs, Ms, Gs), ws)
    assert od.orthdion_muon_last_status(3, ws) == [od.STATUS_NONFINITE, 0, 0]
    assert torch.equal(Xs[0], before[0]) and torch.equal(Ms[0], before[1])
    for k in (1, 2):
        assert rel(Ms[k], want[k][1]) <= 2.0 ** -22 and rel(Xs[k], want[k][0]) <= STATED[1]
    O = torch.full((66, 50), 7.0, dtype=BF16, device="cuda")
    od.orthdion_orthogonalize(hs[0], Gs[0], O, ws)
    assert od.orthdion_muon_last_status(1, ws) == [od.STATUS_NONFINITE] and bool((O == 7).all())
    # and the next step with a clean gradient is an ordinary one
    Gs[0][65, 49] = 0.0
    od.orthdion_muon_step(hs[0], Xs[0], Ms[0], Gs[0], ws)
    assert od.orthdion_muon_last_status(1, ws) == [0]
    assert rel(Ms[0], 0.95 * before[1].double() + 0.05 * Gs[0].double()) <= 2.0 ** -22


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("x,g", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("m,n", [(1, 200), (96, 96), (131, 259), (520, 264)])
def test_muon_chain(m, n, x, g, nesterov):
    """Three steps; the reference carries its own momentum and takes the weights that the library has stored."""
    scale, eta, wd, mu = 0.2 * max(m, n) ** 0.5, 0.02, 0.1, 0.9
    h = plan(m, n, x, g, mu, eta, wd, nesterov, scale=scale)
    ws = workspace([h])
    X = (0.02 * torch.randn(m, n, device="cuda")).to(x)
    M, ref_m = torch.zeros(m, n, device="cuda"), torch.zeros(m, n, device="cuda", dtype=torch.float64)
    for step in range(3):
        G = gradient("spikes", m, n, step, g)
        before = X.clone()
        want, ref_m, B, O = muon(before, ref_m, G, mu, eta, wd, scale, nesterov, [FAST] * 5)
        od.orthdion_muon_step(h, X, M, G, ws)
        assert od.orthdion_muon_last_status(1, ws) == [0]
        # mu M + (1 - mu) G: three roundings and the two constants' a step, carried on
        assert rel(M, ref_m) <= (step + 1) * 5 * 2.0 ** -24
        passes = 3 if x == F32 else 1
        tol = eta * scale * O.norm().item() * min(STATED[passes], bound(B, [FAST] * 5, passes, F32) + 500 * (step + 1) * 5 * 2.0 ** -24)
        tol = tol / want.norm().item() + HALF_STEP[x] + 3 * 2.0 ** -24
        assert rel(X, want) <= tol, (step, rel(X, want), tol)


def test_grouped_call_gives_the_bits_of_single_calls():
    shapes = [(64, 200)] * 70 + [(200, 64)] * 3 + [(300, 300)] * 2 + [(1, 9)] + [(64, 200)] * 2
    hs = [plan(m, n) for m, n in shapes]
    hs[-1] = plan(64, 200, eta=0.5)             # of equal shape, another plan
    Gs = [gradient("spikes", m, n, i, BF16) for i, (m, n) in enumerate(shapes)]
    Xs = [(0.02 * torch.randn(m, n, device="cuda")).to(BF16) for m, n in shapes]
    Ms = [0.1 * torch.randn(m, n, device="cuda") for m, n in shapes]
    single = [(X.clone(), M.clone()) for X, M in zip(Xs, Ms)]
    ws = workspace(hs)
    od.orthdion_muon_step_grouped(od.MuonTable(hs, Xs, Ms, Gs), ws)
    assert od.orthdion_muon_last_status(len(hs), ws) == [0] * len(hs)
    for h, (X, M), G, gx, gm in zip(hs, single, Gs, Xs, Ms):
        od.orthdion_muon_step(h, X, M, G, workspace([h], 0))
        assert torch.equal(X, gx) and torch.equal(M, gm)


@pytest.mark.parametrize("x", [BF16, F32])
@pytest.mark.parametrize("m,n,count", [(257, 513, 9), (513, 257, 9), (700, 333, 5), (100, 37, 30), (520, 2056, 5), (1151, 1153, 2), (2049, 130, 26), (1800, 1800, 1)])
def test_large_tiles(m, n, count, x):
    """Calls with many tiles, which are larger then: against the definition, and the bits of calls with small ones (but where one matrix has
    many tiles of its own)."""
    hs = [plan(m, n, x=x)] * count
    Gs = [gradient(("noise", "spikes", "decay")[i % 3], m, n, i, BF16) for i in range(count)]
    Os = [torch.full((m, n), float("nan"), dtype=x, device="cuda") for _ in range(count)]
    ws = workspace(hs)
    od.orthdion_orthogonalize_grouped(od.MuonTable(hs, Os, None, Gs), ws)
    assert od.orthdion_muon_last_status(count, ws) == [0] * count
    for G, O in list(zip(Gs, Os))[:3]:
        passes = 3 if x == F32 else 1
        tol = min(STATED[passes], bound(G, [FAST] * 5, passes, x, exact_input=True))
        assert rel(O, orthogonalise(G, [FAST] * 5)) <= tol
        assert torch.equal(O, orth(G, x))


@pytest.mark.parametrize("x", [BF16, F32])
@pytest.mark.parametrize("m,n,count", [(64, 2048, 1), (7, 8191, 2), (5000, 100, 1), (300, 2500, 20), (1024, 2100, 2), (1025, 2100, 1),
                                       (3, 200_003, 1), (70_001, 129, 1)])
def test_long_matrices(m, n, count, x):
    """Few rows (or columns) and a long other side, whose first product is computed in parts: against the definition, repeatably, and
    with the same bits in a call of several."""
    hs = [plan(m, n, x=x)] * count
    Gs = [gradient(("spikes", "noise")[i % 2], m, n, i, BF16) for i in range(count)]
    outs = []
    for _ in range(2):
        Os = [torch.full((m, n), float("nan"), dtype=x, device="cuda") for _ in range(count)]
        ws = workspace(hs)
        od.orthdion_orthogonalize_grouped(od.MuonTable(hs, Os, None, Gs), ws)
        assert od.orthdion_muon_last_status(count, ws) == [0] * count
        outs.append(Os)
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    for G, O in list(zip(Gs, outs[0]))[:3]:
        ref = orthogonalise(G if m <= n else G.T, [FAST] * 5)
        passes = 3 if x == F32 else 1
        assert rel(O, ref if m <= n else ref.T) <= STATED[passes]
        assert torch.equal(O, orth(G, x))


def test_more_plans_than_one_launch_takes():
    """Nine plans, both pass counts, in one call: several launches, which use the same scratch one after the other."""
    shapes = [(64 + 8 * k, 200) for k in range(9)] * 2
    hs = [plan(m, n, x=(BF16, F32)[i % 2]) for i, (m, n) in enumerate(shapes)]
    Gs = [gradient("spikes", m, n, i, BF16) for i, (m, n) in enumerate(shapes)]
    Xs = [(0.02 * torch.randn(m, n, device="cuda")).to((BF16, F32)[i % 2]) for i, (m, n) in enumerate(shapes)]
    Ms = [0.1 * torch.randn(m, n, device="cuda") for m, n in shapes]
    single = [(X.clone(), M.clone()) for X, M in zip(Xs, Ms)]
    ws = workspace(hs)
    od.orthdion_muon_step_grouped(od.MuonTable(hs, Xs, Ms, Gs), ws)
    assert od.orthdion_muon_last_status(len(hs), ws) == [0] * len(hs)
    for h, (X, M), G, gx, gm in zip(hs, single, Gs, Xs, Ms):
        od.orthdion_muon_step(h, X, M, G, workspace([h], 0))
        assert torch.equal(X, gx) and torch.equal(M, gm)


@pytest.mark.parametrize("passes", [1, 3])
@pytest.mark.parametrize("tail", [[], [FAST, FAST]], ids=["three", "five"])
def test_steep_schedules(tail, passes):
    """Two steps whose factors together (20 and 7) are beyond what an image holds are taken one by one, in front of a pair or not."""
    steep = [(20.0, -50.0, 32.0), (7.0, -0.9, 0.024), (0.125, 0.0, 0.0)] + tail
    for m, n in ((600, 1300), (100, 260), (260, 200)):
        G = gradient("spikes", m, n, 2, BF16)
        got = orth(G, F32, steep, passes=passes)
        assert rel(got, orthogonalise(G, steep)) <= bound(G, steep, passes, F32, exact_input=True, pairs=(False, True))


def test_grouped_orthogonalise_and_in_place():
    shapes = [(64, 200), (200, 64), (64, 200)]
    hs = [plan(m, n) for m, n in shapes]
    Gs = [gradient("noise", m, n, i, BF16) for i, (m, n) in enumerate(shapes)]
    Os = [torch.empty_like(G) for G in Gs]
    ws = workspace(hs)
    od.orthdion_orthogonalize_grouped(od.MuonTable(hs, Os, None, Gs), ws)
    for h, G, O in zip(hs, Gs, Os):
        assert torch.equal(orth(G), O)
        od.orthdion_orthogonalize(h, G, G, ws)
        assert torch.equal(G, O)


@pytest.mark.parametrize("m,n,lds", [(65, 40, (48, 44, 56)), (65, 41, (43, 47, 42)), (40, 264, (264, 300, 272))])
def test_rows_further_apart(m, n, lds):
    """Columns of wider matrices: what lies beside them is left as it was, NaN there does not count."""
    h, hc = plan(m, n, ld=lds), plan(m, n)
    wide = [torch.full((m, ld), float("nan"), device="cuda", dtype=t) for ld, t in zip(lds, (BF16, F32, BF16))]
    X, M, G = [w[:, :n] for w in wide]
    G.copy_(gradient("spikes", m, n, 5, BF16)); M.normal_(); X.normal_()
    Xc, Mc, Gc = [t.contiguous().clone() for t in (X, M, G)]
    od.orthdion_muon_step(h, X, M, G, workspace([h]))
    od.orthdion_muon_step(hc, Xc, Mc, Gc, workspace([hc]))
    # (columns that start on no 16-byte boundary go another way to the same sums of squares, in another order: 2^-50 of the norm)
    assert torch.equal(M, Mc) and rel(X, Xc) <= HALF_STEP[BF16]
    for w in wide:
        assert bool(w[:, n:].isnan().all())
    O = torch.full((m, lds[0]), 5.0, device="cuda", dtype=BF16)
    od.orthdion_orthogonalize(h, G, O[:, :n], workspace([h]))
    assert bool((O[:, n:] == 5).all()) and rel(O[:, :n], orthogonalise(Gc, [FAST] * 5)) <= STATED[1]


def test_repeatable_and_free_of_what_the_workspace_held():
    G = gradient("spikes", 700, 333, 9, BF16)
    h = plan(700, 333)
    outs = []
    for fill in (0x7f, 0x00, 0xff):
        ws, O = workspace([h], fill), torch.empty(700, 333, dtype=BF16, device="cuda")
        for _ in range(3):
            od.orthdion_orthogonalize(h, G, O, ws)
            outs.append(O.clone())
    assert all(torch.equal(o, outs[0]) for o in outs)


def test_captured_calls_on_other_streams_side_by_side():
    """Two captured steps with a workspace each, replayed at the same time on two streams, against eager calls."""
    shapes = [[(256, 640), (256, 640), (640, 256)], [(512, 512)]]
    states, graphs, streams = [], [], [torch.cuda.Stream() for _ in shapes]
    for k, sh in enumerate(shapes):
        hs = [plan(m, n) for m, n in sh]
        Gs = [gradient("spikes", m, n, 10 * k + i, BF16) for i, (m, n) in enumerate(sh)]
        Xs = [(0.02 * torch.randn(m, n, device="cuda")).to(BF16) for m, n in sh]
        Ms = [torch.zeros(m, n, device="cuda") for m, n in sh]
        eager = ([X.clone() for X in Xs], [M.clone() for M in Ms])
        ws = workspace(hs)
        warm = od.MuonTable(hs, [X.clone() for X in Xs], [M.clone() for M in Ms], Gs)
        od.orthdion_muon_step_grouped(warm, ws)
        torch.cuda.synchronize()
        table, g = od.MuonTable(hs, Xs, Ms, Gs), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[k]):
            od.orthdion_muon_step_grouped(table, ws)
        states.append((hs, Xs, Ms, Gs, eager, ws, table))
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(4):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for hs, Xs, Ms, Gs, (eX, eM), ws, _ in states:
        t = od.MuonTable(hs, eX, eM, Gs)
        for _ in range(4):
            od.orthdion_muon_step_grouped(t, workspace(hs))
        for a, b in zip(Xs + Ms, eX + eM):
            assert torch.equal(a, b)


def test_gpu_refusals():
    h = plan(64, 48)
    ws = workspace([h])
    X, M, G = torch.zeros(64, 48, dtype=BF16, device="cuda"), torch.zeros(64, 48, device="cuda"), torch.zeros(64, 48, dtype=BF16, device="cuda")
    with pytest.raises(od.OrthDionError) as e:
        od.orthdion_muon_step(h, X, M, G, ws[: ws.numel() - 1024])
    assert e.value.code == -4
    with pytest.raises(od.OrthDionError) as e:
        od.orthdion_muon_step(h, X, M, G, ws[16:])
    assert e.value.code == -4
    for bad in ((X.float(), M, G), (X, M.to(BF16), G), (X, M, G.float()), (X.T, M, G), (X[:, :40], M, G), (X.cpu(), M, G),
                (torch.zeros(64, 56, dtype=BF16, device="cuda")[:, :48], M, G)):
        with pytest.raises((ValueError, od.OrthDionError)):
            od.orthdion_muon_step(h, *bad, ws)
    off = torch.zeros(64 * 48 + 1, dtype=BF16, device="cuda")[1:].view(64, 48)
    with pytest.raises(od.OrthDionError) as e:
        od.orthdion_muon_step(h, off, M, G, ws)
    assert e.value.code == -6
    for Xs, Ms in (([X, X], [M, M.clone()]), ([X, X.clone()], [M, M])):
        with pytest.raises(od.OrthDionError) as e:
            od.orthdion_muon_step_grouped(od.MuonTable([h, h], Xs, Ms, [G, G]), workspace([h, h]))
        assert e.value.code == -1
    torch.cuda.synchronize()
    assert X.abs().max().item() == 0 and M.abs().max().item() == 0
