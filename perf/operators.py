"""Full-rank matrix steps and the step of everything that is no matrix, as a training program makes them.

A case is one call of an operator through `binding.py`:

  kind "orth"   the Newton-Schulz orthogonalisation of one matrix, `orthdion_orthogonalize`
  kind "muon"   one Muon step of some matrices of a model, `orthdion_muon_step_grouped`
  kind "adamw"  one AdamW step of some tensors of any length, `orthdion_adamw_step_grouped`

Ranges (`listed` and `draw` alike): matrices from 1 x 64 to 11008 x 4096, wide and tall, even and odd, up to 28 of them
in a call; three to seven steps of the iteration; tensors from one element to about 70 million; bfloat16 and float32
weights and gradients.  Gradients are noise and 64 (or fewer) strong directions, the momentum is what such gradients leave.
"""
import functools
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
#: Coefficients (a, b, c) of one step X <- a X + (b A + c A^2) X, A = X X^T: the ones that grow small singular values
#: fast and leave all of them near 1, and the ones that converge to 1.
POLY = {"fast": (3.4445, -4.7750, 2.0315), "smooth": (1.875, -1.25, 0.375)}
EPS = 1e-7                                   # added to the norm that the matrix is divided by
MU, ETA, WD = 0.95, 0.02, 0.1                # momentum, step size and decay of the Muon step
BETA1, BETA2, ADAM_EPS, ADAM_ETA, ADAM_WD = 0.9, 0.95, 1e-8, 3e-4, 0.1
MOST_FLOPS = 3.5e12                          # of a drawn case: no more than the largest listed one


def _orth(name, m, n, x="bf16", g="bf16", poly="fast", steps=5):
    return dict(name=name, kind="orth", shapes="%dx%d" % (m, n), x=x, g=g, poly=poly, steps=steps)


def _muon(name, shapes, x="bf16", g="bf16", nesterov=True, poly="fast", steps=5):
    return dict(name=name, kind="muon", shapes=shapes, x=x, g=g, nesterov=nesterov, poly=poly, steps=steps)


def _adamw(name, count, numel, x="bf16", g="bf16", odd=0, taken=1000):
    return dict(name=name, kind="adamw", count=count, numel=numel, odd=odd, x=x, g=g, taken=taken)


def listed():
    return [
        # the smallest layers of a model in full precision: one small matrix, latency only
        _orth("orth_256x512_f32", 256, 512, x="f32", g="f32"),
        # one MLP projection of a 320M model
        _orth("orth_768x2048", 768, 2048),
        # sizes that fit no tile, taller than wide, results in full precision
        _orth("orth_1023x777_f32", 1023, 777, x="f32", g="f32"),
        # one attention projection
        _orth("orth_4096x4096", 4096, 4096),
        # one tall MLP projection: the largest
        _orth("orth_11008x4096", 11008, 4096),
        # four layers of a 320M model in one call: many matrices, each too small for the whole GPU
        _muon("muon_320m_4_layers", "768x768*16 2048x768*8 768x2048*4"),
        # one layer of a 1.1B model
        _muon("muon_1b_layer", "2048x2048*4 5632x2048*2 2048x5632*1"),
        # key and value projections: wide, no look-ahead
        _muon("muon_1024x4096", "1024x4096*2", nesterov=False),
        # float32 weights under bfloat16 gradients, odd widths
        _muon("muon_mixed_1000", "1000x1000*4 376x1000*4 2712x1001*2", x="f32"),
        # norm weights: many short tensors
        _adamw("adamw_norms", 65, 4096),
        # an embedding, one element longer than a round number
        _adamw("adamw_embedding", 1, 32000 * 2048 + 1),
        # biases and norms of odd lengths in full precision, first step
        _adamw("adamw_ragged_f32", 40, 250_000, x="f32", g="f32", odd=37, taken=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["orth", "muon", "adamw"], [3, 3, 2])[0]
    x, g = rng.choices([("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")], [4, 2, 1, 1])[0]
    if kind == "adamw":
        count = _log(rng, 1, 60)
        return dict(kind=kind, count=count, numel=_log(rng, 1, 65_000_000 // count), odd=rng.randint(0, 99), x=x, g=g,
                    taken=rng.choice([0, 1, 30, 20000]))
    poly, steps = rng.choices([("fast", 5), ("smooth", 7), ("fast", 3), ("fast", 6)], [5, 1, 1, 1])[0]
    while True:
        if kind == "orth":
            lo = 1 if rng.random() < 0.1 else 64
            m, n = _log(rng, lo, 8192), _log(rng, 64, 8192)
            if rng.random() < 0.5:
                m, n = n, m
            case = dict(kind=kind, shapes="%dx%d" % (m, n), x=x, g=g, poly=poly, steps=steps)
        else:
            d = _log(rng, 128, 4096) // 8 * 8 + rng.choice([0, 0, 0, 1, 5])
            dff, count = int(d * rng.uniform(2, 4)), _log(rng, 1, 8)
            shapes = "%dx%d*%d %dx%d*%d" % (d, d, count, *rng.choice([(d, dff), (dff, d)]), max(1, count // 2))
            case = dict(kind=kind, shapes=shapes, x=x, g=g, nesterov=rng.random() < 0.5, poly=poly, steps=steps)
        terms = 3 if x == "f32" else 1
        if terms * work(case)["flops"] <= MOST_FLOPS and sum(m * n for m, n in _shapes(case)) <= 11008 * 4096:
            return case


def _shapes(case):
    """The matrices of a case, "MxN*COUNT ..." written out."""
    out = []
    for part in case["shapes"].split():
        mn, _, count = part.partition("*")
        m, n = (int(v) for v in mn.split("x"))
        out += [(m, n)] * int(count or 1)
    return out


def _lengths(case):
    """Lengths of the tensors of an AdamW case: `odd` takes something off every one but the first."""
    return [max(1, case["numel"] - k * case["odd"] * (1 + case["numel"] // 9000)) for k in range(case["count"])]


def _scale(m, n):
    return 0.2 * math.sqrt(max(m, n))       # an update as large as an adaptive method's


def _signal(m, n, gen):
    """Strong directions of a gradient: a product of two thin matrices, ten times the noise's largest singular value."""
    k = max(1, min(64, min(m, n) // 4))
    u = torch.randn(m, k, generator=gen, device="cuda") / math.sqrt(m)
    v = torch.randn(n, k, generator=gen, device="cuda") / math.sqrt(n)
    return 10 * (math.sqrt(m) + math.sqrt(n)) / math.sqrt(n) * (u @ v.T)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1009 + 17)
    xt, gt = DTYPES[case["x"]], DTYPES[case["g"]]
    s = {"case": case}
    if case["kind"] == "adamw":
        lengths = _lengths(case)
        new = lambda size: torch.randn(size, generator=gen, device="cuda")  # noqa: E731
        s["X"] = [(0.02 * new(k)).to(xt) for k in lengths]
        s["G"] = [(1e-3 * new(k)).to(gt) for k in lengths]
        first = case["taken"] == 0
        s["M"] = [torch.zeros(k, device="cuda") if first else 3e-4 * new(k) for k in lengths]
        s["V"] = [torch.zeros(k, device="cuda") if first else 1e-6 * new(k).square() + 1e-9 for k in lengths]
        s["step"] = torch.tensor([case["taken"], 0], dtype=torch.int64, device="cuda")
    else:
        shapes = _shapes(case)
        s["X"], s["M"], s["G"] = [], [], []
        for m, n in shapes:
            base = _signal(m, n, gen)
            s["G"].append((base + torch.randn(m, n, generator=gen, device="cuda") / math.sqrt(n)).to(gt))
            if case["kind"] == "muon":
                s["X"].append((0.02 * torch.randn(m, n, generator=gen, device="cuda")).to(xt))
                s["M"].append(0.6 * base + 0.16 / math.sqrt(n) * torch.randn(m, n, generator=gen, device="cuda"))
    if own:
        _plan(s, xt, gt)
    return s


@functools.cache
def _adamw_plan(numel, xt, gt):
    from paper_2605_16341_b200 import binding as od
    h = od.orthdion_adamw_create(numel, BETA1, BETA2, ADAM_EPS, ADAM_ETA, ADAM_WD)
    od.orthdion_adamw_set_dtypes(h, xt, gt)
    return h


@functools.cache
def _muon_plan(m, n, xt, gt, nesterov, poly, steps):
    from paper_2605_16341_b200 import binding as od
    h = od.orthdion_muon_create(m, n, MU, ETA, WD, nesterov)
    od.orthdion_muon_set_dtypes(h, xt, gt)
    od.orthdion_muon_set_scale(h, _scale(m, n))
    od.orthdion_muon_set_schedule(h, [POLY[poly]] * steps, EPS)
    return h


def _plan(s, xt, gt):
    """Handles, workspace and pointer tables, made once as the program starts."""
    from paper_2605_16341_b200 import binding as od
    case = s["case"]
    if case["kind"] == "adamw":
        hs = [_adamw_plan(k, xt, gt) for k in _lengths(case)]
        s["table"] = od.AdamWTable(hs, s["X"], s["M"], s["V"], s["G"])
        return
    hs = [_muon_plan(m, n, xt, gt, case.get("nesterov", True), case["poly"], case["steps"]) for m, n in _shapes(case)]
    s["ws"] = od.alloc_workspace(od.orthdion_muon_workspace_bytes_grouped(hs))
    if case["kind"] == "muon":
        s["table"] = od.MuonTable(hs, s["X"], s["M"], s["G"])
    else:
        s["h"], s["O"] = hs[0], torch.empty(*s["G"][0].shape, dtype=xt, device="cuda")


def _newton_schulz(b, abc, steps):
    """The orthogonalisation in 32 bits, its norm in 64 (a long sum)."""
    a, bb, c = abc
    x = b / (b.double().square().sum().sqrt() + EPS).float()
    wide = x.shape[0] <= x.shape[1]
    for _ in range(steps):
        p = x @ x.T if wide else x.T @ x
        p = bb * p + c * (p @ p)
        x = a * x + (p @ x if wide else x @ p)
    return x


def run(s):
    case = s["case"]
    if own:
        from paper_2605_16341_b200 import binding as od
        if case["kind"] == "orth":
            od.orthdion_orthogonalize(s["h"], s["G"][0], s["O"], s["ws"])
            return s["O"]
        if case["kind"] == "muon":
            od.orthdion_muon_step_grouped(s["table"], s["ws"])
            return s["X"], s["M"]
        od.orthdion_adamw_step_grouped(s["table"], s["step"])
        return _adamw_outputs(s)
    if case["kind"] == "orth":
        return _newton_schulz(s["G"][0].float(), POLY[case["poly"]], case["steps"]).to(DTYPES[case["x"]])
    if case["kind"] == "muon":
        for x, m, g in zip(s["X"], s["M"], s["G"]):
            g = g.float()
            m.copy_(MU * m + (1 - MU) * g)
            b = MU * m + (1 - MU) * g if case["nesterov"] else m
            o = _newton_schulz(b, POLY[case["poly"]], case["steps"])
            x.copy_((1 - ETA * WD) * x.float() - ETA * _scale(*x.shape) * o)
        return s["X"], s["M"]
    s["step"][0] += 1
    t = s["step"][0].double()
    c1, c2 = (1 - BETA1 ** t).float(), (1 - BETA2 ** t).float()
    for x, m, v, g in zip(s["X"], s["M"], s["V"], s["G"]):
        g, w = g.float(), x.float()
        m.copy_(BETA1 * m + (1 - BETA1) * g)
        v.copy_(BETA2 * v + (1 - BETA2) * g * g)
        x.copy_(w - ADAM_ETA * (ADAM_WD * w + (m / c1) / ((v / c2).sqrt() + ADAM_EPS)))
    return _adamw_outputs(s)


def _adamw_outputs(s):
    """All tensors; where that is many, those of one kind behind one another."""
    join = (lambda v: torch.cat(v)) if len(s["X"]) > 20 else (lambda v: v)
    return {"X": join(s["X"]), "M": join(s["M"]), "V": join(s["V"]), "step": s["step"][0]}


def work(case):
    size = {"bf16": 2, "f32": 4}
    x, g = size[case["x"]], size[case["g"]]
    if case["kind"] == "adamw":
        return {"bytes": sum(_lengths(case)) * (2 * x + g + 16), "flops": 0}
    flops = nbytes = 0
    for m, n in _shapes(case):
        # symmetric results are computed by half; the steps act on the matrix, or on the smaller side's products
        s, l, k = min(m, n), max(m, n), case["steps"]
        flops += min(k * (3 * s * s * l + s ** 3), 3 * s * s * l + (4 * k - 3) * s ** 3)
        nbytes += m * n * (g + (x if case["kind"] == "orth" else 2 * x + 8))
    return {"bytes": nbytes, "flops": flops}


def _polynomial(b, abc, steps):
    """X <- a X + b (X X^T) X + c (X X^T)^2 X in 64 bits, term by term on the taller orientation."""
    x = b.T if b.shape[0] < b.shape[1] else b
    x = x / (torch.linalg.matrix_norm(x) + EPS)
    for _ in range(steps):
        gram = x.T @ x
        third = x @ gram
        x = torch.add(torch.add(abc[0] * x, third, alpha=abc[1]), third @ gram, alpha=abc[2])
    return x.T if b.shape[0] < b.shape[1] else x


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adamw":
        t, out = case["taken"] + 1, {"X": [], "M": [], "V": []}
        for x, m, v, g in zip(s["X"], s["M"], s["V"], s["G"]):
            x, m, v, g = x.double(), m.double(), v.double(), g.double()
            m = m + (1 - BETA1) * (g - m)
            v = v + (1 - BETA2) * (g.square() - v)
            update = m / (1 - BETA1 ** t) / (torch.sqrt(v / (1 - BETA2 ** t)) + ADAM_EPS)
            out["X"].append(x * (1 - ADAM_ETA * ADAM_WD) - ADAM_ETA * update)
            out["M"].append(m)
            out["V"].append(v)
        if len(s["X"]) > 20:
            out = {k: torch.cat(v) for k, v in out.items()}
        return {**out, "step": None}
    if case["kind"] == "orth":
        return _polynomial(s["G"][0].double(), POLY[case["poly"]], case["steps"]).contiguous()
    xs, ms = [], []
    for x, m, g in zip(s["X"], s["M"], s["G"]):
        x, m, g = x.double(), m.double(), g.double()
        m = m + (1 - MU) * (g - m)
        b = m + (1 - MU) * (g - m) if case["nesterov"] else m
        o = _polynomial(b, POLY[case["poly"]], case["steps"])
        xs.append(x - ETA * (WD * x + _scale(*x.shape) * o))
        ms.append(m)
    return xs, ms
