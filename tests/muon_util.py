"""Plain statements of the full-rank step and of AdamW in 64 bits, and how far the library's results may be from them.

The bound of the orthogonalisation counts what the library rounds (see `orthogonalise`): every stored intermediate
to u relative to each entry, every sum by gamma relative to the sum of its terms' magnitudes.  A rounding is off by at most half a
step: fp16 2^-11, bf16 2^-8.  Two-term operands are off by 2^-22 and their product drops a term of 2^-22.  An addition in tensor
memory truncates: 2^-23 each; one product of depth K there is K/16 of them (one-term operands), or 12 for each 64 deep and one rounded
addition (2^-24) for each 64; up to 32 partial sums of a long depth are added up (2^-24 each).  Errors in X pass a step with its
Lipschitz constant, max |p'| over the singular values' range (the map of singular values is odd, so this bounds the matrix map in the
Frobenius norm).
"""
import torch

FAST = (3.4445, -4.7750, 2.0315)
SMOOTH = (1.875, -1.25, 0.375)
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
#: What the header says of the error relative to the result: 4e-3 and the rounding of a bf16 result, about 2e-6.
STATED = {1: 5e-3, 3: 1e-5}


def orthogonalise(B, schedule, eps=1e-7):
    """X0 = B / (|B| + eps), X <- a X + (b A + c A^2) X, from the definition in 64 bits."""
    X = B.double()
    X = X / (torch.linalg.matrix_norm(X) + eps)
    for a, b, c in schedule:
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return X


def bound(B, schedule, passes, x_dtype, eps=1e-7, exact_input=False, pairs=(True, True)):
    """Largest ||O - exact||_F / ||exact||_F that the roundings above can add up to."""
    X = B.double()
    if X.shape[0] > X.shape[1]:
        X = X.T
    X = X / (torch.linalg.matrix_norm(X) + eps)
    s, l = X.shape
    u = 2.0 ** -11 if passes == 1 else 2.0 ** -22
    drop = 0.0 if passes == 1 else 2.0 ** -22

    def gamma(depth):
        blocks = -(-depth // 64)
        return drop + 32 * 2.0 ** -24 + (blocks * 4 * 2.0 ** -23 if passes == 1 else 12 * 2.0 ** -23 + blocks * 2.0 ** -24)

    fro = lambda t: torch.linalg.matrix_norm(t).item()  # noqa: E731

    def two(t):         # the square ones are symmetric, or (X itself) of few rows
        sym = t.shape[0] == t.shape[1] and torch.equal(t, t.T)
        return torch.linalg.eigvalsh((t + t.T) / 2 if sym else t @ t.T).abs().max().item() ** (1.0 if sym else 0.5)

    def lipschitz(top, a, b, c):
        t = torch.linspace(0, 1.05 * top, 513, dtype=torch.float64)
        return (a + 3 * b * t ** 2 + 5 * c * t ** 4).abs().max().item()

    eye = torch.eye(s, dtype=torch.float64, device=X.device)
    err = (0.0 if exact_input and passes == 1 else u * fro(X)) + 2.0 ** -23 * fro(X)      # the scale that is left is rounded too
    # steps between two roundings of X: two in front, and two at the end of five or more, where the matrix is twice as long as wide;
    # one by one elsewhere, and where a small matrix has two-term operands
    singles = l < 2 * s or (passes == 3 and s <= 512)
    # (`pairs`: whether the factors of the first two steps, and of the last two, fit the images together)
    k, pair_last = 0, pairs[1] and len(schedule) >= 5 and not singles
    while k < len(schedule):
        steps = schedule[k:k + (2 if (k == 0 and pairs[0] and not singles) or (pair_last and len(schedule) - k == 2) else 1)]
        A = X @ X.T
        dA = u * fro(A) + gamma(l) * fro(X) ** 2 + 2.0 ** -22 * fro(A)
        P = dP = None
        for j, (a, b, c) in enumerate(steps):
            Q = a * eye + b * A + c * (A @ A)
            dQ = u * fro(Q) + (abs(b) + 2 * abs(c) * two(A)) * dA + abs(c) * gamma(s) * fro(A) ** 2
            if P is None:
                P, dP = Q, dQ
            else:
                dP = u * fro(Q @ P) + dQ * two(P) + two(Q) * dP + gamma(s) * fro(Q) * fro(P)
                P = Q @ P
            if j + 1 < len(steps):
                T = Q @ A
                dT = u * fro(T) + dQ * two(A) + gamma(s) * fro(Q) * fro(A)
                dA = u * fro(Q @ T) + two(Q) * dT + dQ * two(T) + two(Q) ** 2 * dA + gamma(s) * fro(Q) * fro(T)
                A = Q @ T
        Y = X
        for a, b, c in steps:
            err *= lipschitz(two(Y), a, b, c)
            G = Y @ Y.T
            Y = a * Y + (b * G + c * (G @ G)) @ Y
        err += dP * two(X) + gamma(s) * fro(P) * fro(X)
        X, k = Y, k + len(steps)
        if k < len(schedule):
            err += u * fro(X)
    return err / max(fro(X), 1e-300) + HALF_STEP[x_dtype] + 2.0 ** -23


def muon(X, M, G, mu, eta, wd, scale, nesterov, schedule, eps=1e-7):
    X, M, G = X.double(), M.double(), G.double()
    M = mu * M + (1 - mu) * G
    B = mu * M + (1 - mu) * G if nesterov else M
    O = orthogonalise(B, schedule, eps)
    return (1 - eta * wd) * X - eta * scale * O, M, B, O


def adamw(X, M, V, G, t, beta1, beta2, eps, eta, wd):
    X, M, V, G = X.double(), M.double(), V.double(), G.double()
    M = beta1 * M + (1 - beta1) * G
    V = beta2 * V + (1 - beta2) * G * G
    return X - eta * (wd * X + M / (1 - beta1 ** t) / ((V / (1 - beta2 ** t)).sqrt() + eps)), M, V


def gradient(kind, m, n, seed, dtype=torch.float32, device="cuda"):
    """Noise; noise and some strong directions; singular values that fall as 1/i."""
    g = torch.Generator(device=device).manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device=device, dtype=torch.float64)  # noqa: E731
    if kind == "noise":
        G = rnd(m, n)
    elif kind == "spikes":
        k = max(1, min(64, min(m, n) // 4))
        G = rnd(m, n) / n ** 0.5 + 10 * (m ** 0.5 + n ** 0.5) / n ** 0.5 * (rnd(m, k) / m ** 0.5) @ (rnd(n, k) / n ** 0.5).T
    else:
        k = min(m, n)
        U, V = torch.linalg.qr(rnd(m, k))[0], torch.linalg.qr(rnd(n, k))[0]
        G = (U / torch.arange(1, k + 1, device=device, dtype=torch.float64)) @ V.T
    return G.to(dtype)


def rel(a, b):
    a, b = a.double(), b.double()
    return ((a - b).norm() / b.norm().clamp_min(1e-300)).item()
