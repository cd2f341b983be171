"""Float64 oracle of the orthogonalised update: the Newton-Schulz iteration and the momentum step around
it, and a model of the iteration with fp16 operands (what a product loses by them, nothing else).  Test
infrastructure only."""
import numpy as np

QUINTIC = (3.4445, -4.7750, 2.0315)


def iterate_short(u, steps=5, eps=1e-7, part=2.0 ** -21):
    """The iteration with every product short of its value by `part` of it: what sums that drop their last places
    do when all of them drop as much."""
    u = np.asarray(u, dtype=np.float64)
    flip = u.shape[0] > u.shape[1]
    x = u.T if flip else u
    x = x / (np.sqrt((x ** 2).sum()) + eps)
    a, b, c = QUINTIC
    for _ in range(steps):
        A = (1 - part) * (x @ x.T)
        x = (1 - part) * ((a * np.eye(len(x)) + b * A + c * (1 - part) * (A @ A)) @ x)
    return x.T if flip else x


def iterate(u, steps=5, coefs=None, eps=1e-7, operand=None):
    """u [rows, cols] -> X after `steps`.  operand: rounds what enters a product (and the Gram matrix as it is
    stored); the last product is (a I + b A + c A^2) X, and what X loses as its operand is added, times a: X
    itself is carried without rounding."""
    u = np.asarray(u, dtype=np.float64)
    flip = u.shape[0] > u.shape[1]
    x = u.T if flip else u
    norm = np.sqrt((x ** 2).sum())
    x = x / (norm + eps) if norm > 0 else x * 0
    for k in range(steps):
        a, b, c = QUINTIC if coefs is None else coefs[k]
        h = x if operand is None else operand(x)
        A = h @ h.T
        if operand is not None:
            A = operand(A)
        B = a * np.eye(A.shape[0]) + b * A + c * (A @ A)
        if operand is not None:
            B = operand(B)
        x = B @ h + a * (x - h)
    return x.T if flip else x


def half_operand(x):
    """To fp16 with the library's power of two."""
    return (x * 1024.0).astype(np.float16).astype(np.float64) / 1024.0


def scaled_operand(x, scale=2.0 ** 14):
    """To fp16 with the power of two that the usual coefficients get."""
    return (x * scale).astype(np.float16).astype(np.float64) / scale


def planes(x, scale=2.0 ** 14, lo=2.0 ** 11):
    """Two fp16 planes: what stands in them, as values."""
    hi = (x * scale).astype(np.float16).astype(np.float64)
    low = ((x * scale - hi) * lo).astype(np.float16).astype(np.float64) / lo
    return hi / scale, low / scale


def iterate_planes(u, steps=5, eps=1e-7, split=planes):
    """What two planes and three products lose, and nothing else: X, A and B are split, the product of two lo
    planes is left out, everything else is exact."""
    def mul(p, q):
        return p[0] @ q[0] + (p[0] @ q[1] + p[1] @ q[0])
    u = np.asarray(u, dtype=np.float64)
    flip = u.shape[0] > u.shape[1]
    x = u.T if flip else u
    x = x / (np.sqrt((x ** 2).sum()) + eps)
    a, b, c = QUINTIC
    for _ in range(steps):
        X = split(x)
        A = split(mul(X, (X[0].T, X[1].T)))
        B = split(a * np.eye(len(x)) + b * (A[0] + A[1]) + c * mul(A, A))
        x = mul(B, X)
    return x.T if flip else x


def iterate_f32(u, steps=5, eps=1e-7):
    """The iteration in float32, products and sums."""
    u = np.asarray(u, dtype=np.float64)
    flip = u.shape[0] > u.shape[1]
    x = u.T if flip else u
    x = (x / (np.sqrt((x ** 2).sum()) + eps)).astype(np.float32)
    a, b, c = (np.float32(v) for v in QUINTIC)
    for _ in range(steps):
        A = x @ x.T
        x = a * x + (b * A + c * (A @ A)) @ x
    x = x.astype(np.float64)
    return x.T if flip else x


def step(w, m, g, lr, momentum=0.95, nesterov=True, decay=0.0, scale=1.0, grad_scale=1.0, **kw):
    """One matrix: (w, m) after the step."""
    g = np.asarray(g, dtype=np.float64) * grad_scale
    m = momentum * np.asarray(m, dtype=np.float64) + g
    u = g + momentum * m if nesterov else m
    w = np.asarray(w, dtype=np.float64)
    return w * (1 - lr * decay) - lr * scale * iterate(u, **kw), m
