"""The numbers that the products of orthogonalised momentum are made of, restated: fp16 operands (one or two for a
number) of which the diagonals are taken out, with all sums in 64 bits.  So its error is that of the operands alone, and
`lost` says what each of them is good for: what would be left without it."""
import numpy as np

from tests.muon_reference import COEFFICIENTS

X_SCALE, B_SCALE = 2.0 ** 15, 2.0 ** 14
ONE, TWO = ("diagonals", "rest of X"), ("X X", "A", "A A", "B", "B X", "rest of X")   # what `lost` may name


def two(v, scale):
    """The two fp16 numbers of each, as the numbers they stand for."""
    y = (v * scale).astype(np.float32)
    hi = y.astype(np.float16)
    return hi.astype(np.float64) / scale, (y - hi.astype(np.float32)).astype(np.float16).astype(np.float64) / scale


def orthogonalise(u, numbers, lost=None, eps=1e-7):
    """X after five steps, `numbers` (1 or 2) of fp16 an operand of a product."""
    a, b, c = COEFFICIENTS
    tall = u.shape[0] > u.shape[1]
    u = u.T if tall else u

    def product(p, q, first_only=False):
        if numbers == 1 or first_only:
            return p[0] @ q[0]
        return p[0] @ q[0] + p[0] @ q[1] + p[1] @ q[0]

    def operand(v, scale, name):
        hi, lo = two(v, scale)
        return hi, lo * (numbers == 2 and lost != name)

    def stored(v):
        hi, lo = two(v, X_SCALE)
        return hi, lo * (lost != "rest of X")

    x = stored(u / (np.linalg.norm(u) + eps))
    for k in range(5):
        gram = product(x, (x[0].T, x[1].T), lost == "X X")
        if lost == "diagonals":
            A = operand(gram, X_SCALE, "A")
            y = a * (x[0] + x[1]) + product(operand(b * (A[0] + A[1]) + c * product(A, A), B_SCALE, "B"), x)
        else:
            d = np.diag(gram).copy()
            np.fill_diagonal(gram, 0.0)
            A = operand(gram, X_SCALE, "A")
            square = product(A, A, lost == "A A")
            B = b * (A[0] + A[1]) + c * (square + (d[:, None] + d) * (A[0] + A[1]))
            D = a + b * d + c * (np.diag(square) + d * d)
            np.fill_diagonal(B, 0.0)
            B = operand(B, B_SCALE, "B")
            y = D[:, None] * (x[0] + x[1]) + (B[0] @ x[0] + B[1] @ x[0] if lost == "B X" else product(B, x))
        if k < 4:
            x = stored(y)
    return y.T if tall else y
