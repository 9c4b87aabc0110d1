"""A call for each kernel instance of the 4-bit products, and measures of their
errors that are tight enough to see a lost part of x."""

import numpy as np
import torch

from oracle import gated

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24

# kernel, row tiles, rows of x, split -> (N, R, widths D): one block of 128 columns and several,
# an odd and an even number of them, whole and cut, on 256 compute units
FORMS = {
    ("dot", 1, 1, 16): (1, 300, (77, 1030, 2304)),
    ("dot", 2, 1, 8): (1, 8200, (200, 1152)),
    ("dot", 4, 1, 8): (1, 16400, (130, 1025)),
    ("dot", 1, 2, 16): (2, 310, (64, 2177)),
    ("dot", 2, 2, 8): (2, 8200, (127, 1152)),
    ("rows", 1, 1, 16): (100, 250, (96, 2177)),
    ("rows", 2, 1, 8): (5, 8200, (130, 1151)),
    ("rows", 4, 1, 8): (16, 16400, (61, 1152)),
    ("rows", 2, 2, 8): (20, 8200, (200, 1153)),
    ("rows", 4, 2, 8): (40, 8200, (128, 1150)),
    ("tile", 4, 2, 1): (1100, 2040, (100, 300, 512)),
    ("tile", 4, 2, 2): (900, 2001, (77, 256, 385, 512, 640)),
    ("tile", 4, 4, 1): (2050, 4000, (64, 300, 513)),
}
OF_F32 = [f for f in FORMS if f != ("tile", 4, 4, 1)]
OF_BF16 = [f for f in FORMS if f[0] != "dot" or f[2] == 1]
ALL = [(f, F32) for f in OF_F32] + [(f, BF16) for f in OF_BF16]
IDS = ["%s-%d-%d-%d-%s" % (*f, "bf16" if d is BF16 else "f32") for f, d in ALL]


def levels(R, D, G, seed=0):
    r = np.random.default_rng([190500689, 12, seed, R, D, G])
    n = -(-D // G)
    q, z = r.integers(0, 16, (R, D)).astype(np.uint8), r.integers(0, 16, (R, n)).astype(np.uint8)
    return q, (r.random((R, n)) + 0.1).astype(np.float32), z


def rms_share(got, q, s, z, G, x):
    """Largest ratio, over the rows of x, of the root mean square error of fp32
    products with x of mean 0 to what roundings may make of it.

    A group's sums of q + o and of x (o = -7.5, or 0 on the vector units) grow as a
    random walk, so a partial sum is no larger, in the mean square, than S = sum
    ((|q + o| + |z + o|) s x)^2 under the root.  On the matrix units a step of 32 columns
    rounds three times to 2u, both sums: 24 roundings a group of 128, 96 u^2 S^2; on
    the vector units 128 products round to u each, 160 u^2 S^2 with the group's sum.
    The sums of groups add at most 18 u^2 S^2 (of 18 groups here): below 16 u S.
    """
    of = np.arange(q.shape[1]) // G
    a = (np.maximum(np.abs(q - 7.5), q) + np.maximum(np.abs(z - 7.5), z)[:, of]) * s.astype(np.float64)[:, of]
    S2 = (x ** 2) @ (a ** 2).T
    want, _ = gated.q4_product(q, s, z, G, x)
    return np.sqrt(np.mean((got - want) ** 2, -1) / (256 * U * U * np.mean(S2, -1))).max()


def one_column(N, R, D, seed):
    """x with one column of 24 random bits, and of either sign, in each row."""
    r = np.random.default_rng([190500689, 13, seed, N, D])
    x = np.zeros((N, D))
    at = np.concatenate([[D - 1, 0], r.integers(0, D, max(0, N - 2))])[:N]
    v = r.integers(1 << 23, 1 << 24, N) * 2.0 ** -23 * r.choice([-1.0, 1.0], N)
    x[np.arange(N), at] = v
    return x, at, v


def one_column_share(got, q, s, z, G, at, v):
    """Largest share of the tolerance of fp32 products with such x.

    A matrix instruction is off by at most 2u of its sum, and the last of the three
    parts has the largest: 2.1 u |q + o| |x|; the sum of x is exact; then two roundings
    of (q - z) x.  On the vector units z x, q x and the same two round to u each.
    """
    d = q[:, at].T.astype(np.float64), z[:, at // G].T.astype(np.float64)
    sv = s[:, at // G].T.astype(np.float64) * np.abs(v)[:, None]
    want = (d[0] - d[1]) * s[:, at // G].T.astype(np.float64) * v[:, None]
    tol = U * sv * (2.1 * np.maximum(np.abs(d[0] - 7.5), d[0]) + d[1] + 2 * np.abs(d[0] - d[1]))
    return np.max(np.abs(got - want) / (tol + 1e-30))
