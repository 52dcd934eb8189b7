"""Linear attention with a decay in chunks, as the matrix cores take it, with the roundings of FP32 and BF16 where they are
asked for: what a test's bound lets through and what it does not, without a GPU."""
import numpy as np

from tests import linear_ref as R

CHUNK = 64


def bf16(x):
    """Nearest BF16, ties to even, of FP32 numbers."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
    return u.astype(np.uint32).view(np.float32)


def parts_of(x, n):
    """What is left of FP32 numbers as the sum of n BF16."""
    left, out = np.asarray(x, np.float32), np.zeros(np.shape(x))
    for _ in range(n):
        p = bf16(left)
        out += p.astype(np.float64)
        left = left - p
    return out


def linear(q, k, v, g, start, scale, sums=np.float64, parts=3):
    """Outputs and last state by chunks.  sums: the type in which a chunk's log decays are added up; parts: BF16 numbers that
    a value with its decay is the sum of (0: as it is).  Products are exact and states FP32."""
    n, h_q, _ = q.shape
    h = k.shape[1]
    grp = h_q // h
    s = start.astype(np.float32)
    out = np.zeros(q.shape)
    for c in range(0, n, CHUNK):
        at = slice(c, min(n, c + CHUNK))
        b = np.cumsum((np.clip(g[at], R.LEAST, 0.0).astype(np.float32).astype(sums)), 0, dtype=sums)
        reach = (b[:, None] - b[None]).astype(np.float64)                                   # [i][j][h]
        inside = np.tril(np.ones(reach.shape[:2], bool))[..., None]
        decay = np.where(inside, np.exp(np.where(inside, np.minimum(reach, 0.0), 0.0)), 0.0).astype(np.float32)
        tail = np.exp(np.minimum((b[-1] - b).astype(np.float64), 0.0)).astype(np.float32)   # [j][h]
        old = np.exp(b.astype(np.float64)).astype(np.float32)
        for hk in range(h):
            x = (k[at, hk] @ q[at, hk * grp:hk * grp + grp].transpose(1, 2, 0)).transpose(0, 2, 1)   # [grp][i][j]
            w = x * decay[..., hk]
            out[at, hk * grp:hk * grp + grp] = scale * (
                w @ v[at, hk] + (q[at, hk * grp:hk * grp + grp].transpose(1, 0, 2) @ s[hk].astype(np.float64)) * old[:, hk][None, :, None]
            ).transpose(1, 0, 2)
            y = v[at, hk].astype(np.float32) * tail[:, hk, None]
            y = parts_of(y, parts) if parts else y.astype(np.float64)
            s[hk] = (s[hk] * old[-1, hk]).astype(np.float64) + k[at, hk].T @ y
    return out, s.astype(np.float64)


def inputs(n, h, seed, g, start=True):
    rng = np.random.default_rng(seed)
    val = lambda heads: bf16(rng.standard_normal((n, heads, R.D))).astype(np.float64)   # noqa: E731
    return val(h), val(h), val(h), np.asarray(g(rng), np.float32).astype(np.float64), (rng.standard_normal((h, R.D, R.D)) if start else np.zeros((h, R.D, R.D))).astype(np.float32).astype(np.float64)


def cleared(rng=None):
    """Log decays of a chunk [64][1]: fifty tokens that clear the state, then fourteen that keep 97 %.  Behind the fifty the
    sum is -10000, of which FP32 keeps a step of 2^-10 = 0.001: of a decay over a token or more that is a relative error of up
    to 5e-4, where the bound is 66 + 2 (5 + 2 * 104) half steps of 2^-24, 3e-5."""
    return np.concatenate([np.full((50, 1), -np.inf), np.linspace(-0.02, -0.04, 14)[:, None]])


FROBENIUS = 10 * R.U
"""Of a state's error, relative to its norm, for tokens of independent channels whose decays sum to 1 to 2.5 over a chunk.
Every state element is a sum of some 64 products of either sign that decay by e^-1 or more a chunk.  Adding them one after
the other in any order, each sum at most a step (2 U) off and uniformly so, 2 U / sqrt(3) in the mean of squares, relative to
the sum so far, whose square grows as their number: sqrt(64 / 2) 2 / sqrt(3) = 6.6 U of the last one; older chunks' errors
decay with the state.  A decay (one step of exp2, 2 U, and half a step of its argument of at most 2.5 log2 e, 3.6 U with the
part of hi and lo that a float leaves) 4.2 U, of a token's products alike but of tokens independent; product with V and third
part 1 U each; the state's own decay a chunk and a join 3 U.  Together sqrt(6.6^2 + 4.2^2 + 2 + 9) = 8.5 U.  Two parts alone
lose, of a value between 1 and 2 times a power of two, an error in a step of 2^-7 of one of 2^-8, both uniform: 2^-16 / 3
to 2^-16 / 6 in the mean of squares, 85 to 43 U over 1.5, at least 28 U."""


def mild(n, h):
    """Log decays a token [n][h] of 1 / 64 to 2.5 / 64."""
    return lambda rng: -rng.uniform(1.0, 2.5, (n, h)) / CHUNK
