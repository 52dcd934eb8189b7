"""Linear attention with a decay in 64 bits, token by token from its definition, with what bounds the
error of FP32 sums; and the norm's definition."""
import numpy as np
import torch

D = 128
U = 2.0 ** -24         # half a step of FP32
BF16 = 2.0 ** -8       # half a step of BF16
LEAST = -200.0


def linear(q, k, v, g, start, scale):
    """q [n][h_q][128], k, v [n][h][128], g [n][h], start [h][128][128] (float64 arrays) -> outputs, last state, and
    the same of absolute values, which the errors are relative to."""
    n, h_q, _ = q.shape
    h = k.shape[1]
    grp = h_q // h
    s, sa = start.copy(), np.abs(start)
    out, outa = np.zeros(q.shape), np.zeros(q.shape)
    for t in range(n):
        a = np.exp(np.clip(g[t], LEAST, 0.0))[:, None, None]
        kv = k[t][:, :, None] * v[t][:, None, :]
        s, sa = a * s + kv, a * sa + np.abs(kv)
        qt = q[t].reshape(h, grp, D)
        out[t] = (scale * (qt @ s)).reshape(h_q, D)
        outa[t] = (abs(scale) * (np.abs(qt) @ sa)).reshape(h_q, D)
    return out, s, outa, sa


def chunk_error(n, g):
    """Relative to the absolute values, per state element: every chunk of 64 adds up to 64 products (64 U) and
    brings what was before it once through a decay and a sum (3 U, with a decay's own error: one step of exp2
    and its argument, at most 104 before the factor is 0 in FP32, to half a step); three BF16 parts lose 1 U.
    A segment joins its states by one more decay and sum, no more than a chunk."""
    chunks = -(-n // 64) + 1
    reach = 0.0
    if n:
        reach = min(104.0, max(float(-np.clip(g[c:c + 64], LEAST, 0.0).sum(0).min()) for c in range(0, n, 64)))
    return (66 + chunks * (5 + 2 * reach)) * U


def check(got, ref, absolute, bound, rounding, what):
    err = np.abs(got - ref)
    limit = bound * absolute + rounding * np.abs(ref) + 1e-30
    worst = np.max(err - limit, initial=-1.0)
    assert worst <= 0 and np.isfinite(got).all(), f"{what}: {worst} over at {np.argmax(err - limit)}, largest error {err.max()}"


def check_out(got, ref, absolute, n, g, what):
    """The state's error, its and the scores' two BF16 parts (2^-16 each, and of each product again), sums of 128
    channels and 64 keys, a decay on either side; then BF16."""
    check(got, ref, absolute, chunk_error(n, g) + 3 * 2.0 ** -16 + (128 + 64 + 8) * U, BF16 * (1 + 2.0 ** -6), what)


def check_state(got, ref, absolute, n, g, what):
    check(got, ref, absolute, chunk_error(n, g), U, what)


def np64(t):
    return t.detach().cpu().double().numpy()


def norm(x, weight, eps, residual=None, group=None):
    """float64: r, y, and with a group codes (torch float8) and scales."""
    x = x.double()
    r = (x + residual.double()).to(torch.bfloat16).double() if residual is not None else x
    rstd = 1 / torch.sqrt((r * r).mean(-1, keepdim=True) + eps)
    w = r * weight.double() if weight is not None else r
    if group is None:
        return r, w * rstd, None, None
    n, width = w.shape
    group = group or width
    codes, scales = torch.empty(n, width, dtype=torch.float8_e4m3fn), torch.empty(n, -(-width // group), dtype=torch.float64)
    for i, c in enumerate(range(0, width, group)):
        part = w[:, c:c + group]
        m = part.abs().amax(-1, keepdim=True)
        codes[:, c:c + group] = torch.where(m > 0, 448 * part / torch.where(m > 0, m, 1.0), 0.0).float().to(torch.float8_e4m3fn)
        scales[:, i] = torch.where(m > 0, m * rstd / 448, 1.0)[:, 0]
    return r, w * rstd, codes, scales
