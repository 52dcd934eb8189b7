"""Linear attention where segments are long and units have two of them, and where the documented precision shows: against the
definition in 64 bits, by chunks."""
import numpy as np
import pytest
import torch

from tests import linear_chunks as L
from tests import linear_ref as R
from tests.test_gpu_linear import Case, mp  # noqa: F401
from tests.test_linear_cut import LONG

pytestmark = pytest.mark.gpu
BLOCK = 256


def _reference(q, k, v, g, start, scale):
    """One sequence, [T][h][128] and [T][h] on the GPU in 64 bits: outputs, last state, and the same of absolute values."""
    n, h_q, d = q.shape
    h = k.shape[1]
    heads = lambda x: x.transpose(0, 1).contiguous()   # noqa: E731
    out = torch.empty(2, n, h_q, d, dtype=torch.float64, device="cuda")
    state = torch.stack([start, start.abs()])
    for c in range(0, n, BLOCK):
        at = slice(c, min(n, c + BLOCK))
        b = heads(g[at].clamp(R.LEAST, 0.0)).cumsum(-1)                                  # [h][m]
        m = b.shape[1]
        inside = torch.ones(m, m, dtype=torch.bool, device="cuda").tril()
        decay = torch.where(inside, torch.exp(torch.where(inside, b[:, :, None] - b[:, None, :], 0.0)), 0.0)
        for i, take in enumerate((lambda x: x, torch.abs)):
            kc, vc = take(heads(k[at])), take(heads(v[at]))
            qc = take(heads(q[at])).view(h, -1, d)                                       # heads of a KV head one after the other
            x = torch.bmm(qc, kc.transpose(1, 2).contiguous()).view(h, -1, m, m) * decay[:, None]
            o = torch.bmm(x.view(h, -1, m), vc) + torch.bmm(qc, state[i]) * torch.exp(b).repeat(1, h_q // h)[..., None]
            out[i, at] = (abs(scale) if i else scale) * o.view(h_q, m, d).transpose(0, 1)
            keep = torch.exp(b[:, -1:] - b)[..., None]
            state[i] = torch.exp(b[:, -1])[:, None, None] * state[i] + torch.bmm((kc * keep).transpose(1, 2).contiguous(), vc)
    return out[0], state[0], out[1], state[1]


def _within(got, ref, absolute, bound, rounding, what):
    over = ((got.double() - ref).abs() - bound * absolute - rounding * ref.abs()).max().item()
    assert over <= 1e-30, f"{what}: {over} over"


def _check(mp, c):   # noqa: F811
    before = c.states.clone()
    c.prefill(mp)
    torch.cuda.synchronize()
    g = c.g.expand(c.q.shape[0], c.h_kv)
    for b, n in enumerate(c.lens):
        at = slice(c.cu[b], c.cu[b] + n)
        o, s, oa, sa = _reference(*(x[at].double() for x in (c.q, c.k, c.v, g)), before[c.src[b]].double(), c.scale)
        bound = R.chunk_error(n, R.np64(g[at]))
        _within(c.out[at], o, oa, bound + 3 * 2.0 ** -16 + (128 + 64 + 8) * R.U, R.BF16 * (1 + 2.0 ** -6), f"outputs of sequence {b}")
        _within(c.states[c.dst[b]], s, sa, bound, R.U, f"state of sequence {b}")


def test_the_reference(mp):   # noqa: F811
    """Chunks against the definition token by token."""
    c = Case([300], 4, 2, seed=30)
    x = [R.np64(t) for t in (c.q, c.k, c.v, c.g, c.states[0])]
    for got, want in zip(_reference(c.q.double(), c.k.double(), c.v.double(), c.g.double(), c.states[0].double(), 0.125), R.linear(*x, 0.125)):
        assert np.abs(R.np64(got) - want).max() < 1e-9


@pytest.mark.parametrize("lens,h_q,h_kv,chunks", LONG, ids=str)
@pytest.mark.parametrize("slow", [True, False])
def test_segments_of_many_chunks(mp, lens, h_q, h_kv, chunks, slow):   # noqa: F811
    """slow: the state keeps some thousand tokens, so that what a segment leaves reaches the next ones."""
    c = Case(lens, h_q, h_kv, seed=31)
    if slow:
        gen = torch.Generator().manual_seed(32)
        c.g = (-0.002 * torch.rand(c.T, h_kv, generator=gen)).cuda()
    _check(mp, c)


@pytest.mark.parametrize("n", [64, 128])
def test_sums_of_decays_are_64_bits(mp, n):   # noqa: F811
    """Of one chunk that the outputs' workgroup takes, and of one whose state the sums' does."""
    c = Case([n], 1, 1, seed=33)
    c.g = torch.from_numpy(np.concatenate([L.cleared()] * (n // 64))).float().cuda()
    c.states[0].zero_()
    c.check(lambda: c.prefill(mp))


@pytest.mark.parametrize("n", [64, 130, 300])
def test_norm_of_the_states_error(mp, n):   # noqa: F811
    """Three parts of what stays in the state, not two."""
    q, k, v, g, start = L.inputs(n, 2, n, L.mild(n, 2), start=False)
    ref = R.linear(q, k, v, g, start, 0.1)[1]
    c = Case([n], 2, 2, src=[-1], dst=[0], slots=1, seed=34)
    for to, x in ((c.q, q), (c.k, k), (c.v, v)):
        to.copy_(torch.from_numpy(x))
    c.g = torch.from_numpy(g).float().cuda()
    c.states.fill_(float("nan"))
    c.prefill(mp)
    error = np.linalg.norm(R.np64(c.states[0]) - ref) / np.linalg.norm(ref)
    print(f"{error / R.U:.2f} half steps")
    assert error < L.FROBENIUS


@pytest.mark.parametrize("batch", [3, 65, 130])
def test_a_first_sequence_behind_other_tokens(mp, batch):   # noqa: F811
    """cu_seqlens of a batch's second half: a mistake by the header, which the debug library names, but nothing is read or
    written out of range for it, and the tokens before are left alone."""
    lens = [70, 0, 1, 130, 64] * (batch // 5) + [5] * (batch % 5)
    c = Case([500] + lens, 4, 2, src=[-1] * (batch + 1), dst=list(range(batch + 1)), seed=35)
    keep = c.states[0].clone()
    cu, src, dst = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (c.cu[1:], c.src[1:], c.dst[1:]))
    size = mp.linear_prefill_workspace_size(batch, c.T, 130, 4, 2)
    mp.linear_prefill(c.q, c.k, c.v, c.g, cu, c.states, src, dst, c.out, 130, workspace=torch.empty(size, dtype=torch.uint8, device="cuda"), scale=c.scale)
    torch.cuda.synchronize()
    assert (c.out[:500] == 7.0).all() and torch.equal(c.states[0], keep)
    before = np.zeros((2, 128, 128))
    for b, n in enumerate(lens):
        at = slice(c.cu[b + 1], c.cu[b + 1] + n)
        g = R.np64(c.g[at])
        o, s, oa, sa = R.linear(*(R.np64(x[at]) for x in (c.q, c.k, c.v)), g, before, c.scale)
        if n:
            R.check_out(R.np64(c.out[at]), o, oa, n, g, b)
        R.check_state(R.np64(c.states[b + 1]), s, sa, n, g, b)
