"""The root-mean-square norm against its definition in 64 bits: widths, groups, residuals in place and not, strides, rows of
zeros, NaN and infinities, streams and graphs; and a layer of linear attention between two norms."""
import numpy as np
import pytest
import torch

from tests import linear_ref as R

pytestmark = pytest.mark.gpu
WIDTHS = [8, 16, 24, 64, 72, 128, 136, 256, 264, 504, 512, 520, 1000, 1024, 4096, 5120, 8200, 16384, 16392, 32768]


@pytest.fixture(scope="module")
def mp():
    import paper_2609_33135_amd as mp
    mp.lib()
    return mp


def _inputs(rows, width, seed=0, gap=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, width + gap, generator=gen) * (1 + 20 * (torch.rand(width + gap, generator=gen) < 0.01))
    return (x.to(torch.bfloat16).cuda()[:, :width], (1 + torch.randn(width, generator=gen)).to(torch.bfloat16).cuda(),
            (3 * torch.randn(rows, width, generator=gen)).to(torch.bfloat16).cuda())


def _check(mp, x, weight, residual, group, eps=1e-5, in_place=False):
    """group None: BF16 outputs.  The root's argument is a sum of `width` squares in FP32 (each of the tree's and a thread's
    16 to 32 sums at most U off, every product U), then a division, a root, a division: 48 U cover half of the sum's and
    those; a product or two more for y."""
    rows, width = x.shape
    r, y, codes, scales = R.norm(x.cpu(), None if weight is None else weight.cpu(), eps, None if residual is None else residual.cpu(), group)
    res_out = None if residual is None else residual if in_place else torch.full_like(residual, 9.0)
    if group is None:
        out = torch.full((rows, width), 9.0, dtype=torch.bfloat16, device="cuda")
        mp.rms_norm(x, weight, out, eps, residual=residual, residual_out=res_out)
        torch.cuda.synchronize()
        R.check(R.np64(out), y.numpy(), np.abs(y.numpy()), 50 * R.U, R.BF16, "y")
    else:
        out = torch.zeros(rows, width, dtype=torch.float8_e4m3fn, device="cuda")
        got = torch.full((rows, -(-width // (group or width))), 9.0, device="cuda")
        mp.rms_norm(x, weight, out, eps, residual=residual, residual_out=res_out, scales=got, group=group)
        torch.cuda.synchronize()
        assert torch.equal(out.cpu().view(torch.uint8), codes.view(torch.uint8)), "codes"
        R.check(R.np64(got), scales.numpy(), np.abs(scales.numpy()), 52 * R.U, 0.0, "scales")
    if residual is not None:
        assert np.array_equal(R.np64(res_out), r.numpy()), "residual"


@pytest.mark.parametrize("group", [None, 0, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(mp, width, group):
    for rows in (1, 37):
        x, w, res = _inputs(rows, width, seed=width)
        _check(mp, x, w, res if rows > 1 else None, group)


@pytest.mark.parametrize("width", [64, 128, 640, 20000])
@pytest.mark.parametrize("group", [None, 0, 64])
def test_strided_rows_without_weight_residual_in_place(mp, width, group):
    x, _, res = _inputs(19, width, seed=1, gap=24)
    assert not x.is_contiguous()
    _check(mp, x, None, res, group, in_place=True)


def test_many_rows(mp):
    x, w, res = _inputs(3001, 128, seed=2)
    _check(mp, x, w, res, 128)
    _check(mp, x, w, None, None)
    x, w, res = _inputs(2000, 768, seed=2)
    _check(mp, x, w, res, 0)


@pytest.mark.parametrize("width", [128, 1024])
@pytest.mark.parametrize("eps", [1e-12, 1e-6, 0.5])
def test_zeros_and_small_rows(mp, width, eps):
    """A row of zeros gives zeros and scales of 1; a group of zeros in another row too."""
    x, w, _ = _inputs(8, width, seed=3)
    x[2] = 0
    x[3, :64] = 0
    x[4] *= 2.0 ** -40
    for group in (None, 0, 64):
        _check(mp, x, w, None, group, eps=eps)


@pytest.mark.parametrize("width", [128, 1024])
def test_rows_do_not_affect_each_other(mp, width):
    """A row with a NaN, one with an infinity and one of zeros but for a NaN beside others: these are as alone."""
    x, w, _ = _inputs(12, width, seed=4)
    for group in (None, 0, 64):
        def run(x):
            out = torch.empty(12, width, dtype=torch.bfloat16 if group is None else torch.float8_e4m3fn, device="cuda")
            s = None if group is None else torch.empty(12, -(-width // (group or width)), device="cuda")
            mp.rms_norm(x, w, out, scales=s, group=group or 0)
            return out.float() if s is None else out.float() * s.repeat_interleave(group or width, 1)[:, :width]
        want = run(x)
        y = x.clone()
        y[3, 7], y[5, 9], y[9] = float("nan"), float("inf"), 0.0
        y[9, 70] = float("nan")
        got = run(y)
        others = [i for i in range(12) if i not in (3, 5, 9)]
        assert torch.equal(got[others], want[others])
        assert got[3].isnan().all() and got[9].isnan().all() and got[5].isnan().any()


def test_heads_and_shapes(mp):
    """The heads' outputs [T][H][128] are rows of 128; a view of more dimensions is rows of its last."""
    x, w, _ = _inputs(60, 128, seed=5)
    a, b = torch.empty_like(x), torch.empty(5, 3, 4, 128, dtype=torch.bfloat16, device="cuda")
    mp.rms_norm(x, w, a)
    mp.rms_norm(x.view(5, 3, 4, 128), w, b)
    assert torch.equal(a, b.view(60, 128))
    none = torch.empty(0, 128, dtype=torch.bfloat16, device="cuda")
    mp.rms_norm(none, w, none)
    with pytest.raises(mp.MpfaError):
        mp.rms_norm(x, w, a, eps=0.0)


def test_graph_and_stream(mp):
    x, w, res = _inputs(33, 640, seed=6)
    out, s = torch.zeros(33, 640, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(33, 5, device="cuda")
    total = torch.zeros_like(res)
    call = lambda: mp.rms_norm(x, w, out, residual=res, residual_out=total, scales=s, group=128)   # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mp.rms_norm(x, w, out, residual=res, residual_out=total, scales=s, group=128, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        x.mul_(1.5)
        call()
        want = out.view(torch.uint8).clone(), s.clone(), total.clone()
        out.view(torch.uint8).zero_(), s.zero_(), total.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out.view(torch.uint8), s, total), want)), i


def test_layer(mp):
    """A layer: the residual stream normalised for the projections, linear attention over a prompt and behind it a decode
    step, its heads normalised, the result added to the stream and normalised into 8 bits.  The plain torch products are
    the projections; every other step against its definition on the inputs that it got."""
    n, h_q, h_kv, width = 150, 4, 2, 256
    gen = torch.Generator(device="cuda").manual_seed(7)
    rnd = lambda *s, std=1.0: (std * torch.randn(*s, generator=gen, device="cuda")).to(torch.bfloat16)   # noqa: E731
    w_in, w_out = rnd((h_q + 2 * h_kv) * 128, width, std=width ** -0.5), rnd(width, h_q * 128, std=(h_q * 128) ** -0.5)
    w1, wh, w2 = rnd(width), rnd(128), rnd(width)
    g = torch.tensor([-0.01, -0.2], device="cuda")
    states, slot, none = torch.zeros(1, h_kv, 128, 128, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((1,), -1, dtype=torch.int32, device="cuda")
    before = np.zeros((h_kv, 128, 128))
    for t in (n, 1, 1):
        x, res = rnd(t, width), rnd(t, width)
        normed = torch.empty_like(x)
        want = R.norm(x.cpu(), w1.cpu(), 1e-6, res.cpu())[1].numpy()
        mp.rms_norm(x, w1, normed, residual=res)
        R.check(R.np64(normed), want, np.abs(want), 50 * R.U, R.BF16, "norm before")
        qkv = (normed.float() @ w_in.float().T).to(torch.bfloat16).unflatten(1, (-1, 128))
        q, k, v = qkv[:, :h_q], qkv[:, h_q:h_q + h_kv], qkv[:, h_q + h_kv:]   # slices of one projection
        out = torch.empty(t, h_q, 128, dtype=torch.bfloat16, device="cuda")
        if t > 1:
            size = mp.linear_prefill_workspace_size(1, t, t, h_q, h_kv)
            mp.linear_prefill(q, k, v, g, torch.tensor([0, t], dtype=torch.int32, device="cuda"), states, none, slot, out, t,
                              workspace=torch.empty(size, dtype=torch.uint8, device="cuda"))
        else:
            mp.linear_decode(q, k, v, g, states, slot, slot, out)
        gg = R.np64(g.expand(t, h_kv))
        o, s, oa, sa = R.linear(R.np64(q), R.np64(k), R.np64(v), gg, before, 128 ** -0.5)
        R.check_out(R.np64(out), o, oa, t, gg, "attention")
        R.check_state(R.np64(states[0]), s, sa, t, gg, "state")
        before = R.np64(states[0])
        heads = torch.empty_like(out)
        mp.rms_norm(out, wh, heads)
        want = R.norm(out.cpu().view(-1, 128), wh.cpu(), 1e-6)[1].numpy()
        R.check(R.np64(heads).reshape(-1, 128), want, np.abs(want), 50 * R.U, R.BF16, "heads")
        y = (heads.flatten(1).float() @ w_out.float().T).to(torch.bfloat16)
        _check(mp, y, w2, res, 0, eps=1e-6, in_place=True)
