"""Linear attention with a decay against its definition in 64 bits: lengths, heads, decays that clear the state, strides,
states that are shared, written in place or not kept, padding, streams, graphs."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests import linear_ref as R

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module")
def mp():
    import paper_2609_33135_amd as mp
    mp.lib()
    return mp


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Case:
    """Packed sequences with random inputs; `clear`: some tokens forget what was before them."""

    def __init__(self, lens, h_q, h_kv, decay="token", src=None, dst=None, slots=None, seed=0, pad=0, clear=False, gap=0):
        gen = torch.Generator().manual_seed(seed)
        self.lens, self.h_q, self.h_kv, b = lens, h_q, h_kv, len(lens)
        self.T = sum(lens)
        t = self.T + pad

        def rows(h):   # with a gap the tokens are slices of wider rows
            x = torch.randn(t, h * D + gap, generator=gen).to(torch.bfloat16).cuda()
            return x[:, :h * D].unflatten(1, (h, D))
        self.q, self.k, self.v = rows(h_q), rows(h_kv), rows(h_kv)
        if decay == "head":
            g = -torch.rand(h_kv, generator=gen) ** 4
        else:
            g = torch.nn.functional.logsigmoid(3 + 2 * torch.randn(t, h_kv, generator=gen))
            if clear:
                hit = torch.rand(t, h_kv, generator=gen)
                g = torch.where(hit < 0.02, -torch.inf, torch.where(hit < 0.04, -1000.0, torch.where(hit < 0.06, -50.0, torch.where(hit < 0.2, 0.0, g))))
        self.g = g.cuda()
        slots = 2 * b if slots is None else slots
        self.states = torch.randn(slots, h_kv, D, D, generator=gen).cuda()
        self.src = list(range(b)) if src is None else src
        self.dst = list(range(b, 2 * b)) if dst is None else dst
        self.cu = [0] + np.cumsum(lens).tolist()
        self.out = torch.full((t, h_q, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.scale = 0.125

    def workspace(self, mp, longest=None):
        size = mp.linear_prefill_workspace_size(len(self.lens), self.q.shape[0], longest or max(self.lens), self.h_q, self.h_kv)
        return torch.empty(size, dtype=torch.uint8, device="cuda") if size else None

    def prefill(self, mp, workspace=None, longest=None, **kw):
        mp.linear_prefill(self.q, self.k, self.v, self.g, _i32(self.cu), self.states, _i32(self.src), _i32(self.dst), self.out,
                          longest or max(self.lens), workspace=self.workspace(mp, longest) if workspace is None else workspace,
                          scale=self.scale, **kw)

    def decode(self, mp, rows):
        mp.linear_decode(self.q, self.k, self.v, self.g, self.states, _i32(self.src), _i32(self.dst), self.out, q_tokens=rows, scale=self.scale)

    def check(self, run):
        before = self.states.clone()
        run()
        torch.cuda.synchronize()
        b4, now, out = R.np64(before), R.np64(self.states), R.np64(self.out)
        q, k, v = R.np64(self.q), R.np64(self.k), R.np64(self.v)
        g = R.np64(self.g.expand(self.q.shape[0], self.h_kv))
        untouched = np.ones(len(b4), bool)
        for b, n in enumerate(self.lens):
            at = slice(self.cu[b], self.cu[b] + n)
            start = b4[self.src[b]] if self.src[b] >= 0 else np.zeros((self.h_kv, D, D))
            o, s, oa, sa = R.linear(q[at], k[at], v[at], g[at], start, self.scale)
            if n:
                R.check_out(out[at], o, oa, n, g[at], f"outputs of sequence {b}")
            if self.dst[b] >= 0:
                untouched[self.dst[b]] = False
                R.check_state(now[self.dst[b]], s, sa, n, g[at], f"state of sequence {b}")
                if n == 0:
                    assert np.array_equal(now[self.dst[b]], start)
        assert np.array_equal(now[untouched], b4[untouched]), "a slot that no sequence ends in was written"
        assert (out[self.T:] == 7.0).all(), "padding was written"


HEADS = [(1, 1), (4, 4), (8, 2), (5, 1), (16, 1)]


@pytest.mark.parametrize("decay", ["head", "token"])
@pytest.mark.parametrize("h_q,h_kv", HEADS)
@pytest.mark.parametrize("lens", [[1], [63], [64], [65], [200], [1, 63, 0, 64, 65, 129, 2, 300]], ids=str)
def test_prefill(mp, lens, h_q, h_kv, decay):
    c = Case(lens, h_q, h_kv, decay, seed=len(lens) * 100 + lens[0])
    c.check(lambda: c.prefill(mp))


@pytest.mark.parametrize("lens,h_q,h_kv", [([2500, 300], 16, 16), ([1700], 32, 32), ([129] * 40, 16, 16), ([33] * 300, 2, 2), ([700, 1] * 3, 40, 8),
                                           ([5000, 70, 1], 1, 1), ([2600], 2, 2), ([1100], 4, 4), ([4200], 12, 4), ([70, 1, 200] * 30, 2, 2), ([66] * 65, 4, 1), ([66] * 64, 4, 1), ([0, 500, 0] * 3, 10, 2),
                                           ([90, 7], 256, 1)], ids=lambda x: str(x)[:24])
def test_prefill_longer_segments(mp, lens, h_q, h_kv):
    """Segments of several chunks, sequences that lie in one, and such whose segments are joined in several turns; few
    sequences, whose segments are numbered without gaps, and many."""
    c = Case(lens, h_q, h_kv, seed=3)
    c.check(lambda: c.prefill(mp))


@pytest.mark.parametrize("h_q,h_kv,batch,rows", [(1, 1, 1, 1), (4, 4, 3, 1), (8, 2, 5, 2), (24, 1, 2, 3), (16, 1, 7, 8), (40, 8, 33, 1), (256, 256, 2, 1),
                                                 (256, 1, 1, 2), (32, 32, 130, 1), (9, 3, 2, 70), (2, 2, 3, 23), (34, 2, 2, 5)])
@pytest.mark.parametrize("decay", ["head", "token"])
def test_decode(mp, h_q, h_kv, batch, rows, decay):
    c = Case([rows] * batch, h_q, h_kv, decay, seed=rows)
    c.check(lambda: c.decode(mp, rows))


@pytest.mark.parametrize("lens", [[300], [1, 70, 130]], ids=str)
def test_tokens_that_clear_the_state(mp, lens):
    """-inf, -1000, -50 and 0 among the log decays: no NaN, nothing of what was before."""
    c = Case(lens, 4, 4, clear=True, seed=11)
    c.check(lambda: c.prefill(mp))
    c = Case([9] * 4, 4, 2, clear=True, seed=12)
    c.check(lambda: c.decode(mp, 9))


def test_every_token_clears(mp):
    c = Case([150], 2, 2, seed=1)
    c.g.fill_(-torch.inf)
    c.check(lambda: c.prefill(mp))


def test_no_decay(mp):
    c = Case([500], 2, 2, "head", seed=1)
    c.g.zero_()
    c.check(lambda: c.prefill(mp))


@pytest.mark.parametrize("kind", ["prefill", "decode"])
def test_values_above_zero_count_as_zero(mp, kind):
    c = Case([8] * 3, 2, 2, seed=2)
    c.g = torch.where(c.g < -0.1, 0.5, c.g)
    c.check(lambda: c.prefill(mp) if kind == "prefill" else c.decode(mp, 8))


@pytest.mark.parametrize("kind", ["prefill", "decode"])
def test_slots(mp, kind):
    """Two sequences from one slot, one in place, one from zeros, one whose state is not kept, one that reads none and keeps none."""
    lens = [200] * 6 if kind == "prefill" else [3] * 6
    c = Case(lens, 4, 2, src=[4, 4, 6, -1, 7, -1], dst=[0, 1, 6, 3, -1, -1], slots=9, seed=5)
    c.check(lambda: c.prefill(mp) if kind == "prefill" else c.decode(mp, 3))


def test_in_place_many_segments(mp):
    """The last segment's workgroup writes the slot that the first one starts from."""
    c = Case([1500, 700], 4, 2, src=[1, 0], dst=[1, 0], slots=2, seed=6)
    c.check(lambda: c.prefill(mp))


@pytest.mark.parametrize("h_q,h_kv", [(16, 1), (40, 8)])
def test_in_place_heads_apart(mp, h_q, h_kv):
    """Workgroups that share a state start from what it was, though one of them replaces it, and whenever each of them
    gets to run: beside large products on another stream, against the same call out of place."""
    lens = [40, 0, 1, 64, 130]
    a = Case(lens, h_q, h_kv, src=[3, 1, 4, 0, 2], dst=[3, 1, 4, 0, 2], slots=5, seed=20)
    b = Case(lens, h_q, h_kv, src=[3, 1, 4, 0, 2], dst=[8, 6, 9, 5, 7], slots=10, seed=20)
    b.states[:5] = a.states
    b.prefill(mp)
    ws = a.workspace(mp).fill_(255)
    start, x, side = a.states.clone(), torch.zeros(4096, 4096, dtype=torch.bfloat16, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        a.states.copy_(start)
        a.out.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(4):
                x @ x
        a.prefill(mp, workspace=ws)
        ws.fill_(255)
        torch.cuda.synchronize()
        assert torch.equal(a.states, b.states[5:]) and torch.equal(a.out, b.out)
    a.states.copy_(start)
    a.check(lambda: a.prefill(mp))


@pytest.mark.parametrize("kind", ["prefill", "decode"])
def test_strides_and_padding(mp, kind):
    """Tokens that are slices of wider rows, decays of a wider matrix; rows behind the last sequence hold NaN and stay."""
    lens = [130, 1, 64] if kind == "prefill" else [2, 2, 2]
    c = Case(lens, 4, 2, pad=70 if kind == "prefill" else 0, gap=72, seed=7)
    wide = torch.full((c.q.shape[0], 5), float("nan"), device="cuda")
    wide[:, 1:3] = c.g
    c.g = wide[:, 1:3]
    for x in (c.q, c.k, c.v, c.g):
        x[c.T:] = float("nan")
    keep = c.q, c.k, c.v, c.g
    c.check(lambda: c.prefill(mp, longest=1000 if kind == "prefill" else None) if kind == "prefill" else c.decode(mp, 2))
    assert all(a is b for a, b in zip(keep, (c.q, c.k, c.v, c.g)))


def test_decay_of_one_row_for_all(mp):
    """An expanded [T][Hkv] decay is one decay per head."""
    a, b = Case([100], 4, 2, "head", seed=8), Case([100], 4, 2, "head", seed=8)
    b.g = b.g[None].expand(100, 2)
    a.prefill(mp), b.prefill(mp)
    assert torch.equal(a.out, b.out) and torch.equal(a.states, b.states)


def test_no_tokens(mp):
    """A call of empty sequences moves states alone."""
    c = Case([0, 0, 0], 4, 2, src=[4, -1, 5], dst=[0, 1, -1], slots=6, seed=9)
    c.check(lambda: c.prefill(mp, longest=1))


def test_identical_calls_give_identical_bytes(mp):
    """Also with a workspace that holds anything, and beside itself on another stream."""
    a, b = Case([900, 64, 401], 8, 2, seed=10), Case([900, 64, 401], 8, 2, seed=10)
    ws = a.workspace(mp)
    ws.fill_(255)
    side = torch.cuda.Stream()
    other = b.workspace(mp)
    side.wait_stream(torch.cuda.current_stream())
    a.prefill(mp, workspace=ws)
    with torch.cuda.stream(side):
        b.prefill(mp, workspace=other)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(a.out, b.out) and torch.equal(a.states, b.states)


def test_prompt_then_steps_equal_one_prompt(mp):
    """A prompt in two calls and decode steps behind it, in place, against the whole in one call."""
    n, h_q, h_kv = 333, 8, 2
    whole = Case([n], h_q, h_kv, src=[-1], dst=[0], slots=1, seed=13)
    whole.check(lambda: whole.prefill(mp))
    states, outs, scale = torch.empty_like(whole.states), [], whole.scale
    src, at = [-1], 0
    for m in [200, 120] + [1] * 7 + [3, 3]:
        part = lambda x: x[at:at + m]   # noqa: E731
        out = torch.empty_like(part(whole.out))
        args = part(whole.q), part(whole.k), part(whole.v), part(whole.g)
        if m > 3:
            size = mp.linear_prefill_workspace_size(1, m, m, h_q, h_kv)
            mp.linear_prefill(*args, _i32([0, m]), states, _i32(src), _i32([0]), out, m, scale=scale,
                              workspace=torch.empty(size, dtype=torch.uint8, device="cuda") if size else None)
        else:
            mp.linear_decode(*args, states, _i32(src), _i32([0]), out, q_tokens=m, scale=scale)
        outs.append(out)
        src, at = [0], at + m
    assert at == n
    q, k, v, g = (R.np64(x) for x in (whole.q, whole.k, whole.v, whole.g))
    o, s, oa, sa = R.linear(q, k, v, g, np.zeros((h_kv, D, D)), scale)
    R.check_out(R.np64(torch.cat(outs)), o, oa, 64 * 13 + n, g, "outputs")   # every call counts as a chunk more
    R.check_state(R.np64(states[0]), s, sa, 64 * 13 + n, g, "state")


def test_default_scale(mp):
    a, b = Case([70], 2, 1, seed=14), Case([70], 2, 1, seed=14)
    a.scale, b.scale = None, 128 ** -0.5
    a.prefill(mp), b.prefill(mp)
    assert torch.equal(a.out, b.out)


def test_far_offsets(mp):
    """A state slot and tokens more than 2^31 elements into their tensors."""
    if torch.cuda.get_device_properties(0).total_memory < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    slots = (1 << 31) // (D * D) + 5
    c = Case([70, 70], 1, 1, src=[0, 1], dst=[2, 3], slots=4, seed=15)
    ref_out, ref_states = c.out.clone(), c.states
    c.prefill(mp)
    states = torch.empty(slots, 1, D, D, device="cuda")
    far = [slots - 4 + i for i in range(4)]
    rows = 140
    wide = torch.empty(rows, 1 << 24, dtype=torch.bfloat16, device="cuda")   # 2^24 elements between tokens
    out = torch.empty_like(ref_out)
    lay = lambda x, n: wide[:, n * D:(n + 1) * D].unflatten(1, (1, D)).copy_(x)   # noqa: E731
    q, k, v = lay(c.q, 0), lay(c.k, 1), lay(c.v, 2)
    states[far[0]], states[far[1]] = ref_states[0], ref_states[1]
    mp.linear_prefill(q, k, v, c.g, _i32(c.cu), states, _i32(far[:2]), _i32(far[2:]), out, 70, workspace=c.workspace(mp), scale=c.scale)
    assert torch.equal(out, c.out) and torch.equal(states[far[2]], ref_states[2]) and torch.equal(states[far[3]], ref_states[3])
    a, b = torch.empty_like(out), torch.empty_like(out)
    mp.linear_decode(q, k, v, c.g, states, _i32(far[:2]), _i32(far[2:]), a, q_tokens=70, scale=c.scale)
    mp.linear_decode(c.q, c.k, c.v, c.g, ref_states, _i32([0, 1]), _i32([2, 3]), b, q_tokens=70, scale=c.scale)
    assert torch.equal(a, b) and torch.equal(states[far[3]], ref_states[3])


def test_widest_strides(mp):
    """Tokens as far apart as a call may have them: more than 64 of them lie more than 2^32 bytes apart."""
    if torch.cuda.get_device_properties(0).total_memory < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    h, lens = 128, [100, 50]
    c = Case(lens, h, h, seed=21)
    out, states = torch.empty_like(c.out), c.states.clone()
    c.prefill(mp)
    wide = torch.empty(sum(lens), (1 << 25) - 8, dtype=torch.bfloat16, device="cuda")
    lay = lambda x, n: wide[:, n * h * D:(n + 1) * h * D].unflatten(1, (h, D)).copy_(x)   # noqa: E731
    mp.linear_prefill(lay(c.q, 0), lay(c.k, 1), lay(c.v, 2), c.g, _i32(c.cu), states, _i32(c.src), _i32(c.dst), out, 100,
                      workspace=c.workspace(mp), scale=c.scale)
    assert torch.equal(out, c.out) and torch.equal(states, c.states)


def test_graph(mp):
    """A captured prompt and two decode steps in place, replayed with eager work and synchronisations between; lengths and
    slots are read at replay."""
    h_q, h_kv = 4, 2
    c = Case([300, 150], h_q, h_kv, src=[-1, 2], dst=[0, 1], slots=4, seed=16, pad=30)
    d = Case([1, 1], h_q, h_kv, src=[0, 1], dst=[0, 1], slots=1, seed=17)
    cu, src, dst = _i32(c.cu), _i32(c.src), _i32(c.dst)
    at, ws = _i32([0, 1]), c.workspace(mp, 330)

    def step(states, out, step_out):
        mp.linear_prefill(c.q, c.k, c.v, c.g, cu, states, src, dst, out, 330, workspace=ws, scale=c.scale)
        for _ in range(2):
            mp.linear_decode(d.q, d.k, d.v, d.g, states, at, at, step_out, scale=d.scale)
    states, out, step_out = c.states.clone(), torch.zeros_like(c.out), torch.zeros_like(d.out)
    step(c.states.clone(), torch.zeros_like(out), torch.zeros_like(step_out))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(states, out, step_out)
    for lens in ([300, 150], [300, 150], [1, 330], [0, 64], [300, 150]):
        cu.copy_(_i32([0, lens[0], sum(lens)]))
        want = c.states.clone(), torch.full_like(out, 3.0), torch.zeros_like(step_out)
        ws.fill_(255)
        step(*want)
        torch.cuda.synchronize()
        ws.fill_(255)
        states.copy_(c.states)
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((states, out, step_out), want):
            assert torch.equal(got, w), lens


def test_debug_library(mp):
    """The twin library takes what is right, with the same bytes, and names what is wrong before it launches anything."""
    good = Case([130, 64, 0], 4, 2, src=[3, 3, -1], dst=[0, 1, 2], slots=4, seed=18, pad=3)
    want = Case([130, 64, 0], 4, 2, src=[3, 3, -1], dst=[0, 1, 2], slots=4, seed=18, pad=3)
    want.prefill(mp)
    L = mp.debug_lib()

    def call(c, decode=False, longest=130, **kw):
        cu, src, dst, ws = _i32(kw.get("cu", c.cu)), _i32(kw.get("src", c.src)), _i32(kw.get("dst", c.dst)), c.workspace(mp)
        _, a = mp._linear_args("test", c.q, c.k, c.v, c.g, c.states, src, dst, c.out, len(c.lens), longest, 2 if decode else 0, cu.data_ptr(), c.scale)
        if decode:
            return L.mpfa_linear_decode(C.byref(a), None)
        return L.mpfa_linear_prefill(C.byref(a), mp._ptr(ws), 0 if ws is None else ws.numel(), None)
    assert call(good) == 0
    torch.cuda.synchronize()
    assert torch.equal(good.out, want.out) and torch.equal(good.states, want.states)
    for kw in (dict(cu=[0, 131, 130, 194]), dict(cu=[0, 100, 130, 198]), dict(cu=[1, 130, 194, 194]), dict(longest=129), dict(src=[4, 3, -1]),
               dict(dst=[0, 0, 2]), dict(dst=[0, 1, 4]), dict(src=[1, 3, -1])):
        assert call(good, **kw) == mp.MPFA_ERR_DATA, kw
    for n in "qkvg":
        c = Case([130, 64, 0], 4, 2, src=[3, 3, -1], dst=[0, 1, 2], slots=4, seed=18, pad=3)
        getattr(c, n)[193, -1] = float("nan")
        assert call(c) == mp.MPFA_ERR_DATA, n
    c = Case([2, 2], 4, 2, "head", seed=19)
    assert call(c, decode=True) == 0
    c.g[1] = 1e-6
    assert call(c, decode=True) == mp.MPFA_ERR_DATA
