"""The 4-bit cache's operators together, as a serving program uses them: prompts written
and prefilled, decode steps that write, attend and accumulate, an eviction, and decode
steps behind it; eagerly, on other streams, and captured into graphs."""
import math

import pytest
import torch

from tests import kv4_ref as R
from tests.test_gpu_kv4 import PAGE, D, check_rows, cumulative, i32, mp, slots_of  # noqa: F401

pytestmark = pytest.mark.gpu

H_Q, H_KV = 8, 2


class Server:
    """Sequences with room for `room` keys each; every buffer exists before the first step."""

    def __init__(self, mp, prompts, room, window=0, sinks=0, seed=1):
        self.mp, self.B, self.room, self.window, self.sinks = mp, len(prompts), room, window, sinks
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        pages = self.B * room // PAGE
        self.cache = mp.PagedCache4(pages + 1, H_KV, weights=True)
        self.rows = R.page_rows([room] * self.B, pages, seed)
        self.table = self.rows.cuda()
        R.stale(self.cache, self.rows, [0] * self.B)
        self.stats = mp.SeqStats4(self.B, H_KV)
        self.kv = list(prompts)
        self.kv_len = i32(self.kv)
        self.one = cumulative([1] * self.B)
        self.plan = mp.kv4_decode_plan([room] * self.B, H_Q, H_KV, 1, window, sinks, weights=True)
        self.slots = torch.zeros(self.B, dtype=torch.int64, device="cuda")
        self.q, self.k, self.v = self.values(self.B)
        self.out = torch.zeros(self.B, H_Q, D, dtype=torch.bfloat16, device="cuda")

    def values(self, n):
        r = lambda h: torch.randn(n, h, D, generator=self.gen, device="cuda").bfloat16()
        return r(H_Q), r(H_KV) + 2, r(H_KV)

    def prompt(self):
        mp, T = self.mp, sum(self.kv)
        q, k, v = self.values(T)
        cu = cumulative(self.kv)
        ws = torch.empty(mp.kv4_write_workspace_size(self.B, T, H_KV), dtype=torch.uint8, device="cuda")
        mp.kv4_write(k, v, cu, slots_of(self.rows, [0] * self.B, self.kv), self.cache, self.stats, mp.SMOOTH | mp.COMPUTE_STATS,
                     max(self.kv), workspace=ws)
        out = torch.empty_like(q)
        plan = mp.kv4_prefill_plan(self.kv, self.kv, H_Q, H_KV, self.window, self.sinks)
        mp.kv4_prefill(q, self.cache, self.stats, cu, i32([0] * self.B), self.kv_len, self.table, out, plan, window=self.window,
                       sinks=self.sinks)
        return q, out, k

    def next(self):
        """Inputs of the next step in the step's buffers."""
        for dst, src in zip((self.q, self.k, self.v), self.values(self.B)):
            dst.copy_(src)
        self.slots.copy_(slots_of(self.rows, self.kv, [1] * self.B))
        self.kv = [n + 1 for n in self.kv]
        self.kv_len.copy_(i32(self.kv))

    def step(self):
        self.mp.kv4_write(self.k, self.v, self.one, self.slots, self.cache, self.stats, self.mp.SMOOTH, 1)
        self.mp.kv4_decode(self.q, self.cache, self.stats, self.kv_len, self.table, self.out, self.plan, window=self.window,
                           sinks=self.sinks)

    def check(self, before):
        """The last step's outputs and weights; before: the weights of every sequence before it."""
        torch.cuda.synchronize()
        for b, n in enumerate(self.kv):
            t = R.Tokens(self.cache, self.table[b], n)
            want, tol, share, stol = R.attention(self.q[b:b + 1], t, self.stats.k_tscale[b], self.stats.v_tscale[b], n - 1, self.window,
                                                 self.sinks)
            check_rows(self.out[b:b + 1], want, tol, f"sequence {b}")
            w0 = torch.cat([before[b], torch.zeros(1, H_KV, dtype=torch.float64, device="cuda")])
            assert ((t.weights.double() - w0 - share).abs() <= stol + 2.0 ** -24 * (w0 + share)).all()

    def weights(self):
        return [R.Tokens(self.cache, self.table[b], n).weights.double() for b, n in enumerate(self.kv)]

    def evict(self, budget, kept, **kw):
        self.mp.kv4_evict(self.cache, self.kv_len, self.table, self.table, budget, kept, self.kv_len, in_place=True, **kw)


@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 5)])
def test_prompt_decode_evict_decode(mp, window, sinks):
    print(f"serving run, window {window}", flush=True)
    s = Server(mp, [300, 77, 129], 640, window, sinks)
    q, out, k = s.prompt()
    torch.cuda.synchronize()
    at = 0
    for b, n in enumerate(s.kv):
        t = R.Tokens(s.cache, s.table[b], n)
        assert (t.weights == 0).all()
        want, tol, _, _ = R.attention(q[at:at + n], t, s.stats.k_tscale[b], s.stats.v_tscale[b], 0, window, sinks)
        check_rows(out[at:at + n], want, tol, f"prompt {b}")
        # against the unquantized keys the cache is a 4-bit one: near, not equal
        kk = k[at:at + n].double() - s.stats.k_mean[b].double()
        err = t.k() * s.stats.k_tscale[b].double()[None, :, None] - kk
        assert err.norm() < 0.2 * kk.norm()
        at += n
    for _ in range(4):
        before = s.weights()
        s.next()
        s.step()
        s.check(before)
    budget = 100
    kept = torch.empty(s.B, H_KV, budget, dtype=torch.int32, device="cuda")
    old, w = [R.Tokens(s.cache, s.table[b], n).k_codes.clone() for b, n in enumerate(s.kv)], s.weights()
    s.evict(budget, kept, sinks=5, recent=20)
    torch.cuda.synchronize()
    for b, n in enumerate(s.kv):
        for h in range(H_KV):
            idx = R.keep(w[b][:, h].cpu(), budget, 5, 20)
            assert kept[b, h, :len(idx)].tolist() == idx
            assert torch.equal(R.Tokens(s.cache, s.table[b], len(idx)).k_codes[:, h], old[b][idx, h])
    s.kv = [min(n, budget) for n in s.kv]
    assert s.kv_len.tolist() == s.kv
    for _ in range(3):
        before = s.weights()
        s.next()
        s.step()
        s.check(before)


def test_step_and_eviction_in_graphs(mp):
    """A decode step and an eviction, each captured once and replayed with eager work between the
    replays; every replay is checked as the eager steps are."""
    print("serving run in graphs", flush=True)
    s = Server(mp, [400, 250], 640, seed=3)
    s.prompt()
    s.next()
    s.step()   # warm
    torch.cuda.synchronize()
    budget = 200
    kept = torch.empty(s.B, H_KV, budget, dtype=torch.int32, device="cuda")
    step, cut = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(step):
        s.step()
    with torch.cuda.graph(cut):
        s.evict(budget, kept, sinks=4, recent=8)
    for turn in range(3):
        for _ in range(3):
            before = s.weights()
            s.next()
            step.replay()
            s.check(before)
        w = s.weights()
        cut.replay()
        torch.cuda.synchronize()
        for b in range(s.B):
            for h in range(H_KV):
                idx = R.keep(w[b][:, h].cpu(), budget, 4, 8)
                assert kept[b, h, :len(idx)].tolist() == idx
        s.kv = [min(n, budget) for n in s.kv]
        assert s.kv_len.tolist() == s.kv


def test_two_servers_on_two_streams(mp):
    """Two servers whose steps overlap on streams of their own give the bytes that each gives alone."""
    print("serving runs on two streams", flush=True)

    def run(streams):
        servers = [Server(mp, [500, 100], 640, seed=5), Server(mp, [130, 600], 640, seed=6)]
        torch.cuda.synchronize()
        for s, st in zip(servers, streams):
            with torch.cuda.stream(st):
                s.prompt()
        for _ in range(5):
            for s, st in zip(servers, streams):
                with torch.cuda.stream(st):
                    s.next()
                    s.step()
        torch.cuda.synchronize()
        return [x.clone() for s in servers for x in (s.out, s.cache.weights, s.cache.k_codes, s.cache.v_codes, s.stats.k_mean)]

    alone = run([torch.cuda.current_stream()] * 2)
    apart = run([torch.cuda.Stream(), torch.cuda.Stream()])
    for a, b in zip(alone, apart):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_step_on_a_given_stream(mp):
    print("serving step on the stream argument", flush=True)
    s = Server(mp, [200], 320, seed=8)
    s.prompt()
    before = s.weights()
    s.next()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    mp.kv4_write(s.k, s.v, s.one, s.slots, s.cache, s.stats, mp.SMOOTH, 1, stream=st)
    mp.kv4_decode(s.q, s.cache, s.stats, s.kv_len, s.table, s.out, s.plan, stream=st)
    st.synchronize()
    s.check(before)


def test_debug_library_accepts_the_run_and_refuses_bad_data(mp, monkeypatch):
    """The data checks; every bad input stays inside its buffers."""
    print("debug library", flush=True)
    monkeypatch.setattr(mp, "lib", mp.debug_lib)
    s = Server(mp, [200, 70], 320, seed=9)
    s.prompt()
    before = s.weights()
    s.next()
    s.step()
    s.check(before)
    kept = torch.empty(2, H_KV, 64, dtype=torch.int32, device="cuda")

    def refused(call, *args, **kw):
        with pytest.raises(mp.MpfaError) as e:
            call(*args, **kw)
        assert e.value.status == mp.MPFA_ERR_DATA

    same = s.slots.clone()
    same[1] = same[0]
    write = lambda k=s.k, cu=s.one, slots=s.slots: mp.kv4_write(k, s.v, cu, slots, s.cache, s.stats, mp.SMOOTH, 1)
    refused(write, slots=same)
    refused(write, cu=i32([0, 2, 2]))
    refused(write, slots=s.slots + 64 * s.cache.num_pages)
    bad = s.k.clone()
    bad[1, 1, 7] = math.inf
    refused(write, k=bad)
    write(slots=torch.full_like(s.slots, -1))   # padding is fine
    dec = lambda kv=s.kv_len, table=s.table, q=s.q: mp.kv4_decode(q, s.cache, s.stats, kv, table, s.out, s.plan)
    refused(dec, kv=s.kv_len - 1000)
    refused(dec, kv=s.kv_len + 1000)
    refused(dec, table=torch.full_like(s.table, -1))
    refused(dec, table=s.table[:1].repeat(2, 1))   # weights of shared pages
    refused(dec, table=torch.full_like(s.table, s.cache.num_pages))
    bad = s.q.clone()
    bad[0, 0, 0] = math.nan
    refused(dec, q=bad)
    pre = lambda start, plan=None: mp.kv4_prefill(s.q, s.cache, s.stats, s.one, start, s.kv_len, s.table, s.out, plan)
    pre(s.kv_len - 1)
    refused(pre, s.kv_len)
    refused(pre, s.kv_len * 0 - 1)
    plan = mp.kv4_prefill_plan([1, 1], s.kv, H_Q, H_KV)
    pre(s.kv_len - 1, plan)
    for at, value in ((0, 2), (0, -1), (1, 64), (3, 9), (2, 1), (4, 0), (4, -2)):   # sequence, row, last, first, state
        items = plan.items.clone()
        items[0, at] = value
        refused(pre, s.kv_len - 1, mp.Kv4Plan(plan.what, plan.workspace, n_items=plan.n_items, n_merges=plan.n_merges,
                                              n_states=plan.n_states, half=plan.half, max_rows=1, items=items))
    evict = lambda dst, in_place: mp.kv4_evict(s.cache, s.kv_len, s.table, dst, 64, kept, s.kv_len.clone(), in_place=in_place)
    refused(evict, s.table, False)
    refused(evict, s.table.flip(1).contiguous(), True)
    refused(evict, s.table.flip(0).contiguous(), True)
    evict(s.table, True)


def test_prompt_and_prefill_in_graphs(mp):
    """A prompt's write and its prefill, by a plan and in one pass, captured once and replayed on other
    values with eager work between the replays; rows behind the last sequence stay as they were."""
    print("prompt in graphs", flush=True)
    lens, window, sinks = [1500, 3, 260], 600, 7
    T, B = sum(lens), len(lens)
    rows = R.page_rows(lens, 32, 4)
    table, slots, cu, kv = rows.cuda(), slots_of(rows, [0] * B, lens), cumulative(lens), i32(lens)
    zero = i32([0] * B)
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    q, k, v = torch.empty(T + 9, H_Q, D, **bf16), torch.empty(T, H_KV, D, **bf16), torch.empty(T, H_KV, D, **bf16)
    made = lambda: (mp.PagedCache4(32, H_KV), mp.SeqStats4(B, H_KV), torch.empty_like(q), torch.empty_like(q))
    plan = mp.kv4_prefill_plan(lens, lens, H_Q, H_KV, window, sinks)
    ws = torch.empty(mp.kv4_write_workspace_size(B, T, H_KV), dtype=torch.uint8, device="cuda")

    def run(cache, stats, by_plan, one_pass):
        mp.kv4_write(k, v, cu, slots, cache, stats, mp.SMOOTH | mp.COMPUTE_STATS, max(lens), workspace=ws)
        att = dict(window=window, sinks=sinks)
        mp.kv4_prefill(q, cache, stats, cu, zero, kv, table, by_plan, plan, **att)
        mp.kv4_prefill(q, cache, stats, cu, zero, kv, table, one_pass, max_seqlen_q=max(lens), **att)

    gen = torch.Generator(device="cuda").manual_seed(12)

    def fill():
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))

    fill()
    captured, eager = made(), made()
    run(*eager)   # warm
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(*captured)
    for _ in range(4):
        fill()
        for x in (captured, eager):
            for out in x[2:]:
                out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        run(*eager)
        torch.cuda.synchronize()
        for n in ("k_codes", "k_scales", "v_codes", "v_scales"):
            assert torch.equal(getattr(captured[0], n), getattr(eager[0], n))
        assert torch.equal(captured[1].k_mean, eager[1].k_mean)
        for a, b in zip(captured[2:], eager[2:]):
            assert torch.equal(a, b) and (a[T:] == 7).all()
    at = 0
    for b, n in enumerate(lens):
        want, tol, _, _ = R.attention(q[at:at + n], R.Tokens(eager[0], table[b], n), eager[1].k_tscale[b], eager[1].v_tscale[b], 0,
                                      window, sinks)
        for out in captured[2:]:
            check_rows(out[at:at + n], want, tol, f"prompt {b}")
        at += n


def test_plan_of_another_device_is_refused(mp):
    s = Server(mp, [200, 70], 320, seed=9)
    plan = mp.kv4_prefill_plan([1, 1], s.kv, H_Q, H_KV)
    plan.items, plan.workspace = plan.items.cpu(), None
    with pytest.raises(ValueError, match="another device"):
        mp.kv4_prefill(s.q, s.cache, s.stats, s.one, s.kv_len - 1, s.kv_len, s.table, s.out, plan)
