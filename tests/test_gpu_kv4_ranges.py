"""The 4-bit cache at the ends of its ranges.  Definitions and tolerances: tests/kv4_ref.py."""
import math

import pytest
import torch

from tests import kv4_ref as R
from tests.test_gpu_kv4 import (D, PAGE, attn_case, check_prefill, check_rows, check_stats, check_write, cumulative, i32, mp,  # noqa: F401
                                slots_of)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ weights over many keys and partitions
@pytest.mark.parametrize("part", [None, 128, 640])
@pytest.mark.parametrize("h_q,h_kv,q_tokens,window,sinks", [(8, 2, 1, 0, 0), (10, 2, 4, 0, 0), (12, 3, 1, 3000, 70), (80, 1, 1, 0, 0)])
def test_weights_of_long_contexts(mp, h_q, h_kv, q_tokens, window, sinks, part):
    """More than 64 partitions, partitions of several tiles, more keys than one workgroup adds, more rows than
    are held at a time; by the plan's own cut and by others."""
    kv = [9001, 1030, 130]
    print(f"weights of {kv}, heads {h_q}:{h_kv}, rows {q_tokens}, window {window}, parts {part}", flush=True)
    rows, cache, stats, q = attn_case(mp, kv, h_q, h_kv, [q_tokens] * len(kv), 23, weights=True)
    before = cache.weights.clone()
    longest = 12000
    plan = mp.kv4_decode_plan([longest] * len(kv), h_q, h_kv, q_tokens, window, sinks, weights=True)
    if part:
        plan.partition_tokens, plan.max_partitions = part, -(-longest // part)
        r = len(kv) * q_tokens * h_q
        states = (r * plan.max_partitions * 130 * 4 + 255) // 256 * 256
        plan.workspace = torch.empty(states + r * plan.max_partitions * part * 4, dtype=torch.uint8, device="cuda")
    plan.workspace.fill_(255)
    out = torch.full_like(q, math.nan)
    mp.kv4_decode(q, cache, stats, i32(kv), rows.cuda(), out, plan, window=window, sinks=sinks)
    torch.cuda.synchronize()
    touched = torch.zeros_like(before, dtype=torch.bool)
    for b, n in enumerate(kv):
        x = slice(b * q_tokens, (b + 1) * q_tokens)
        toks = R.Tokens(cache, rows[b].cuda(), n)
        want, tol, share, stol = R.attention(q[x], toks, stats.k_tscale[b], stats.v_tscale[b], n - q_tokens, window, sinks)
        check_rows(out[x], want, tol, f"sequence {b}")
        i = torch.arange(n, device="cuda")
        pg, o = rows[b].cuda()[i // PAGE].long(), i % PAGE
        w0 = before[pg, :, o].double()
        off = (toks.weights.double() - (w0 + share)).abs() > stol + 2.0 ** -24 * (w0 + share)
        assert not off.any(), f"sequence {b}: {int(off.sum())} weights off, the first at {off.nonzero()[0].tolist()}"
        touched[pg, :, o] = True
    assert torch.equal(cache.weights[~touched].nan_to_num(5.0), before[~touched].nan_to_num(5.0))


# ------------------------------------------------------------------ statistics of many prompts together
@pytest.mark.parametrize("lens,h_kv", [([(i * 37) % 97 + 500 for i in range(60)] + [0, 1, 1500], 2), ([4100] * 8 + [700], 1)])
def test_write_of_many_prompts_together(mp, lens, h_kv):
    """Partials of 512 tokens that the write pass itself finishes."""
    T, B = sum(lens), len(lens)
    assert T >= 32768 and -(-max(lens) // 512) <= 32
    print(f"write {B} prompts, {T} tokens x {h_kv}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(h_kv)
    rows = R.page_rows(lens, sum(-(-n // PAGE) for n in lens) + 2, 3)
    k = (torch.randn(T, h_kv, D, generator=gen, device="cuda") + 2 * torch.randn(1, h_kv, D, generator=gen, device="cuda")).bfloat16()
    v = torch.randn(T, h_kv, D, generator=gen, device="cuda").bfloat16()
    cache, stats, cu = mp.PagedCache4(int(rows.max()) + 1, h_kv), mp.SeqStats4(B, h_kv), cumulative(lens)
    before = [x.clone() for x in (stats.k_mean, stats.k_tscale)]
    ws = torch.full((mp.kv4_write_workspace_size(B, T, h_kv),), 255, dtype=torch.uint8, device="cuda")
    mp.kv4_write(k, v, cu, slots_of(rows, [0] * B, lens), cache, stats, mp.SMOOTH | mp.COMPUTE_STATS, max(lens), workspace=ws)
    torch.cuda.synchronize()
    check_stats(stats, before, lens, k, v, True, cu)
    check_write(mp, cache, rows, [0] * B, lens, k, v, stats, True, cu)


# ------------------------------------------------------------------ scores of any size
def both(mp, q, cache, stats, kv, rows, weights=False):
    """The call's rows by decode and by prefill, in one pass and in halves that split the keys."""
    n, (r, h_q) = kv[0], q.shape[:2]
    dec, pre, cut = (torch.full_like(q, math.nan) for _ in range(3))
    args = (cumulative([r]), i32([n - r]), i32(kv), rows.cuda())
    mp.kv4_decode(q, cache, stats, i32(kv), rows.cuda(), dec, mp.kv4_decode_plan(kv, h_q, cache.h_kv, r, weights=weights))
    mp.kv4_prefill(q, cache, stats, *args, pre)
    mp.kv4_prefill(q, cache, stats, *args, cut, mp.kv4_prefill_plan([r], kv, h_q, cache.h_kv))
    torch.cuda.synchronize()
    return {"decode": dec, "prefill": pre, "prefill by plan": cut}


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("q_exp,t_exp", [(10, 0), (16, 0), (20, 0), (30, 3), (60, -3), (100, 0), (60, 63), (110, 63), (-50, 63), (118, -63)])
def test_one_key_takes_all(mp, q_exp, t_exp, weights):
    """Queries so large that the best key's weight is 1 and every other one's 0: its V comes out, exactly (a V
    value has six bits, and 1 times it divided by 1 is off by a few 2^-24 before the rounding to bf16)."""
    print(f"one key takes all: q about 2^{q_exp}, K in units of 2^{t_exp}, weights {weights}", flush=True)
    kv, h_q, h_kv, r = [700], 4, 2, 6
    rows, cache, stats, q = attn_case(mp, kv, h_q, h_kv, [r], 61, weights=weights)
    stats.k_tscale.fill_(2.0 ** t_exp)
    q = (q.double() * 2.0 ** q_exp).bfloat16()
    toks = R.Tokens(cache, rows[0].cuda(), kv[0])
    k, v, w0 = toks.k() * 2.0 ** t_exp, toks.v() * stats.v_tscale[0].double()[None, :, None], toks.weights
    want, share = torch.empty(r, h_q, D, dtype=torch.float64, device="cuda"), torch.zeros(kv[0], h_kv, dtype=torch.float64, device="cuda")
    for i in range(r):
        for h in range(h_q):
            n, hk = kv[0] - r + 1 + i, h // (h_q // h_kv)
            s = (k[:n, hk] @ q[i, h].double()) / math.sqrt(D)
            size = (k[:n, hk].abs() @ q[i, h].double().abs()).max() / math.sqrt(D)
            top = s.topk(2)
            # the distance outweighs what FP32 sums of 128 products may be off by, and any other key's weight is below
            # 2^-40 of the best one's, which its FP16 value does not hold
            assert top.values[0] - top.values[1] > 2 * 136 * 2.0 ** -24 * size + 40
            want[i, h] = v[top.indices[0], hk]
            share[top.indices[0], hk] += 1
    for name, out in both(mp, q, cache, stats, kv, rows, weights).items():
        assert torch.equal(out.double(), want), f"{name}: {int((out.double() != want).sum())} values off, {int(out.isnan().sum())} NaN"
    if weights:
        got = R.Tokens(cache, rows[0].cuda(), kv[0]).weights.double()
        # a share is 2^15 / L times 2^0: two roundings, then the additions
        assert ((got - (w0.double() + share)).abs() <= 2.0 ** -20 * (w0.double() + share)).all()


# ------------------------------------------------------------------ small queries, large keys
@pytest.mark.parametrize("q_exp", [-70, -76, -78, -79, -90])
def test_small_queries_against_large_keys(mp, q_exp):
    """Queries far below bf16's middle against keys far above it: ordinary scores, to the ordinary tolerance.  Every
    second key is 0 with V = 1, the others 2688 * 2^63 in all channels with V = -1; every query value is
    129 / 128 * 2^q_exp, so that a loss of bits would not average out."""
    print(f"q about 2^{q_exp} against keys in units of 2^63", flush=True)
    kv, h_q, h_kv, r = [500], 4, 2, 5
    rows, cache, stats, q = attn_case(mp, kv, h_q, h_kv, [r], 67)
    cache.k_codes[:, :, 0::2], cache.k_codes[:, :, 1::2] = 0x00, 0x77
    vc = cache.v_codes.view(-1, h_kv, 16, 16, 4, 4)
    vc[:, :, :, :, 0::2], vc[:, :, :, :, 1::2] = 0x22, 0xAA
    cache.k_scales.fill_(0x7E)
    cache.v_scales.fill_(0x38)
    stats.k_tscale.fill_(2.0 ** 63)
    q.fill_(129 / 128 * 2.0 ** q_exp)
    want, tol, _, _ = R.attention(q, R.Tokens(cache, rows[0].cuda(), kv[0]), stats.k_tscale[0], stats.v_tscale[0], kv[0] - r, 0, 0)
    for name, out in both(mp, q, cache, stats, kv, rows).items():
        assert not out.isnan().any(), name
        check_rows(out, want, tol, name)


# ------------------------------------------------------------------ plans of other lengths
@pytest.mark.parametrize("new,ctx", [([70], [500]), ([40], [0]), ([70], [100])])
def test_prefill_by_a_plan_for_longer_prompts(mp, new, ctx):
    """Parts of a cut block that have no tiles left add nothing to it."""
    print(f"prefill {new} behind {ctx} by a plan for 70 behind 30000", flush=True)
    h_q, h_kv = 8, 2
    kv = [a + b for a, b in zip(new, ctx)]
    rows, cache, stats, q = attn_case(mp, kv, h_q, h_kv, new, 43)
    q = torch.cat([q, torch.zeros(70 - new[0], h_q, D, device="cuda").bfloat16()])
    plan = mp.kv4_prefill_plan([70], [30000], h_q, h_kv)
    assert plan.n_merges > 0
    plan.workspace.fill_(255)
    out = torch.full_like(q, 7.0)
    mp.kv4_prefill(q, cache, stats, cumulative(new), i32(ctx), i32(kv), rows.cuda(), out, plan)
    torch.cuda.synchronize()
    check_prefill(q[:new[0]], out[:new[0]], rows, cache, stats, new, ctx, 0, 0)
    assert (out[new[0]:] == 7).all()


# ------------------------------------------------------------------ padded batches
def test_debug_library_takes_padded_batches(mp, monkeypatch):
    """Rows behind the last sequence are neither read nor written, whatever they and their slots hold."""
    print("debug library: padded batches", flush=True)
    monkeypatch.setattr(mp, "lib", mp.debug_lib)
    lens, h_q, h_kv, pad = [70, 5], 8, 2, 9
    T, B = sum(lens), len(lens)
    rows = R.page_rows(lens, 6, 2)
    val = lambda h: torch.randn(T + pad, h, D, device="cuda").bfloat16()
    q, k, v = val(h_q), val(h_kv), val(h_kv)
    for x in (q, k, v):
        x[T:] = math.nan
    cu, slots = cumulative(lens), torch.cat([slots_of(rows, [0] * B, lens), torch.full((pad,), 5, dtype=torch.int64, device="cuda")])
    cache, stats = mp.PagedCache4(6, h_kv), mp.SeqStats4(B, h_kv)
    ws = torch.empty(mp.kv4_write_workspace_size(B, T + pad, h_kv), dtype=torch.uint8, device="cuda")
    ko = torch.full_like(k, 7.0)
    mp.kv4_write(k, v, cu, slots, cache, stats, mp.SMOOTH | mp.COMPUTE_STATS, max(lens), workspace=ws, k_out=ko)
    out = torch.full_like(q, 7.0)
    args = (q, cache, stats, cu, i32([0] * B), i32(lens), rows.cuda(), out)
    mp.kv4_prefill(*args)
    torch.cuda.synchronize()
    check_write(mp, cache, rows, [0] * B, lens, k, v, stats, True, cu)
    check_prefill(q[:T], out[:T], rows, cache, stats, lens, [0] * B, 0, 0)
    mp.kv4_prefill(*args, mp.kv4_prefill_plan(lens, lens, h_q, h_kv))
    torch.cuda.synchronize()
    check_prefill(q[:T], out[:T], rows, cache, stats, lens, [0] * B, 0, 0)
    assert (out[T:] == 7).all() and (ko[T:] == 7).all()
    with pytest.raises(mp.MpfaError) as e:   # fewer rows than the sequences say
        mp.kv4_prefill(q[:T - 1], cache, stats, cu, i32([0] * B), i32(lens), rows.cuda(), out[:T - 1])
    assert e.value.status == mp.MPFA_ERR_DATA


# ------------------------------------------------------------------ plans used on another stream
@pytest.mark.parametrize("prefill", [False, True])
def test_plan_dropped_after_a_call_on_another_stream(mp, prefill):
    """Its memory is not handed out again before the call has ended."""
    print(f"plan dropped behind a call on another stream, prefill {prefill}", flush=True)
    kv, h_q, h_kv, r = [9000], 8, 2, 2
    rows, cache, stats, q = attn_case(mp, kv, h_q, h_kv, [r], 29)
    table, kv_len, out = rows.cuda(), i32(kv), torch.full_like(q, math.nan)
    cu, start = cumulative([r]), i32([kv[0] - r])
    plan = mp.kv4_prefill_plan([r], kv, h_q, h_kv) if prefill else mp.kv4_decode_plan(kv, h_q, h_kv, r)
    size, at = plan.workspace.numel(), {t.data_ptr() for t in (plan.workspace, plan.items) if t is not None}
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        torch.cuda._sleep(200_000_000)   # the call waits behind it
    if prefill:
        mp.kv4_prefill(q, cache, stats, cu, start, kv_len, table, out, plan, stream=other)
    else:
        mp.kv4_decode(q, cache, stats, kv_len, table, out, plan, stream=other)
    items = 0 if plan.items is None else plan.items.numel()
    del plan
    new = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(3)] + \
        [torch.empty(items, dtype=torch.int32, device="cuda") for _ in range(3 if items else 0)]
    assert not other.query(), "the other stream was to be busy still"
    assert not at & {t.data_ptr() for t in new}
    other.synchronize()
    check_prefill(q, out, rows, cache, stats, [r], [kv[0] - r], 0, 0)


# ------------------------------------------------------------------ what the interface promises
@pytest.mark.parametrize("kv,rows_n,window,sinks", [([700, 1500], 1, 100, 0), ([2000, 900], 5, 200, 70), ([1500, 1000], 40, 64, 3)])
def test_pages_before_a_window_may_hold_anything_written(mp, kv, rows_n, window, sinks):
    """Entries of pages that no row sees may name other sequences' pages: every output byte stays."""
    print(f"{kv} keys, {rows_n} rows, window {window}: entries before it replaced", flush=True)
    h_q, h_kv, n_rows = 8, 2, [rows_n] * len(kv)
    rows, cache, stats, q = attn_case(mp, kv, h_q, h_kv, n_rows, 73)
    other = rows.clone()
    for b, n in enumerate(kv):
        first = n - rows_n - window + 1   # first key of the first row's window
        for pg in range(-(-n // PAGE)):
            if pg * PAGE >= sinks and (pg + 1) * PAGE <= first:
                other[b, pg] = rows[1 - b, pg % (min(kv) // PAGE)]   # a whole page of the other sequence
    assert (other != rows).any(1).all()
    outs = []
    for table in (rows.cuda(), other.cuda()):
        dec, pre, cut = (torch.full_like(q, math.nan) for _ in range(3))
        att = dict(window=window, sinks=sinks)
        args = (q, cache, stats, cumulative(n_rows), i32([n - rows_n for n in kv]), i32(kv), table)
        mp.kv4_decode(q, cache, stats, i32(kv), table, dec, mp.kv4_decode_plan(kv, h_q, h_kv, rows_n, window, sinks), **att)
        mp.kv4_prefill(*args, pre, max_seqlen_q=rows_n, **att)
        mp.kv4_prefill(*args, cut, mp.kv4_prefill_plan(n_rows, kv, h_q, h_kv, window, sinks), **att)
        outs.append((dec, pre, cut))
    torch.cuda.synchronize()
    for a, b in zip(*outs):
        assert not a.isnan().any() and torch.equal(a, b)


def test_eviction_right_behind_a_prompt(mp):
    """The prompt's last rows decoded once more give its tokens their weights, and the prefill's outputs."""
    print("eviction behind a prompt", flush=True)
    T, n, h_q, h_kv, budget = 500, 32, 8, 2, 100
    rows = R.page_rows([T], 10, 3)
    table, kv_len, cu = rows.cuda(), i32([T]), cumulative([T])
    cache, stats = mp.PagedCache4(10, h_kv, weights=True), mp.SeqStats4(1, h_kv)
    gen = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn(T, h, D, generator=gen, device="cuda").bfloat16() for h in (h_q, h_kv, h_kv))
    ws = torch.empty(mp.kv4_write_workspace_size(1, T, h_kv), dtype=torch.uint8, device="cuda")
    mp.kv4_write(k, v, cu, slots_of(rows, [0], [T]), cache, stats, mp.SMOOTH | mp.COMPUTE_STATS, T, workspace=ws)
    out, last = torch.empty_like(q), torch.empty_like(q[-n:])
    mp.kv4_prefill(q, cache, stats, cu, i32([0]), kv_len, table, out, mp.kv4_prefill_plan([T], [T], h_q, h_kv))
    mp.kv4_decode(q[-n:], cache, stats, kv_len, table, last, mp.kv4_decode_plan([T], h_q, h_kv, n, weights=True))
    torch.cuda.synchronize()
    toks = R.Tokens(cache, table[0], T)
    want, tol, share, stol = R.attention(q[-n:], toks, stats.k_tscale[0], stats.v_tscale[0], T - n, 0, 0)
    check_rows(last, want, tol, "decode")
    check_rows(out[-n:], want, tol, "prefill")
    assert ((toks.weights.double() - share).abs() <= stol + 2.0 ** -24 * share).all()
    kept = torch.empty(1, h_kv, budget, dtype=torch.int32, device="cuda")
    mp.kv4_evict(cache, kv_len, table, table, budget, kept, kv_len, sinks=4, recent=20, in_place=True)
    torch.cuda.synchronize()
    for h in range(h_kv):
        assert kept[0, h].tolist() == R.keep(toks.weights[:, h].cpu(), budget, 4, 20)
