"""What the entry points of the 4-bit cache refuse on the host, before any HIP call."""
import ctypes as C

import pytest

from tests.test_abi_fuzz import ALLOWED, FLAGS, I64, INTS, SET, _ints, mp  # noqa: F401
from hypothesis import given, strategies as st

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
PLANES = ("k_codes", "k_scales", "v_codes", "v_scales", "weights")


def _cache(mp, **kw):
    c = mp.Kv4Cache(num_pages=4)
    for n in PLANES:
        setattr(c, n, 0x1000)   # never dereferenced: every call here fails before a launch
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def _fill(a, names, kw):
    for n in names:
        setattr(a, n, 0x1000)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def _write(mp, **kw):
    a = mp.Kv4WriteArgs(batch=2, total_tokens=10, max_seqlen=7, h_kv=2, head_dim=128, flags=3, k_stride=256, v_stride=256,
                        cache=_cache(mp, **kw.pop("cache", {})))
    return _fill(a, ("cu_seqlens", "k", "v", "slot_mapping", "k_mean", "k_tscale", "v_tscale", "k_out", "v_out"), kw)


def _attn(mp, **kw):
    a = mp.Kv4AttnArgs(batch=2, h_q=8, h_kv=2, head_dim=128, max_pages=4, total_tokens=10, max_seqlen_q=7, q_tokens=0,
                       q_stride=1024, cache=_cache(mp, **kw.pop("cache", {})))
    return _fill(a, ("cu_seqlens_q", "q_start", "kv_len", "page_table", "q", "k_tscale", "v_tscale", "out"), kw)


def _decode(mp, **kw):
    return _attn(mp, **{**dict(q_tokens=1, partition_tokens=128, max_partitions=2), **kw})


def _evict(mp, **kw):
    a = mp.Kv4EvictArgs(batch=2, h_kv=2, max_pages=4, dst_max_pages=1, budget=64, sinks=4, recent=8,
                        cache=_cache(mp, **kw.pop("cache", {})))
    return _fill(a, ("kv_len", "page_table", "dst_page_table", "kept", "new_len"), kw)


BAD_CACHE = [dict(cache={n: v}) for n in PLANES[:4] for v in (None, 0x1008)] + \
    [dict(cache=dict(weights=0x1004)), dict(cache=dict(num_pages=0)), dict(cache=dict(num_pages=1 << 31))]


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), INVALID), (dict(total_tokens=-1), INVALID), (dict(max_seqlen=-1), INVALID), (dict(h_kv=0), INVALID),
    (dict(h_kv=33), INVALID), (dict(head_dim=64), UNSUPPORTED), (dict(head_dim=0), INVALID), (dict(flags=4), INVALID),
    (dict(flags=16 | 1), INVALID), (dict(flags=256), INVALID), (dict(k_stride=255), INVALID), (dict(k_stride=128), INVALID),
    (dict(v_stride=260), INVALID), (dict(k_stride=1 << 31), INVALID), (dict(cu_seqlens=None), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(slot_mapping=None), INVALID), (dict(k_mean=None), INVALID), (dict(k_tscale=None), INVALID),
    (dict(v_tscale=None), INVALID), (dict(k=0x1002), INVALID), (dict(v=0x1008), INVALID), (dict(k_out=0x1008), INVALID),
    (dict(v_out=0x1004), INVALID), (dict(batch=65536), UNSUPPORTED),
    (dict(total_tokens=1 << 28, max_seqlen=1 << 28), UNSUPPORTED),
    (dict(total_tokens=(1 << 28) + 1), UNSUPPORTED)] + [(c, INVALID) for c in BAD_CACHE])
def test_write(mp, kw, status):
    assert mp.lib().mpfa_kv4_write(C.byref(_write(mp, **kw)), 0x1000, 1 << 40, None) == status


def test_write_workspace(mp):
    need = mp.kv4_write_workspace_size(2, 10, 2)
    for ws, size in ((None, need), (0x1000, need - 1), (0x1008, need)):
        assert mp.lib().mpfa_kv4_write(C.byref(_write(mp)), ws, size, None) == WORKSPACE
    assert mp.lib().mpfa_kv4_write(None, 0x1000, need, None) == INVALID
    out = C.c_size_t(0)
    for args in ((0, 1, 1), (1, -1, 1), (1, 1, 0), (1, 1, 33)):
        assert mp.lib().mpfa_kv4_write_workspace_size(*args, C.byref(out)) == INVALID
    assert mp.lib().mpfa_kv4_write_workspace_size(1, 1, 1, None) == INVALID


ATTN_BAD = [
    (dict(batch=0), INVALID), (dict(batch=65536), INVALID), (dict(h_q=7), INVALID), (dict(h_kv=0), INVALID),
    (dict(h_kv=33, h_q=33), INVALID), (dict(h_q=258), INVALID), (dict(head_dim=256), UNSUPPORTED), (dict(head_dim=-1), INVALID),
    (dict(max_pages=0), INVALID), (dict(max_pages=1 << 26), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID),
    (dict(partition_tokens=100), INVALID), (dict(partition_tokens=-128), INVALID), (dict(max_partitions=-1), INVALID),
    (dict(q_stride=1000), INVALID), (dict(q_stride=1028), INVALID), (dict(q=None), INVALID), (dict(q=0x1008), INVALID),
    (dict(out=None), INVALID), (dict(out=0x1004), INVALID), (dict(kv_len=None), INVALID), (dict(page_table=None), INVALID),
    (dict(k_tscale=None), INVALID), (dict(v_tscale=None), INVALID)] + [(c, INVALID) for c in BAD_CACHE]


@pytest.mark.parametrize("kw,status", ATTN_BAD + [
    (dict(flags=512), INVALID), (dict(flags=1), INVALID), (dict(q_tokens=1), INVALID), (dict(cu_seqlens_q=None), INVALID),
    (dict(q_start=None), INVALID), (dict(max_seqlen_q=-1), INVALID), (dict(total_tokens=-1), INVALID),
    (dict(items=0x1000), INVALID), (dict(items=0x1000, n_items=2, n_merges=3), INVALID),
    (dict(items=0x1000, n_items=2, n_merges=-1), INVALID), (dict(items=0x1000, n_items=2, n_states=3), INVALID),
    (dict(items=0x1000, n_items=2, n_states=-1), INVALID), (dict(items=0x1000, n_items=2, half=2), INVALID),
    (dict(items=0x1000, n_items=2, half=1, h_q=256, h_kv=1, q_stride=256 * 128), INVALID),
    (dict(items=0x1000, n_items=1 << 22), UNSUPPORTED), (dict(items=0x1000, n_items=70000, n_merges=65536), UNSUPPORTED),
    (dict(total_tokens=1 << 28, max_seqlen_q=2 ** 31 - 1, batch=65535), UNSUPPORTED),
    (dict(total_tokens=(1 << 28) + 1), UNSUPPORTED)])
def test_prefill(mp, kw, status):
    assert mp.lib().mpfa_kv4_prefill(C.byref(_attn(mp, **kw)), 0x1000, 1 << 60, None) == status


@pytest.mark.parametrize("half", [0, 1])
def test_prefill_workspace(mp, half):
    a = _attn(mp, items=0x1000, n_items=5, n_merges=2, n_states=4, half=half)
    need = 4 * 2 * (128 if half else 256) * 130 * 4
    for ws, size in ((None, need), (0x1000, need - 1), (0x1008, need)):
        assert mp.lib().mpfa_kv4_prefill(C.byref(a), ws, size, None) == WORKSPACE
    assert mp.lib().mpfa_kv4_prefill(None, None, 0, None) == INVALID


@pytest.mark.parametrize("kw,status", ATTN_BAD + [
    (dict(flags=1), INVALID), (dict(flags=256), INVALID), (dict(q_tokens=0), INVALID), (dict(q_tokens=-1), INVALID),
    (dict(q_tokens=65536), INVALID), (dict(partition_tokens=0), INVALID), (dict(max_partitions=0), INVALID),
    (dict(flags=512, cache=dict(weights=None)), INVALID), (dict(q_tokens=65535, h_q=256, h_kv=32, q_stride=256 * 128, max_partitions=8192), UNSUPPORTED),
    (dict(max_partitions=1 << 24), UNSUPPORTED)])
def test_decode(mp, kw, status):
    assert mp.lib().mpfa_kv4_decode(C.byref(_decode(mp, **kw)), 0x1000, 1 << 60, None) == status


def test_decode_workspace(mp):
    states = 2 * 8 * 2 * 130 * 4
    for ws, size in ((None, states), (0x1000, states - 1), (0x1008, 1 << 30)):
        assert mp.lib().mpfa_kv4_decode(C.byref(_decode(mp)), ws, size, None) == WORKSPACE
    with_scores = (states + 255) // 256 * 256 + 2 * 8 * 2 * 128 * 4
    assert mp.lib().mpfa_kv4_decode(C.byref(_decode(mp, flags=512)), 0x1000, with_scores - 1, None) == WORKSPACE
    assert mp.lib().mpfa_kv4_decode(None, 0x1000, 1 << 30, None) == INVALID


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), INVALID), (dict(h_kv=0), INVALID), (dict(h_kv=33), INVALID), (dict(max_pages=0), INVALID),
    (dict(dst_max_pages=0), INVALID), (dict(max_pages=1 << 26), INVALID), (dict(budget=0), INVALID), (dict(sinks=-1), INVALID),
    (dict(recent=-1), INVALID), (dict(sinks=60, recent=5), INVALID), (dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), INVALID),
    (dict(flags=512), INVALID), (dict(cache=dict(weights=None)), INVALID), (dict(kv_len=None), INVALID),
    (dict(page_table=None), INVALID), (dict(dst_page_table=None), INVALID), (dict(kept=None), INVALID), (dict(new_len=None), INVALID),
    (dict(batch=65536), UNSUPPORTED)] + [(c, INVALID) for c in BAD_CACHE])
def test_evict(mp, kw, status):
    assert mp.lib().mpfa_kv4_evict(C.byref(_evict(mp, **kw)), None) == status


def test_evict_null(mp):
    assert mp.lib().mpfa_kv4_evict(None, None) == INVALID


def test_calls_without_tokens_do_nothing(mp):
    assert mp.lib().mpfa_kv4_write(C.byref(_write(mp, total_tokens=0, k=None)), None, 0, None) == 0
    assert mp.lib().mpfa_kv4_prefill(C.byref(_attn(mp, total_tokens=0, q=None)), None, 0, None) == 0


def _plan(mp, name, *args, outs=2):
    import numpy as np
    arrays = [np.asarray(a, np.int32) if isinstance(a, list) else a for a in args]
    out = *(C.c_int32(-7) for _ in range(outs)), C.c_size_t(7)
    ptrs = [a.ctypes.data if hasattr(a, "ctypes") else a for a in arrays]
    rc = getattr(mp.lib(), name)(*ptrs, *(C.byref(o) for o in out))
    return rc, [o.value for o in out]


def _prefill_plan(mp, rows, kv, h_q, h_kv, window, sinks, cus=256):
    """The plan's items and merges, the number of states and whether the items are halved."""
    import numpy as np
    rc, (n, merges, states, half, size) = _plan(mp, "mpfa_kv4_prefill_plan", len(rows), rows, kv, h_q, h_kv, window, sinks, cus,
                                                None, 0, outs=4)
    assert rc == 0 and size == states * h_kv * (128 if half else 256) * 130 * 4
    table = np.full((n + merges, 6), -9, np.int32)
    few = np.empty((max(n + merges - 1, 0), 6), np.int32)
    args = (len(rows), rows, kv, h_q, h_kv, window, sinks, cus)
    if n + merges:
        assert _plan(mp, "mpfa_kv4_prefill_plan", *args, few.ctypes.data, n + merges - 1, outs=4)[0] == WORKSPACE
    assert _plan(mp, "mpfa_kv4_prefill_plan", *args, table.ctypes.data, n + merges, outs=4) == (0, [n, merges, states, half, size])
    return table[:n].tolist(), table[n:].tolist(), states, half


@pytest.mark.parametrize("args", [
    (0, [1], 8, 2, 1, 0, 0, 0, 256), (1, None, 8, 2, 1, 0, 0, 0, 256), (1, [-1], 8, 2, 1, 0, 0, 0, 256),
    (1, [1], 7, 2, 1, 0, 0, 0, 256), (1, [1], 8, 2, 0, 0, 0, 0, 256), (1, [1], 8, 2, 1, -1, 0, 0, 256),
    (1, [1], 8, 2, 1, 0, -1, 0, 256), (1, [1], 8, 2, 1, 0, 0, 1, 256), (1, [1], 8, 2, 1, 0, 0, 0, 0), (1, [1], 8, 2, 65536, 0, 0, 0, 256),
    (65535, [2 ** 31 - 1] * 65535, 256, 32, 65535, 0, 0, 0, 256)])
def test_decode_plan_refuses(mp, args):
    assert _plan(mp, "mpfa_kv4_decode_plan", *args)[0] == INVALID


@pytest.mark.parametrize("args", [
    (0, [1], [1], 8, 2, 0, 0, 256, None, 0), (1, None, [1], 8, 2, 0, 0, 256, None, 0), (1, [1], None, 8, 2, 0, 0, 256, None, 0),
    (1, [2], [1], 8, 2, 0, 0, 256, None, 0), (1, [-1], [1], 8, 2, 0, 0, 256, None, 0), (1, [1], [1], 8, 3, 0, 0, 256, None, 0),
    (1, [1], [1], 8, 2, -1, 0, 256, None, 0), (1, [1], [1], 8, 2, 0, 0, 0, None, 0), (1, [1], [1], 8, 2, 0, 0, 256, None, -1),
    (65536, [1], [1], 8, 2, 0, 0, 256, None, 0)])
def test_prefill_plan_refuses(mp, args):
    assert _plan(mp, "mpfa_kv4_prefill_plan", *args, outs=4)[0] == INVALID


def _visible_tiles(first, last, window, sinks):
    """By enumeration: 128-key tiles with a key that some row at first .. last sees."""
    tiles = set()
    for pos in (range(max(first, 0), last + 1)):
        lo = max(0, pos - window + 1) if window else 0
        tiles |= set(range(lo // 128, pos // 128 + 1))
        if window:
            tiles |= set(range(0, (min(sinks, pos + 1) + 127) // 128))
    return len(tiles)


@pytest.mark.parametrize("kv,q_tokens,window,sinks", [
    ([1, 129, 5000], 1, 0, 0), ([100000], 1, 1000, 4), ([100000], 8, 1, 300), ([700, 0, 3], 4, 128, 128), ([65536] * 3, 1, 0, 9),
    ([900], 1, 2 ** 31 - 1, 2 ** 31 - 1), ([4096], 1, 128, 0), ([4096, 200], 3, 126, 5), ([640], 1, 130, 513)])
def test_decode_plan_covers_the_visible_tiles(mp, kv, q_tokens, window, sinks):
    rc, (part, maxp, size) = _plan(mp, "mpfa_kv4_decode_plan", len(kv), kv, 8, 2, q_tokens, window, sinks, 512, 256)
    assert rc == 0 and part % 128 == 0 and maxp >= 1
    # of these lengths and of every shorter one (which may lie across one tile more)
    most = max(_visible_tiles(m - q_tokens, m - 1, window, sinks) for n in kv for m in range(max(n - 128, 0), n + 1))
    assert maxp * part >= most * 128 and (maxp - 1) * part < max(most, 1) * 128
    rows = len(kv) * q_tokens * 8
    assert size >= rows * (maxp * 130 + maxp * part) * 4


@pytest.mark.parametrize("rows,kv,h_q,h_kv,window,sinks", [
    ([1], [50000], 8, 2, 0, 0), ([70], [30000], 8, 2, 0, 0), ([5, 0], [9000, 1], 8, 2, 700, 70), ([777], [777], 32, 8, 0, 0),
    ([8192], [8192], 32, 8, 0, 0), ([512, 2048, 1000], [15512, 7049, 13345], 40, 8, 4096, 4), ([300] * 9, [300] * 9, 16, 1, 0, 0),
    ([40], [20000], 256, 1, 0, 0), ([3], [3], 32, 32, 1, 0), ([0], [7], 8, 8, 0, 0), ([20000], [90000], 10, 2, 0, 0)])
def test_prefill_plan_has_every_tile_once(mp, rows, kv, h_q, h_kv, window, sinks):
    items, merges, states, half = _prefill_plan(mp, rows, kv, h_q, h_kv, window, sinks)
    tm = (128 if half else 256) // (h_q // h_kv)
    want = {}
    for b, (r, n) in enumerate(zip(rows, kv)):
        for t in range(0, r, tm):
            want[b, t] = _visible_tiles(n - r + t, n - r + min(t + tm, r) - 1, window, sinks)
    got, kept = {}, {}
    for seq, row, first, last, state, parts in items:
        got.setdefault((seq, row), []).append((first, last))
        if parts > 1:
            kept.setdefault((seq, row), []).append((first, state, parts))
        else:
            assert state == -1
    assert got.keys() == want.keys()
    for k, spans in got.items():
        spans.sort()
        assert spans[0][0] == 0 and spans[-1][1] == want[k]
        assert all(a < b for a, b in spans) and all(x[1] == y[0] for x, y in zip(spans, spans[1:]))
    assert {(s, r) for s, r, *_ in merges} == kept.keys() and len(merges) == len(kept)
    used = []
    for seq, row, first, last, state, parts in merges:
        spans = sorted(kept[seq, row])
        assert [x[1] for x in spans] == list(range(state, state + parts)) and {x[2] for x in spans} == {parts}
        used += [x[1] for x in spans]
    assert sorted(used) == list(range(states))
    lengths = [x[3] - x[2] for x in items]
    assert lengths == sorted(lengths, reverse=True)


def _struct(mp, data, cls):
    a = cls()
    for name, ctype in cls._fields_:
        if ctype is mp.Kv4Cache:
            a.cache = mp.Kv4Cache(num_pages=data.draw(I64))
        elif ctype is not C.c_void_p:
            v = data.draw(FLAGS if name == "flags" else (I64 if ctype is C.c_int64 else INTS))
            setattr(a, name, v & 0xFFFFFFFF if ctype is C.c_uint32 else v)
    return a


@SET
@given(data=st.data())
def test_null_pointers_never_launch(mp, data):
    L, size = mp.lib(), data.draw(st.sampled_from([0, 1 << 20, 1 << 40]))
    assert L.mpfa_kv4_write(C.byref(_struct(mp, data, mp.Kv4WriteArgs)), None, size, None) in ALLOWED
    a = _struct(mp, data, mp.Kv4AttnArgs)
    assert L.mpfa_kv4_prefill(C.byref(a), None, size, None) in ALLOWED
    assert L.mpfa_kv4_decode(C.byref(a), None, size, None) in ALLOWED
    assert L.mpfa_kv4_evict(C.byref(_struct(mp, data, mp.Kv4EvictArgs)), None) in ALLOWED


def test_binding_refuses_what_it_cannot_pass_on(mp):
    import torch
    c, s = mp.PagedCache4(2, 2, device="cpu", weights=True), mp.SeqStats4(1, 2, device="cpu")
    k = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    cu, slots = torch.tensor([0, 3], dtype=torch.int32), torch.arange(3)
    with pytest.raises(ValueError):
        mp.kv4_write(k.float(), k, cu, slots, c, s, 0, 3)
    with pytest.raises(ValueError):
        mp.kv4_write(k.transpose(0, 1).contiguous().transpose(0, 1), k, cu, slots, c, s, 0, 3)   # heads lie apart
    with pytest.raises(ValueError):
        mp.kv4_write(k, k, cu.long(), slots, c, s, 0, 3)
    with pytest.raises(ValueError):
        mp.kv4_write(k, k, cu, slots[:2], c, s, 0, 3)
    with pytest.raises(ValueError):
        mp.kv4_write(k, k, torch.tensor([0, 1, 3], dtype=torch.int32), slots, c, s, 0, 3)         # statistics of one sequence
    with pytest.raises(ValueError):
        mp.PagedCache4(3, 2, planes=dict(k_codes=c.k_codes, k_scales=c.k_scales, v_codes=c.v_codes, v_scales=c.v_scales))
    i32 = dict(dtype=torch.int32)
    table, one = torch.zeros(1, 1, **i32), torch.ones(1, **i32)
    plan = mp.Kv4Plan(("decode", 1, 4, 2, 0, 0), None, partition_tokens=128, max_partitions=1, q_tokens=1, flags=0)
    q = torch.zeros(1, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        mp.kv4_decode(q, c, s, one, table, torch.empty_like(q), plan, window=5)                    # a plan of another window
    with pytest.raises(ValueError):
        mp.kv4_decode(torch.cat([q, q]), c, s, one, table, torch.empty_like(q), plan)
    with pytest.raises(ValueError):
        mp.kv4_evict(c, one, table, table, 4, torch.zeros(1, 2, 5, **i32), one)
    with pytest.raises(ValueError, match="another call"):
        mp.kv4_prefill(q, c, s, torch.tensor([0, 1], **i32), one, one, table, torch.empty_like(q), plan)   # a decode's plan
    # tensors of the right shapes in host memory
    with pytest.raises(ValueError, match="GPU"):
        mp.kv4_write(k, k, cu, slots, c, s, 0, 3)
    with pytest.raises(ValueError, match="GPU"):
        mp.kv4_decode(q, c, s, one, table, torch.empty_like(q), plan)
    with pytest.raises(ValueError, match="GPU"):
        mp.kv4_prefill(q, c, s, torch.tensor([0, 1], **i32), one, one, table, torch.empty_like(q))
    with pytest.raises(ValueError, match="GPU"):
        mp.kv4_evict(c, one, table, table, 4, torch.zeros(1, 2, 4, **i32), one)
    with pytest.raises(AttributeError):
        c.k_codes = c.v_codes   # the addresses are taken once
