"""What linear attention and the norm refuse on the host, before any HIP call."""
import ctypes as C

import pytest

from tests.test_abi_fuzz import ALLOWED, FLAGS, I64, INTS, SET, _ints, mp  # noqa: F401
from hypothesis import given, strategies as st

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
POINTERS = ("cu_seqlens", "q", "k", "v", "log_decay", "state_src", "state_dst", "states", "out")


def _linear(mp, **kw):
    a = mp.LinearArgs(batch=2, total_tokens=10, max_seqlen=7, q_tokens=1, h_q=8, h_kv=2, head_dim=128, scale=0.1, num_states=4,
                      q_stride=1024, k_stride=256, v_stride=256, decay_stride=2)
    for n in POINTERS:
        setattr(a, n, 0x1000)   # never dereferenced: every call here fails before a launch
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def _norm(mp, **kw):
    a = mp.RmsNormArgs(rows=4, width=256, group=0, eps=1e-6, x_stride=256)
    for n in ("x", "weight", "residual", "residual_out", "out", "scales"):
        setattr(a, n, 0x1000)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


BAD = [(dict(batch=0), INVALID), (dict(batch=65536), INVALID), (dict(h_q=7), INVALID), (dict(h_kv=0), INVALID),
       (dict(h_q=258), INVALID), (dict(h_q=0), INVALID), (dict(head_dim=64), UNSUPPORTED), (dict(head_dim=0), INVALID),
       (dict(flags=1), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
       (dict(num_states=-1), INVALID), (dict(q_stride=1016), INVALID), (dict(q_stride=1028), INVALID),
       (dict(k_stride=128), INVALID), (dict(v_stride=257), INVALID), (dict(k_stride=1 << 31), INVALID),
       (dict(q_stride=1 << 25), INVALID), (dict(k_stride=1 << 25), INVALID), (dict(v_stride=1 << 25), INVALID), (dict(decay_stride=1 << 25), INVALID),
       (dict(decay_stride=1), INVALID), (dict(decay_stride=-1), INVALID), (dict(decay_stride=1 << 31), INVALID)] + \
    [({n: None}, INVALID) for n in POINTERS[1:]] + [({n: 0x1008}, INVALID) for n in ("q", "k", "v", "states", "out")]


@pytest.mark.parametrize("kw,status", BAD + [
    (dict(total_tokens=-1), INVALID), (dict(max_seqlen=-1), INVALID), (dict(cu_seqlens=None), INVALID),
    (dict(total_tokens=(1 << 28) + 1), UNSUPPORTED), (dict(batch=65535, h_q=256, h_kv=256, q_stride=1 << 15, k_stride=1 << 15, v_stride=1 << 15,
                                                           decay_stride=256, total_tokens=1 << 20), UNSUPPORTED)])
def test_prefill(mp, kw, status):   # noqa: F811
    assert mp.lib().mpfa_linear_prefill(C.byref(_linear(mp, **kw)), 0x1000, 1 << 60, None) == status


@pytest.mark.parametrize("kw,status", BAD + [
    (dict(q_tokens=0), INVALID), (dict(q_tokens=-1), INVALID), (dict(q_tokens=1025), INVALID)])
def test_decode(mp, kw, status):   # noqa: F811
    assert mp.lib().mpfa_linear_decode(C.byref(_linear(mp, **kw)), None) == status


def test_workspace(mp):   # noqa: F811
    a = _linear(mp, total_tokens=1000, max_seqlen=900)
    need = mp.linear_prefill_workspace_size(2, 1000, 900, 8, 2)
    assert need > 0 and mp.linear_prefill_workspace_size(2, 10, 7, 2, 2) == 0
    for ws, size in ((None, need), (0x1000, need - 1), (0x1008, need)):
        assert mp.lib().mpfa_linear_prefill(C.byref(a), ws, size, None) == WORKSPACE
    out = C.c_size_t(0)
    for args in ((0, 1, 1, 1, 1), (65536, 1, 1, 1, 1), (1, -1, 1, 1, 1), (1, 1, -1, 1, 1), (1, 1, 1, 3, 2), (1, 1, 1, 1, 0)):
        assert mp.lib().mpfa_linear_prefill_workspace_size(*args, C.byref(out)) == INVALID
    assert mp.lib().mpfa_linear_prefill_workspace_size(1, 1, 1, 1, 1, None) == INVALID
    assert mp.lib().mpfa_linear_prefill_workspace_size(1, (1 << 28) + 1, 1, 1, 1, C.byref(out)) == UNSUPPORTED
    assert mp.lib().mpfa_linear_prefill(None, None, 0, None) == INVALID
    assert mp.lib().mpfa_linear_decode(None, None) == INVALID


@pytest.mark.parametrize("batch,total,longest,h_q,h_kv", [
    (1, 1, 1, 1, 1), (1, 64, 64, 256, 256), (1, 65, 65, 1, 1), (3, 1000, 700, 8, 2), (1, 65536, 65536, 32, 8), (512, 40000, 9000, 8, 8),
    (65535, 1 << 20, 1 << 20, 1, 1), (1, 1 << 28, 1 << 28, 8, 1)])
def test_workspace_holds_every_segment(mp, batch, total, longest, h_q, h_kv):   # noqa: F811
    """A state and a decay per segment and KV head, at least one segment per sequence; none for prompts of one segment
    whose heads one workgroup takes."""
    size = mp.linear_prefill_workspace_size(batch, total, longest, h_q, h_kv)
    if longest <= 64 and h_q == h_kv:
        assert size == 0
    if size:
        assert size >= batch * h_kv * (65536 + 4)


@pytest.mark.parametrize("h_q,h_kv", [(8, 1), (40, 8), (256, 1)])
def test_workspace_where_workgroups_share_a_state(mp, h_q, h_kv):   # noqa: F811
    """Query heads that several workgroups take start from one state, which one of them replaces: it is read from a copy."""
    assert mp.linear_prefill_workspace_size(1, 10, 10, h_q, h_kv) >= h_kv * (65536 + 4)
    a = _linear(mp, batch=1, h_q=h_q, h_kv=h_kv, max_seqlen=10, q_stride=h_q * 128, k_stride=h_kv * 128, v_stride=h_kv * 128, decay_stride=0)
    assert mp.lib().mpfa_linear_prefill(C.byref(a), None, 0, None) == WORKSPACE


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), INVALID), (dict(width=0), INVALID), (dict(width=-8), INVALID), (dict(width=12), INVALID), (dict(width=32776, x_stride=32776), UNSUPPORTED),
    (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(group=16), INVALID), (dict(group=48), INVALID), (dict(group=1024), INVALID), (dict(group=-32), INVALID),
    (dict(group=32, scales=None), INVALID), (dict(x_stride=248), INVALID), (dict(x_stride=260), INVALID), (dict(x_stride=1 << 31), INVALID),
    (dict(x=None), INVALID), (dict(out=None), INVALID), (dict(residual=None), INVALID), (dict(residual_out=None), INVALID),
    (dict(x=0x1008), INVALID), (dict(weight=0x1008), INVALID), (dict(residual=0x1008), INVALID), (dict(residual_out=0x1008), INVALID),
    (dict(out=0x1004), INVALID), (dict(out=0x1008, scales=None), INVALID), (dict(scales=0x1002), INVALID),
    (dict(rows=2 ** 31 - 1, width=8192, x_stride=8192), UNSUPPORTED)])
def test_norm(mp, kw, status):   # noqa: F811
    assert mp.lib().mpfa_rms_norm(C.byref(_norm(mp, **kw)), None) == status


def test_norm_null_and_nothing(mp):   # noqa: F811
    assert mp.lib().mpfa_rms_norm(None, None) == INVALID
    assert mp.lib().mpfa_rms_norm(C.byref(_norm(mp, rows=0, x=None, out=None)), None) == 0


@SET
@given(data=st.data())
def test_null_pointers(mp, data):   # noqa: F811
    draw = lambda s: [data.draw(FLAGS if f[0] == "flags" else I64 if f[1] is C.c_int64 else st.floats() if f[1] is C.c_float else INTS)   # noqa: E731
                      for f in s._fields_ if f[1] is not C.c_void_p]
    a, n = _ints(mp.LinearArgs, draw(mp.LinearArgs)), _ints(mp.RmsNormArgs, draw(mp.RmsNormArgs))
    L = mp.lib()
    assert L.mpfa_linear_prefill(C.byref(a), None, 1 << 40, None) in ALLOWED
    assert L.mpfa_linear_decode(C.byref(a), None) in ALLOWED
    assert L.mpfa_rms_norm(C.byref(n), None) in ALLOWED
    assert L.mpfa_linear_prefill_workspace_size(*(data.draw(INTS) for _ in range(5)), C.byref(C.c_size_t())) in ALLOWED


def test_binding_refuses_on_the_host(mp):   # noqa: F811
    """Wrong shapes, types and strides raise ValueError before the library is asked; no GPU is needed."""
    import torch
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)   # noqa: E731
    i, st_ = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2, 128, 128)
    good = dict(q=z(10, 4, 128), k=z(10, 2, 128), v=z(10, 2, 128), log_decay=torch.zeros(2), states=st_, state_src=i, state_dst=i, out=z(10, 4, 128))
    bad = [dict(q=z(10, 512)), dict(q=z(10, 4, 64)), dict(k=z(9, 2, 128)), dict(k=z(10, 3, 128)), dict(v=z(10, 2, 128).float()),
           dict(v=z(10, 2, 256)[..., :128]), dict(log_decay=torch.zeros(3)), dict(log_decay=torch.zeros(9, 2)),
           dict(log_decay=torch.zeros(10, 4)[:, ::2]), dict(log_decay=torch.zeros(2).double()), dict(states=st_[..., :64]),
           dict(states=st_.half()), dict(states=st_.transpose(2, 3)), dict(state_src=i.long()), dict(state_dst=i[:1]),
           dict(out=z(9, 4, 128)), dict(out=z(10, 4, 256)[..., :128]), dict(out=torch.zeros(10, 4, 128))]
    cu = torch.zeros(3, dtype=torch.int32)
    for kw in bad:
        with pytest.raises(ValueError):
            mp.linear_prefill(cu_seqlens=cu, max_seqlen=7, **{**good, **kw})
        with pytest.raises(ValueError):
            mp.linear_decode(q_tokens=5, **{**good, **kw})
    with pytest.raises(ValueError):
        mp.linear_decode(q_tokens=4, **good)
    with pytest.raises(ValueError):
        mp.linear_prefill(cu_seqlens=cu.long(), max_seqlen=7, **good)
    with pytest.raises(ValueError, match="GPU"):   # all else in order: tensors in host memory
        mp.linear_prefill(cu_seqlens=cu, max_seqlen=7, **good)
    x, f8, s = z(4, 256), torch.zeros(4, 256).to(torch.float8_e4m3fn), torch.zeros(4, 2)
    for kw in (dict(x=x.float()), dict(x=z(4, 512)[:, ::2]), dict(x=z(2, 2, 512)[..., :256]), dict(weight=z(255)), dict(weight=z(256).float()),
               dict(out=f8), dict(out=z(3, 256)), dict(residual=z(3, 256)), dict(residual=x.float()), dict(residual_out=x),
               dict(scales=s), dict(scales=s, out=f8, group=64), dict(scales=s.double(), out=f8, group=128), dict(scales=s, out=f8, group=-1)):
        with pytest.raises(ValueError):
            mp.rms_norm(**{**dict(x=x, weight=z(256), out=z(4, 256)), **kw})
    with pytest.raises(ValueError, match="GPU"):
        mp.rms_norm(x, z(256), f8, scales=s, group=128)
