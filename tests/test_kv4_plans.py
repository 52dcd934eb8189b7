"""Plans and the calls that use them.  A plan's workspace and items belong to the plan, which a
caller may drop as soon as a call returns: on a stream other than the one they were made on they
are recorded as in use there."""
import ctypes as C
import types

import pytest
import torch

from tests.test_abi_fuzz import mp  # noqa: F401


class Memory:
    """What the binding asks of a plan's tensors."""

    def __init__(self):
        self.used_on = []

    def get_device(self):
        return -1

    def data_ptr(self):
        return 0x1000

    def numel(self):
        return 1 << 20

    def record_stream(self, stream):
        self.used_on.append(stream.cuda_stream)


class Library:
    """Accepts every call."""

    def __getattr__(self, name):
        return lambda *args: 0


@pytest.fixture
def launches(mp, monkeypatch):   # noqa: F811
    """The binding with host tensors taken for a device's, its stream 7 the current one."""
    monkeypatch.setattr(mp, "lib", Library)
    call = mp._call
    monkeypatch.setattr(mp, "_call", lambda name, dev, stream, *args: call(name, 0, stream, *args))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(mp, "_stream", lambda stream: 7 if stream is None else stream.cuda_stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: types.SimpleNamespace(cuda_stream=handle))
    i32 = dict(dtype=torch.int32)
    c, s = mp.PagedCache4(2, 2, device="cpu"), mp.SeqStats4(1, 2, device="cpu")
    q, one, table = torch.zeros(1, 4, 128, dtype=torch.bfloat16), torch.ones(1, **i32), torch.zeros(1, 1, **i32)

    def decode(plan, stream=None):
        mp.kv4_decode(q, c, s, one, table, torch.empty_like(q), plan, stream=stream)

    def prefill(plan, stream=None):
        mp.kv4_prefill(q, c, s, torch.tensor([0, 1], **i32), one * 0, one, table, torch.empty_like(q), plan, stream=stream)

    return decode, prefill


def decode_plan(mp, **kw):   # noqa: F811
    return mp.Kv4Plan(("decode", 1, 4, 2, 0, 0), Memory(), partition_tokens=128, max_partitions=1, q_tokens=1, **kw)


def prefill_plan(mp, **kw):   # noqa: F811
    return mp.Kv4Plan(("prefill", 1, 4, 2, 0, 0), Memory(), n_items=2, n_merges=1, n_states=2, max_rows=1, items=Memory(), **kw)


@pytest.mark.parametrize("home,stream,used_on", [(7, None, []), (3, None, [7]), (7, 5, [5]), (5, 5, []), (None, None, [7])])
def test_memory_of_a_plan_is_recorded_on_another_stream(mp, launches, home, stream, used_on):   # noqa: F811
    decode, prefill = launches
    on = None if stream is None else types.SimpleNamespace(cuda_stream=stream)
    plan = decode_plan(mp, home=home)
    decode(plan, on)
    assert plan.workspace.used_on == used_on
    plan = prefill_plan(mp, home=home)
    prefill(plan, on)
    assert plan.workspace.used_on == used_on and plan.items.used_on == used_on


def test_prefill_plan_of_more_rows_is_refused(mp, launches):   # noqa: F811
    _, prefill = launches   # one row
    prefill(prefill_plan(mp, rows=1))
    with pytest.raises(ValueError, match="rows"):
        prefill(prefill_plan(mp, rows=2))


def test_grid_of_the_weights_stays_below_its_bound(mp):   # noqa: F811
    """2^30 keys of 32 KV heads, 1024 to a workgroup: 2^25 workgroups of 256 threads are more than a grid takes."""
    a = mp.Kv4AttnArgs(batch=1, h_q=32, h_kv=32, head_dim=128, max_pages=1 << 24, q_tokens=1, q_stride=32 * 128, flags=mp.KV4_WEIGHTS,
                       partition_tokens=1 << 20, max_partitions=1 << 10, cache=mp.Kv4Cache(num_pages=1 << 24))
    for n in ("k_codes", "k_scales", "v_codes", "v_scales", "weights"):
        setattr(a.cache, n, 0x1000)
    for n in ("kv_len", "page_table", "q", "k_tscale", "v_tscale", "out"):
        setattr(a, n, 0x1000)   # never dereferenced
    assert mp.lib().mpfa_kv4_decode(C.byref(a), 0x1000, 1 << 60, None) == mp.MPFA_ERR_UNSUPPORTED
    out = C.c_int32(0), C.c_int32(0), C.c_size_t(0)
    for n, flags, status in ((1 << 30, mp.KV4_WEIGHTS, mp.MPFA_ERR_UNSUPPORTED), ((1 << 30) + 1, 0, mp.MPFA_ERR_UNSUPPORTED),
                             (1 << 28, mp.KV4_WEIGHTS, mp.MPFA_OK), (1 << 30, 0, mp.MPFA_OK)):
        kv = (C.c_int32 * 1)(n)   # a plan that no call would take is none
        assert mp.lib().mpfa_kv4_decode_plan(1, C.addressof(kv), 32, 32, 1, 0, 0, flags, 256, *(C.byref(x) for x in out)) == status, n


@pytest.mark.parametrize("tokens", [0, 1])
@pytest.mark.parametrize("stride", [0, 1001, 1 << 33])
def test_token_stride_of_a_single_token_does_not_matter(mp, tokens, stride):   # noqa: F811
    x = torch.zeros(256, dtype=torch.bfloat16).as_strided((tokens, 2, 128), (stride, 128, 1))
    assert mp._rows("x", x, 2, -1) == 256
