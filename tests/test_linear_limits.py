"""The sizes from which linear attention and the norm are refused, as the header states them; nothing is launched."""
import ctypes as C

import pytest

from tests.test_abi_fuzz import mp  # noqa: F401
from tests.test_linear_refusals import UNSUPPORTED, _linear, _norm

WIDE = dict(q_stride=1 << 15, k_stride=1 << 15, v_stride=1 << 15, decay_stride=0)


@pytest.mark.parametrize("batch,heads", [(1 << 15, 256), (65535, 129), (65535, 256)])
@pytest.mark.parametrize("tokens", [0, 1, 1 << 28])
def test_prefill_grid(mp, batch, heads, tokens):   # noqa: F811
    a = _linear(mp, batch=batch, h_q=heads, h_kv=heads, total_tokens=tokens, max_seqlen=tokens, **WIDE)
    assert mp.lib().mpfa_linear_prefill(C.byref(a), 0x1000, 1 << 62, None) == UNSUPPORTED


@pytest.mark.parametrize("batch,heads", [(1 << 14, 256), (1 << 15, 128), (65535, 256), (65535, 65)])
def test_decode_grid(mp, batch, heads):   # noqa: F811
    a = _linear(mp, batch=batch, h_q=heads, h_kv=heads, **WIDE)
    assert mp.lib().mpfa_linear_decode(C.byref(a), None) == UNSUPPORTED


@pytest.mark.parametrize("width,threads", [(8, 8), (64, 8), (72, 16), (128, 16), (136, 32), (256, 32), (264, 64), (512, 64), (520, 64), (1024, 64),
                                           (1032, 128), (16384, 1024), (16392, 576), (32768, 1024)])
def test_norm_grid(mp, width, threads):   # noqa: F811
    rows = -(-(2 ** 32 - 256) // threads)
    if rows < 2 ** 31:
        assert mp.lib().mpfa_rms_norm(C.byref(_norm(mp, rows=rows, width=width, x_stride=width)), None) == UNSUPPORTED
