"""The norm's outputs in the place of its inputs, where that is allowed: the bytes of the same call out of place."""
import pytest
import torch

from tests.test_gpu_rms_norm import _inputs, mp  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width", [8, 64, 72, 128, 264, 512, 520, 4096, 16392, 32768])
@pytest.mark.parametrize("rows", [1, 300])
def test_in_place(mp, rows, width):   # noqa: F811
    x, w, res = _inputs(rows, width, seed=rows + width)
    group = 128
    for residual in (None, res):
        want, total = torch.empty_like(x), None if residual is None else torch.empty_like(res)
        mp.rms_norm(x, w, want, residual=residual, residual_out=total)
        y = x.clone()                     # out in the place of x
        got = None if residual is None else torch.empty_like(res)
        mp.rms_norm(y, w, y, residual=residual, residual_out=got)
        assert torch.equal(y, want) and (residual is None or torch.equal(got, total))
    y, keep, out = x.clone(), res.clone(), torch.empty_like(x)   # the sum in the place of x
    mp.rms_norm(y, w, out, residual=keep, residual_out=y)
    assert torch.equal(y, total) and torch.equal(out, want) and torch.equal(keep, res)
    y, r = x.clone(), res.clone()         # out in that of x, the sum in that of the residual
    mp.rms_norm(y, w, y, residual=r)
    assert torch.equal(y, want) and torch.equal(r, total)
    codes = torch.empty(rows, width, dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty(rows, -(-width // group), device="cuda")
    wc, ws = torch.empty_like(codes), torch.empty_like(scales)
    mp.rms_norm(x, w, wc, residual=res.clone(), scales=ws, group=group)
    y = x.clone()                         # the sum in the place of x, codes
    mp.rms_norm(y, w, codes, residual=res, residual_out=y, scales=scales, group=group)
    assert torch.equal(codes.view(torch.uint8), wc.view(torch.uint8)) and torch.equal(scales, ws) and torch.equal(y, total)
