"""Sizes of linear attention and the norm that do not fit the numbers they are handed on as."""
import pytest
import torch

from tests.test_abi_fuzz import mp  # noqa: F401

F32, I32, F8 = torch.float32, torch.int32, torch.float8_e4m3fn
MOST = 2 ** 31 - 1


def _z(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="meta")   # sizes alone


@pytest.fixture
def taken(mp, monkeypatch):   # noqa: F811
    """The arguments that the binding hands to the library."""
    seen = []
    monkeypatch.setattr(mp, "_call", lambda name, dev, stream, args, *more: seen.append(args._obj))
    return seen


@pytest.mark.parametrize("shape", [(2 ** 31, 8), (2 ** 32 + 4, 8), (2 ** 32 + 8,), (1, 2 ** 33 + 256), (2 ** 16, 2 ** 16, 8)], ids=str)
def test_norm_of_more_rows_or_channels_than_32_bits(mp, taken, shape):   # noqa: F811
    """Not the first few of them: nothing."""
    with pytest.raises(ValueError, match="32-bit"):
        mp.rms_norm(_z(*shape), None, _z(*shape))
    mp.rms_norm(_z(MOST, 8), None, _z(MOST, 8))
    assert len(taken) == 1 and taken[0].rows == MOST and taken[0].width == 8


@pytest.mark.parametrize("group", [2 ** 32, 2 ** 32 + 32, -2 ** 32, 2 ** 31])
def test_norm_groups(mp, taken, group):   # noqa: F811
    """One scale a row would be written as eight."""
    with pytest.raises(ValueError):
        mp.rms_norm(_z(4, 256), None, _z(4, 256, dtype=F8), scales=_z(4, 1, dtype=F32), group=group)
    with pytest.raises(ValueError):
        mp.rms_norm(_z(4, 256), None, _z(4, 256), group=group)
    assert not taken


def _prefill(mp, longest, batch=1):   # noqa: F811
    slots = _z(batch, dtype=I32)
    mp.linear_prefill(_z(10, 4, 128), _z(10, 2, 128), _z(10, 2, 128), _z(2, dtype=F32), _z(batch + 1, dtype=I32), _z(1, 2, 128, 128, dtype=F32),
                      slots, slots, _z(10, 4, 128), longest)


@pytest.mark.parametrize("longest", [2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 32 + 10, 2 ** 63])
def test_longest_prompt(mp, taken, longest):   # noqa: F811
    """A bound far above the tokens would be handed on as one far below them, by which prompts are not cut."""
    with pytest.raises(ValueError, match="32-bit"):
        _prefill(mp, longest)
    with pytest.raises(ValueError, match="32-bit"):
        mp.linear_prefill_workspace_size(1, 10, longest, 4, 2)
    _prefill(mp, MOST)
    assert len(taken) == 1 and taken[0].max_seqlen == MOST
    assert mp.linear_prefill_workspace_size(1, 10, MOST, 4, 2) == mp.linear_prefill_workspace_size(1, 10, 10, 4, 2)


def test_more_sequences_than_32_bits(mp, taken):   # noqa: F811
    with pytest.raises(ValueError, match="32-bit"):
        _prefill(mp, 10, batch=2 ** 32 + 1)
    with pytest.raises(ValueError, match="32-bit"):
        mp.linear_prefill_workspace_size(2 ** 32 + 1, 10, 10, 4, 2)
    assert not taken
