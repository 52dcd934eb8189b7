"""One workspace for all calls of a server: the size for its largest call is enough for every smaller one."""
import random

import pytest

from tests.test_abi_fuzz import mp  # noqa: F401

HEADS = [(1, 1), (8, 8), (32, 32), (8, 2), (32, 8), (40, 8), (10, 2), (16, 1), (256, 1), (256, 256)]


@pytest.mark.parametrize("h_q,h_kv", HEADS)
def test_longer_calls_take_no_less(mp, h_q, h_kv):   # noqa: F811
    size = lambda batch, total, longest: mp.linear_prefill_workspace_size(batch, total, longest, h_q, h_kv)   # noqa: E731
    for batch in (1, 3, 64, 65, 500):
        lengths = [size(batch, n, n) for n in range(0, 100000, 37)]
        assert lengths == sorted(lengths), batch
    lengths = [size(1, 90000, n) for n in range(0, 90000, 37)]   # the longest prompt alone
    assert lengths == sorted(lengths)
    batches = [size(n, 5000, 5000) for n in range(1, 600)]
    assert batches == sorted(batches)


def test_any_smaller_call(mp):   # noqa: F811
    rng = random.Random(0)
    up_to = lambda n: rng.randint(0, n) if rng.random() < 0.5 else int(n ** rng.random())   # noqa: E731
    for _ in range(20000):
        h_q, h_kv = rng.choice(HEADS)
        batch, total, longest = 1 + up_to(999), up_to(1 << 28), up_to(1 << 28)
        small = 1 + up_to(batch - 1), up_to(total), up_to(longest)
        assert mp.linear_prefill_workspace_size(*small, h_q, h_kv) <= mp.linear_prefill_workspace_size(batch, total, longest, h_q, h_kv), \
            (small, batch, total, longest, h_q, h_kv)
