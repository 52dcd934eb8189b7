"""How prompts are cut: every segment has a number of its own below those that are launched, with places in the workspace
for it.  The rules are the library's own header, compiled for the host."""
import ctypes as C
import os
import random
import subprocess

import pytest

from tests.test_abi_fuzz import mp  # noqa: F401

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_33135_amd", "csrc")
SOURCE = """
#include "linear_cut.h"
using namespace mpfa;
extern "C" {
void space(int batch, int total, int longest, int h_q, int h_kv, int64_t* out) {
  const LinearSpace s = linear_space(batch, total, longest, h_q, h_kv);
  const int64_t x[] = {s.segment, s.parts, s.heads, s.split, s.items, (int64_t)s.starts, (int64_t)s.bytes};
  for (int i = 0; i < 7; ++i) out[i] = x[i];
}
int count(int len, int segment, int split) { return linear_count(len, segment, split); }
int first(int begin, int segment, int b) { return linear_first(begin, segment, b); }
// the sequence that number id is looked up in, -1 if offsets out of range are read
int search(const int* cu, int batch, int segment, int id) {
  struct Offsets {
    const int* cu;
    int n;
    bool* bad;
    int operator[](int i) const {
      if (i < 0 || i >= n) *bad = true;
      return i < 0 || i >= n ? 0 : cu[i];
    }
  };
  bool bad = false;
  const int b = linear_search(Offsets{cu, batch, &bad}, batch, segment, id, [](auto before) {
    int n = 0;
    for (int lane = 0; lane < 64; ++lane) n += before(lane);
    return n;
  });
  return bad ? -1 : b;
}
}
"""
STATE, UNITS, DENSE, CHUNK = 128 * 128 * 4, 256, 64, 64


class Space:
    def __init__(self, cut, *sizes):
        x = (C.c_int64 * 7)()
        cut.space(*sizes, x)
        self.segment, self.parts, self.heads, self.split, self.items, self.starts, self.bytes = x


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    at = tmp_path_factory.mktemp("cut")
    (at / "cut.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, "-o", str(at / "cut.so"), str(at / "cut.cpp")])
    return C.CDLL(str(at / "cut.so"))


def _numbers(cut, lens, s):
    """Per sequence the first number and the count of its segments, as the kernels have them."""
    out, begin, dense = [], 0, 0
    for b, n in enumerate(lens):
        count = cut.count(n, s.segment, s.split)
        out.append((dense if len(lens) <= DENSE else cut.first(begin, s.segment, b), count))
        begin, dense = begin + n, dense + count
    return out


def _check(cut, mp, lens, total, longest, h_q, h_kv):   # noqa: F811
    what = (lens, total, longest, h_q, h_kv)
    s = Space(cut, len(lens), total, longest, h_q, h_kv)
    assert s.segment > 0 and s.segment % CHUNK == 0 and s.items % h_kv == 0, what
    if len(lens) * h_kv < 2 ** 23 - 1024:   # such a call is taken
        assert s.items <= (2 ** 32 - 1) // 512 - 8, what
    grp = h_q // h_kv
    assert 1 <= s.parts <= grp and (s.parts - 1) * s.heads < grp <= s.parts * s.heads, what
    behind = 0   # numbers of the sequences so far end here
    needed = False
    for (first, count), n in zip(_numbers(cut, lens, s), lens):
        assert first >= behind, what
        behind = first + count
        assert count == max(1, -(-n // s.segment)), what   # all its tokens
        needed |= count > 1 or s.parts > 1
    assert behind * h_kv <= s.items, what
    size = mp.linear_prefill_workspace_size(len(lens), total, longest, h_q, h_kv)
    assert s.bytes <= size, what
    if needed:   # a state and a decay for each number and KV head
        assert s.starts >= behind * h_kv * STATE and s.starts % 16 == 0 and s.bytes >= s.starts + behind * h_kv * 4, what


HEADS = [(1, 1), (8, 8), (32, 32), (8, 2), (32, 8), (40, 8), (10, 2), (16, 1), (12, 4), (256, 1), (256, 256)]


@pytest.mark.parametrize("h_q,h_kv", HEADS)
def test_segments_have_numbers_and_places(cut, mp, h_q, h_kv):   # noqa: F811
    rng = random.Random(h_q * 1000 + h_kv)
    for _ in range(1500):
        batch = rng.choice([1, 2, 3, 5, 8, 30, 63, 64, 65, 66, 130, 300])
        most = int(10 ** rng.uniform(0, 5))
        lens = [0 if rng.random() < 0.1 else rng.choice([rng.randint(1, most), most, min(most, 64), min(most, 65)]) for _ in range(batch)]
        total = sum(lens) + rng.choice([0, 0, 1, rng.randint(0, most)])
        longest = rng.choice([max(lens), max(lens) + 1, total, 2 ** 31 - 1])
        _check(cut, mp, lens, total, max(longest, max(lens)), h_q, h_kv)


@pytest.mark.parametrize("lens,h_q,h_kv", [([1 << 28], 32, 8), ([1 << 28], 256, 256), ([1] * 65535, 8, 8), ([70] * 65535, 128, 128),
                                           ([0] * 65534 + [1 << 28], 8, 1), ([1 << 22] * 64, 1, 1), ([1 << 21] * 65, 2, 1)], ids=lambda x: str(x)[:16])
def test_largest_calls(cut, mp, lens, h_q, h_kv):   # noqa: F811
    _check(cut, mp, lens, sum(lens), max(lens), h_q, h_kv)


# Beside the GPU tests that go by these: segments of so many chunks, more of them than units.
LONG = [([16383, 1], 32, 32, 16), ([60000, 700, 1], 8, 2, 4)]


@pytest.mark.parametrize("lens,h_q,h_kv,chunks", LONG, ids=str)
def test_long_calls_have_two_items_a_unit(cut, mp, lens, h_q, h_kv, chunks):   # noqa: F811
    s = Space(cut, len(lens), sum(lens), max(lens), h_q, h_kv)
    items = sum(count for _, count in _numbers(cut, lens, s)) * h_kv
    assert s.split and s.segment == chunks * CHUNK and UNITS < items <= 2 * UNITS + len(lens) * h_kv
    _check(cut, mp, lens, sum(lens), max(lens), h_q, h_kv)


@pytest.mark.parametrize("begin", [0, 1, 64, 5000, 100000])
@pytest.mark.parametrize("batch", [65, 66, 130, 4096, 5000])
def test_numbers_are_found(cut, batch, begin):
    """Every number by its sequence, and those before a first sequence that does not begin at token 0 (a mistake of the caller)
    within the offsets."""
    rng, segment = random.Random(batch), 64
    lens = [0 if rng.random() < 0.2 else rng.randint(1, 300) for _ in range(batch)]
    cu = [begin]
    for n in lens:
        cu.append(cu[-1] + n)
    of, behind = {}, 0
    for b, n in enumerate(lens):
        behind = cut.first(cu[b], segment, b)
        for i in range(cut.count(n, segment, 1)):
            assert behind + i not in of
            of[behind + i] = b
    at = (C.c_int * (batch + 1))(*cu)
    for number in range(max(of) + 3):
        got = cut.search(at, batch, segment, number)
        assert 0 <= got < batch and got == of.get(number, got), (number, got)


def test_the_check_notices(cut, mp, monkeypatch):   # noqa: F811
    """A place or a number too few in what the check is told."""
    for field in ("items", "starts"):
        class Short(Space):
            def __init__(self, *args, field=field):
                super().__init__(*args)
                setattr(self, field, getattr(self, field) - (8 if field == "items" else 8 * STATE))
        with monkeypatch.context() as m:
            m.setitem(globals(), "Space", Short)
            with pytest.raises(AssertionError):
                _check(cut, mp, [64 * 12 + 1], 64 * 12 + 1, 64 * 12 + 1, 32, 8)
