"""The key that parts the blocks taken from the others (csrc/parting.h), on the host: both numbers of parts against sorting, at the borders of what a key can be.
The compiled program counts as the kernels do: every key with key - lo <= width, in 32 bits."""
import subprocess

import numpy as np
import pytest

from paper_2605_02218_amd import build as B

PROGRAM = r"""
#include <stdio.h>
#include <vector>
#include "parting.h"
using namespace covspec;
template <int BITS> int take(const std::vector<uint32_t>& keys, int top, std::vector<int>& out) {
  uint32_t lo = kAlways, hi = 0;
  int always = 0, there = 0;
  for (uint32_t x : keys) {
    always += x == kAlways;
    there += x != kNone;
    if (x != kNone && x != kAlways) { if (x < lo) lo = x; if (x > hi) hi = x; }
  }
  int passes = 0;
  Parting p = {0, 0};
  if (there - always > top - always)
    p = parting_key<BITS>(lo, hi, top - always, [&](int pass, uint32_t lo, uint32_t width, int shift, int need) {
      passes = pass + 1;
      std::vector<int> bins(1 << BITS);
      for (uint32_t x : keys)
        if (x - lo <= width) {
          if (((x - lo) >> shift) >= bins.size()) { puts("a part that is not there"); fflush(stdout); _Exit(3); }
          ++bins[(x - lo) >> shift];
        }
      int before = 0;
      for (int b = (1 << BITS) - 1; b >= 0; --b) {
        if (before + bins[b] >= need) return Part{b, before, bins[b]};
        before += bins[b];
      }
      puts("no part");
      fflush(stdout);
      _Exit(3);
    });
  int more = p.more;
  for (size_t i = 0; i < keys.size(); ++i) {
    const bool eq = keys[i] == p.at && p.at != 0 && more > 0;
    if (keys[i] > p.at || eq) out.push_back((int)i);
    more -= eq;
  }
  return passes;
}
int main() {
  int n, top, bits;
  while (fread(&n, 4, 1, stdin) == 1 && fread(&top, 4, 1, stdin) == 1 && fread(&bits, 4, 1, stdin) == 1) {
    std::vector<uint32_t> keys(n);
    if (fread(keys.data(), 4, n, stdin) != (size_t)n) return 1;
    std::vector<int> out;
    printf("%d", bits == 8 ? take<8>(keys, top, out) : take<10>(keys, top, out));
    for (int i : out) printf(" %d", i);
    puts("");
  }
}
"""
NONE, ALWAYS, NAN = 0, 0xFFFFFFFF, 0xFFC00000


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("parting")
    (d / "parting.hip").write_text(PROGRAM)
    subprocess.run([B._hipcc(), "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", B.CSRC, str(d / "parting.hip"), "-o", str(d / "parting")], check=True, capture_output=True)
    return str(d / "parting")


def key_of(score):
    u = np.asarray(score, dtype=np.float32).view(np.uint32)
    return u ^ np.where(u >> 31, np.uint32(0xFFFFFFFF), np.uint32(0x80000000))


def check(program, keys, top, bits):
    keys = np.ascontiguousarray(keys, dtype=np.uint32)
    assert (keys == ALWAYS).sum() <= top
    run = subprocess.run([program], input=np.array([len(keys), top, bits], dtype=np.int32).tobytes() + keys.tobytes(), capture_output=True, timeout=60)
    assert run.returncode == 0, run.stdout.decode()
    got = [int(x) for x in run.stdout.split()]
    want = sorted(sorted(np.flatnonzero(keys != NONE).tolist(), key=lambda i: (-int(keys[i]), i))[:top])
    assert got[1:] == want and got[0] <= 4


@pytest.mark.parametrize("bits", [8, 10])
@pytest.mark.parametrize("nb", [300, 500, 1500, 2000])
@pytest.mark.parametrize("low", [-1.0, -3e38, -1e-30, 0.0, 1.0])
def test_more_nans_than_places_beside_negative_scores(program, bits, nb, low):
    rng = np.random.default_rng(nb)
    keys = key_of(np.ones(nb)).copy()
    keys[rng.permutation(np.arange(2, nb - 2))[:100]] = NAN
    keys[1] = key_of(low)
    keys[[0, nb - 1]] = ALWAYS
    check(program, keys, 48, bits)
    keys[5::7] = NONE
    check(program, keys, 48, bits)


@pytest.mark.parametrize("bits", [8, 10])
@pytest.mark.parametrize("seed", range(12))
def test_keys_of_any_kind(program, bits, seed):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(60, 2049))
    kinds = [rng.integers(0, 1 << 32, n, dtype=np.uint64), key_of(rng.standard_normal(n)), key_of(np.round(rng.standard_normal(n) * 3)),
             rng.choice(np.array([1, 2, 0x7FFFFF, 0x800000, 0x7FFFFFFF, 0x80000000, 0xFF7FFFFF, 0xFF800000, NAN, 0xFFFFFFFD, 0xFFFFFFFE], dtype=np.uint64), n),
             0xFFFFFFFE - rng.integers(0, 300, n, dtype=np.uint64), 1 + rng.integers(0, 1 << 24, n, dtype=np.uint64)]
    for k in kinds:
        k = k.astype(np.uint32)
        k[k == ALWAYS] = ALWAYS - 1
        for top in (1, 5, 48):
            keys = k.copy()
            keys[rng.integers(0, n, n // 9)] = NONE
            keys[rng.integers(0, n, min(top, 4))] = ALWAYS
            check(program, keys, top, bits)
