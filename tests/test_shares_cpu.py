"""The shares of a long axis of rounds (csrc/paged_shares.h), compiled for the host with wrapping integers and compared with
whole numbers that have no width: up to the largest count of rounds that kv_paged_attention takes, 2^31 - 1, where a share's
begin and its rounds add up to more than a signed number of 32 bits."""
import shutil
import subprocess

import pytest

from paper_2609_30738_amd import build

PROGRAM = """
#define __host__
#define __device__
#include "paged_shares.h"
#include <cstdio>
int main() {
  int T, n, share;
  while (scanf("%d %d %d", &T, &n, &share) == 3) {
    const int S = kv::share_of(T, n), at = kv::share_begin(T, S, share);
    printf("%d %d %d\\n", S, at, kv::share_end(T, S, at));
  }
}
"""

LEAST = 2  # rounds of a share
LARGEST = 2 ** 31 - 1
CASES = [(T, n) for n in (1, 2, 3, 96, 97, 105, 512, 520, 768, 776)
         for T in (0, 1, 2, 3, 4, 95, 96, 97, 191, 192, 193, 256, 100003, LARGEST // 2 + 1, LARGEST - 900, LARGEST - 2, LARGEST - 1, LARGEST)]


@pytest.fixture(scope="module")
def bounds(tmp_path_factory):
    """(T, n, share) -> rounds to a share, the share's first one and the one behind its last."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("needs g++")
    at = tmp_path_factory.mktemp("shares")
    src, exe = at / "shares.cpp", at / "shares"
    src.write_text(PROGRAM)
    subprocess.run([gxx, "-std=c++17", "-O1", "-fwrapv", f"-I{build.CSRC}", str(src), "-o", str(exe)], check=True)
    asked = [(T, n, share) for T, n in CASES for share in range(n)]
    out = subprocess.run([str(exe)], input="\n".join("%d %d %d" % x for x in asked), capture_output=True, text=True, check=True).stdout
    return dict(zip(asked, (tuple(map(int, line.split())) for line in out.splitlines())))


@pytest.mark.parametrize("T,n", CASES)
def test_shares_are_the_rounds(bounds, T, n):
    """Each share is what the definition gives, and all of them are the rounds from 0 to T - 1, one after the other."""
    S = max(-(-T // n), LEAST)
    behind = 0
    for share in range(n):
        begin, end = min(share * S, T), min((share + 1) * S, T)
        assert bounds[T, n, share] == (S, begin, end), share
        assert begin == behind
        behind = end
    assert behind == T


def test_the_largest_call(bounds):
    """32767 requests over 8,388,800 rows of one head: 2^31 - 2 rounds of 128 rows in 768 shares, whose last one would end
    past 2^31 if T did not cut it."""
    T, n = 32767 * -(-8388800 // 128), 768
    assert T == LARGEST - 1 and (T, n) in CASES
    S, begin, end = bounds[T, n, n - 1]
    assert begin + S > LARGEST and end == T
