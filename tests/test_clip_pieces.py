"""How the clipping call cuts tiles into pieces, on the host: every element of every tile in exactly one piece, and nothing behind a tile, also
where a tile has more than 2^31 elements and the last one of its axis is smaller."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_13236_amd", "csrc")

PROGRAM = r"""
#include "clip_pieces.hpp"
#include <algorithm>
#include <cstdio>
#include <cstdlib>
using namespace nnt;

// arguments: axes, then shape and base of each axis
int main(int argc, char** argv) {
    const int nd = atoi(argv[1]);
    List l{};
    l.n = 2;
    Listed& one = l.t[0];                     // one piece in front
    Listed& t = l.t[1];
    int64_t tiles = 1, base_n = 1;
    for (int d = 0; d < kMaxDim; d++) {
        one.shape[d] = one.base[d] = one.grid[d] = 1;
        t.shape[d] = d < nd ? atoi(argv[2 + 2 * d]) : 1;
        t.base[d] = d < nd ? atoi(argv[3 + 2 * d]) : 1;
        t.grid[d] = (int32_t)(((int64_t)t.shape[d] + t.base[d] - 1) / t.base[d]);
        tiles *= t.grid[d];
        base_n *= t.base[d];
    }
    one.per_tile = 1;
    t.first = 1;
    t.per_tile = (int32_t)((base_n + kPiece - 1) / kPiece);
    l.pieces = 1 + (int32_t)(tiles * t.per_tile);
    int64_t seen = 0, behind = 0, at = 0;
    for (int w = 1; w < l.pieces; w++) {
        const Piece p = piece_of(l, w);
        int64_t n = 1;
        for (int d = 0, c = p.tile; d < kMaxDim; c /= t.grid[d], d++) n *= std::min<int64_t>(t.base[d], t.shape[d] - (int64_t)(c % t.grid[d]) * t.base[d]);
        if (p.first == 0) at = 0;
        if (p.count <= 0) continue;
        seen += p.count;
        if (p.t != &t || p.count > kPiece || p.first != at || p.first + p.count > n) behind++;
        at += p.count;
    }
    printf("%lld %lld\n", (long long)seen, (long long)behind);
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("pieces")
    (at / "pieces.hip").write_text(PROGRAM)
    subprocess.run(["hipcc", "-std=c++17", "-O1", "--offload-host-only", "-I" + CSRC, "-I" + os.path.join(ROOT, "include"), str(at / "pieces.hip"), "-o",
                    str(at / "pieces")], check=True, capture_output=True, timeout=300)
    return str(at / "pieces")


@pytest.mark.parametrize("shape,base", [
    ((1,), (1,)), ((16385,), (16384,)), ((7, 5), (3, 2)), ((300, 401), (128, 400)), ((5, 4, 3, 2), (2, 4, 2, 1)),
    ((65536, 32771), (65536, 32770)),          # 65536 elements in a tile that others fill with 2147614720
    ((65536, 65537), (65536, 65536)),          # 2^32
    ((1 << 20, 3, 3000), (1 << 20, 2, 2999)),
    ((2147483647,), (2147483646,)),
])
def test_pieces_are_the_tiles(program, shape, base):
    args = [str(len(shape))] + [str(v) for pair in zip(shape, base) for v in pair]
    seen, behind = (int(v) for v in subprocess.run([program] + args, check=True, capture_output=True, timeout=120, text=True).stdout.split())
    n = 1
    for v in shape:
        n *= v
    assert (seen, behind) == (n, 0)
