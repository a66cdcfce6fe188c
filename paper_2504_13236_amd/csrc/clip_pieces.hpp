// How the tiles of a list of tensors are cut into pieces that the workgroups of a launch take in turn (clip.hip).
#pragma once
#include "internal.hpp"

namespace nnt {
namespace {

constexpr int kPiece = 16384;          // elements: 64 KB of fp32
constexpr int kListed = 48;            // tensors of a launch: their geometry travels in its arguments (4 KB at most)

struct Listed {
    void* const* in;
    void* const* out;
    int32_t shape[kMaxDim], base[kMaxDim], grid[kMaxDim];
    int32_t first;                     // number of its first piece
    int32_t per_tile;                  // pieces of its largest tile
    int32_t bf16;
};
struct List {
    Listed t[kListed];
    int32_t n, pieces;
};

// Piece number `w`: tile and elements [first, first + count) of it (count 0: beyond the end of a smaller tile).
struct Piece {
    const Listed* t;
    int32_t tile;
    int64_t first;
    int32_t count;
};
__host__ __device__ __forceinline__ Piece piece_of(const List& a, int w) {
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.t[mid].first <= w) lo = mid;
        else hi = mid - 1;
    }
    const Listed& t = a.t[lo];
    const int k = w - t.first;
    Piece p;
    p.t = &t;
    p.tile = k / t.per_tile;
    p.first = (int64_t)(k - p.tile * t.per_tile) * kPiece;
    int64_t n = 1;
    int c = p.tile;
#pragma unroll
    for (int d = 0; d < kMaxDim; d++) {
        const int at = c % t.grid[d];
        c /= t.grid[d];
        n *= min(t.base[d], t.shape[d] - at * t.base[d]);
    }
    // (in 64 bits: a small tile may end more than 2^31 elements before a piece that only larger ones have)
    const int64_t left = n - p.first;
    p.count = left <= 0 ? 0 : left < kPiece ? (int)left : kPiece;
    return p;
}

}  // namespace
}  // namespace nnt
