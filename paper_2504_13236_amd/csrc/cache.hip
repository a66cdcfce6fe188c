// A paged cache of keys and values, and the attention of new tokens over it (rollouts of a trained model, token by token or a
// part of a prompt at a time).
//
//   append     K[page][:, slot, j] = rot_p k_j,  V[page][:, slot, j] = v_j         p = start + s, page = pages[p / P], slot = p % P
//   attention  B = sum_k V[k] P[k],  P = softmax_k(scale K[k] . rot_p q),  k <= p  (and > p - window)
//
// A page is a tile (h, P, N_kv) of the cache's tensors: what one cached head reads of it is contiguous.
//
// The append is a copy; 58 MB take 17 us.  The attention reads what a (sequence, cached head) pair has cached once for all query rows of the pair, up to 128 of them,
// and is bound by that read while there are few: 510 MB of 64 sequences, one row each, 84 us; 535 MB of one sequence, four turned rows, 107 us (a large copy's rate would
// be 103 and 108); 200 tokens of four sequences of up to 3200 keys, 25 heads of 64, 35 us.  Long axes are split over workgroups, whose partial results a second kernel joins; short calls (4.5 us for 100
// keys) are launches.  These figures are of calls one after the other on two streams, which overlap; the launches of a call that is waited for take 22, 98 and 5, 128 and 10, 50 and 8, and 7 us.
#include "attention_tile.hpp"
#include "device_util.hpp"
#include "internal.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace nnt {
namespace {

constexpr int kE = 8;                       // components per lane

// Division of numbers below 2^31 by a fixed one: q = (n * mul) >> 32 >> shift.
struct Divide {
    uint32_t mul, shift, d;
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return d == 1 ? n : __umulhi(n, mul) >> shift; }
};

// [rows, N_s, N_b] with the heads side by side along the first axis
struct Rows {
    void* const* tiles;
    int32_t n0, n1, n2, b0, b1, b2, g0, g1;
    Divide by0, by1, by2;
};
// where a token's column lies: the number of its first row tile, and its place among the columns of a tile
struct TokenAt {
    int tile;
    int64_t col;
};
__device__ __forceinline__ TokenAt token_at(const Rows& r, int s, int b) {
    const int t1 = (int)r.by1((uint32_t)s), t2 = (int)r.by2((uint32_t)b), e1 = min(r.b1, r.n1 - t1 * r.b1);
    return TokenAt{r.g0 * (t1 + r.g1 * t2), (s - t1 * r.b1) + (int64_t)e1 * (b - t2 * r.b2)};
}
template <typename T>
__device__ __forceinline__ T* row_at(const Rows& r, const TokenAt& t, int row) {
    const int t0 = (int)r.by0((uint32_t)row), e0 = min(r.b0, r.n0 - t0 * r.b0);
    return global_as<T>(r.tiles[t0 + t.tile]) + (row - t0 * r.b0) + e0 * t.col;
}
template <typename T>
__device__ __forceinline__ T* row_at(const Rows& r, int row, int s, int b) { return row_at<T>(r, token_at(r, s, b), row); }

struct Cache {
    Rows z;                                  // queries, keys, values of the new tokens
    void* const* K;
    void* const* V;
    const int32_t *pages, *start, *count;
    const float* const* rot;                 // tiles of the rotation, NULL: none
    int32_t rot_r, rot_n, rot_base, rot_pairs;
    int32_t h, N_h, N_kv, P, n_pages, max_pages, window;
    bool rot_whole;                          // halves in whole vectors
    Divide by_P, by_rot;
};

__device__ __forceinline__ int new_tokens(const Cache& c, int b) { return c.count ? min(max(c.count[b], 0), c.z.n1) : c.z.n1; }

__device__ __forceinline__ void eight(const bf16_t* p, float (&x)[kE]) { ldv<8>(p, x); }
__device__ __forceinline__ void eight(const float* p, float (&x)[kE]) {
    float lo[4], hi[4];
    ldv<4>(p, lo);
    ldv<4>(p + 4, hi);
#pragma unroll
    for (int i = 0; i < 4; i++) { x[i] = lo[i]; x[i + 4] = hi[i]; }
}

// Components i0 .. i0 + 7 of R heads' rows, turned by the rotations of their positions p (0 <= p < rot_n).  The kind of rotation is asked for once, around all rows: their
// loads are then on their way together.
template <typename T, int R>
__device__ __forceinline__ void turned(const Cache& c, const T* const (&row)[R], int i0, const int (&p)[R], float (&x)[R][kE]) {
#pragma unroll
    for (int r = 0; r < R; r++) eight(row[r] + i0, x[r]);
    if (!c.rot || i0 >= c.rot_r) return;
    const int half = c.rot_r / 2;
    const float* cs[R];
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int t = (int)c.by_rot((uint32_t)p[r]);
        cs[r] = in_global(c.rot[t]) + (int64_t)(p[r] - t * c.rot_base) * c.rot_r;
    }
    if (c.rot_pairs) {
        float co[R][kE / 2], si[R][kE / 2];
        // (a pair behind the rotation's end is not turned)
#pragma unroll
        for (int r = 0; r < R; r++)
#pragma unroll
            for (int i = 0; i < kE / 2; i++) {
                const int k = min(i0 / 2 + i, half - 1);
                co[r][i] = cs[r][k];
                si[r][i] = cs[r][half + k];
            }
#pragma unroll
        for (int r = 0; r < R; r++)
#pragma unroll
            for (int i = 0; i < kE / 2; i++)
                if (i0 + 2 * i < c.rot_r) {
                    const float a = x[r][2 * i], b = x[r][2 * i + 1];
                    x[r][2 * i] = a * co[r][i] - b * si[r][i];
                    x[r][2 * i + 1] = a * si[r][i] + b * co[r][i];
                }
    } else if (c.rot_whole) {
        // all eight in one half, the others' eight and the eight angles in a row
        const bool second = i0 >= half;
        const int k = second ? i0 - half : i0;
        float other[R][kE], co[R][kE], si[R][kE];
#pragma unroll
        for (int r = 0; r < R; r++) {
            eight(row[r] + (second ? k : i0 + half), other[r]);
            eight(cs[r] + k, co[r]);
            eight(cs[r] + half + k, si[r]);
        }
#pragma unroll
        for (int r = 0; r < R; r++)
#pragma unroll
            for (int i = 0; i < kE; i++) x[r][i] = second ? other[r][i] * si[r][i] + x[r][i] * co[r][i] : x[r][i] * co[r][i] - other[r][i] * si[r][i];
    } else {
#pragma unroll
        for (int r = 0; r < R; r++)
#pragma unroll
            for (int i = 0; i < kE; i++) {
                const int at = i0 + i;
                if (at >= c.rot_r) continue;
                const bool second = at >= half;
                const int k = second ? at - half : at;
                float other[1];
                ldv<1>(row[r] + (second ? k : at + half), other);
                x[r][i] = second ? other[0] * cs[r][half + k] + x[r][i] * cs[r][k] : x[r][i] * cs[r][k] - other[0] * cs[r][half + k];
            }
    }
}
template <typename T>
__device__ __forceinline__ void turned(const Cache& c, const T* row, int i0, int p, float (&x)[kE]) {
    const T* const rows[1] = {row};
    const int ps[1] = {p};
    float y[1][kE];
    turned<T, 1>(c, rows, i0, ps, y);
#pragma unroll
    for (int i = 0; i < kE; i++) x[i] = y[0][i];
}

template <typename T>
__device__ __forceinline__ void put(T* p, const float (&x)[kE]) {
    if constexpr (sizeof(T) == 2) {
        stv<8>(p, x);
    } else {
        const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
        stv<4>(p, lo);
        stv<4>(p + 4, hi);
    }
}

// Where a new token goes: false where its page (or its rotation) is not there.
__device__ __forceinline__ bool slot_of(const Cache& c, int s, int b, int64_t& p, int& page, uint32_t& slot) {
    if (s >= new_tokens(c, b)) return false;
    p = (int64_t)c.start[b] + s;
    if (p < 0 || p >= (int64_t)c.max_pages * c.P || (c.rot && p >= c.rot_n)) return false;
    const uint32_t q = c.by_P((uint32_t)p);
    slot = (uint32_t)p - q * c.P;
    page = c.pages[(int64_t)b * c.max_pages + q];
    return page >= 0 && page < c.n_pages;
}
template <typename T>
__device__ __forceinline__ void copy_eight(const T* from, T* to) {      // (values leave as they came, whatever their bits)
    uint4 v[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; i++) v[i] = reinterpret_cast<const uint4*>(from)[i];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; i++) reinterpret_cast<uint4*>(to)[i] = v[i];
}

// A thread moves eight components of a key and of its value.
template <typename T>
__global__ void __launch_bounds__(256) append_kernel(Cache c, Divide by_token, Divide by_head) {
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, s = by_token(at), k = at - s * by_token.d, j = by_head(k);
    const int b = blockIdx.y, i0 = (int)(k - j * by_head.d) * kE;
    int64_t p;
    int page;
    uint32_t slot;
    if (s >= (uint32_t)c.z.n1 || !slot_of(c, (int)s, b, p, page, slot)) return;
    const int64_t to = ((int64_t)j * c.P + slot) * c.h + i0;
    const TokenAt token = token_at(c.z, (int)s, b);
    float x[kE];
    turned<T>(c, row_at<const T>(c.z, token, (c.N_h + (int)j) * c.h), i0, (int)p, x);
    put(global_as<T>(c.K[page]) + to, x);
    copy_eight<T>(row_at<const T>(c.z, token, (c.N_h + c.N_kv + (int)j) * c.h) + i0, global_as<T>(c.V[page]) + to);
}

// The same where nothing is turned, or all of a head by halves in whole vectors: a thread has eight components of each half, so that what is turned
// together, and its angles, is read once.  Eight prompts of up to 1024 tokens of 12 heads of 64 in fp32 (58 MB moved), turned: 19 -> 17 us.
template <typename T, bool kTurn>
__global__ void __launch_bounds__(256) append_halves_kernel(Cache c, Divide by_token, Divide by_head) {
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, s = by_token(at), k = at - s * by_token.d, j = by_head(k);
    const int b = blockIdx.y, i0 = (int)(k - j * by_head.d) * kE, half = c.h / 2;
    int64_t p;
    int page;
    uint32_t slot;
    if (s >= (uint32_t)c.z.n1 || !slot_of(c, (int)s, b, p, page, slot)) return;
    const int64_t to = ((int64_t)j * c.P + slot) * c.h + i0;
    const TokenAt token = token_at(c.z, (int)s, b);
    const T* key = row_at<const T>(c.z, token, (c.N_h + (int)j) * c.h) + i0;
    const T* value = row_at<const T>(c.z, token, (c.N_h + c.N_kv + (int)j) * c.h) + i0;
    T *ko = global_as<T>(c.K[page]) + to, *vo = global_as<T>(c.V[page]) + to;
    if constexpr (kTurn) {
        const int t = (int)c.by_rot((uint32_t)p);
        const float* cs = in_global(c.rot[t]) + (int64_t)((int)p - t * c.rot_base) * c.rot_r + i0;
        float x[kE], y[kE], co[kE], si[kE];
        eight(key, x);
        eight(key + half, y);
        eight(cs, co);
        eight(cs + half, si);
        uint4 v[sizeof(T)];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; i++) {
            v[i] = reinterpret_cast<const uint4*>(value)[i];
            v[i + sizeof(T) / 2] = reinterpret_cast<const uint4*>(value + half)[i];
        }
#pragma unroll
        for (int i = 0; i < kE; i++) {
            const float a = x[i], e = y[i];
            x[i] = a * co[i] - e * si[i];
            y[i] = a * si[i] + e * co[i];
        }
        put(ko, x);
        put(ko + half, y);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; i++) {
            reinterpret_cast<uint4*>(vo)[i] = v[i];
            reinterpret_cast<uint4*>(vo + half)[i] = v[i + sizeof(T) / 2];
        }
    } else {
        uint4 v[4][sizeof(T) / 2];
        const T* from[4] = {key, key + half, value, value + half};
        T* dst[4] = {ko, ko + half, vo, vo + half};
#pragma unroll
        for (int r = 0; r < 4; r++)
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; i++) v[r][i] = reinterpret_cast<const uint4*>(from[r])[i];
#pragma unroll
        for (int r = 0; r < 4; r++)
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; i++) reinterpret_cast<uint4*>(dst[r])[i] = v[r][i];
    }
}

// ---------------------------------------------------------------- attention
struct Attend {
    Cache c;
    Rows out;
    float scale;              // times log2(e): scores are exponents of two
    int32_t splits;           // workgroups that share the keys of a row, at most
    int32_t chunks;           // row chunks of a (sequence, cached head) pair
    Divide by_G, by_kv;       // query heads of a cached one, cached heads
    float* partial;           // [row][split][h + 2]: result of a split (not divided), its maximum, its sum
};

constexpr int kWaves = 4;
constexpr int kMostSplits = 128;
constexpr int kUnroll = 4;    // keys a lane has on their way at a time
constexpr int kTable = 512;   // pages whose addresses a workgroup keeps at a time

// The keys of a row chunk's split: the positions [lo, hi), of which a split takes `per`, whole steps.  (The host keeps the table's end, and 65536 more, below 2^31.)
struct Range {
    int lo, hi, per;
};
// rows r0 .. r0 + R - 1 of a (sequence, cached head) pair: row r is token r / G, query head j G + r % G
__device__ __forceinline__ Range range_of(const Attend& a, int start, int s_first, int s_last, uint32_t step) {
    Range g;
    const int64_t end = (int64_t)a.c.max_pages * a.c.P;
    g.hi = (int)max((int64_t)0, min((int64_t)start + s_last + 1, end));
    g.lo = a.c.window > 0 ? (int)min((int64_t)g.hi, max((int64_t)0, (int64_t)start + s_first + 1 - a.c.window)) : 0;
    const uint32_t steps = ((uint32_t)(g.hi - g.lo) + step - 1) / step;
    g.per = (int)(max(1u, (steps + (uint32_t)a.splits - 1) / (uint32_t)a.splits) * step);
    return g;
}
// a position between -1 and the last one a table may have
__device__ __forceinline__ int clamped(int64_t p) { return (int)max((int64_t)-1, min(p, (int64_t)INT32_MAX - 1)); }

template <typename T>
struct Eight {
    uint4 v[sizeof(T) == 2 ? 1 : 2];
    __device__ __forceinline__ void load(const T* p) {
        v[0] = *reinterpret_cast<const uint4*>(p);
        if constexpr (sizeof(T) == 4) v[1] = *(reinterpret_cast<const uint4*>(p) + 1);
    }
    __device__ __forceinline__ void zero() {
        v[0] = make_uint4(0u, 0u, 0u, 0u);
        if constexpr (sizeof(T) == 4) v[1] = v[0];
    }
    __device__ __forceinline__ void get(float (&f)[kE]) const {
        const uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                f[2 * i] = __uint_as_float(w[i] << 16);
                f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
            const uint32_t u[4] = {v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                f[i] = __uint_as_float(w[i]);
                f[i + 4] = __uint_as_float(u[i]);
            }
        }
    }
};

// The sum over the LPK lanes that share a key, in each of them: exchanges of neighbours, of pairs, of quads (halves of a row mirrored) and of eights as
// data-parallel moves, which cost an addition each; only what crosses a row of 16 goes through LDS.
template <int LPK>
__device__ __forceinline__ float lanes_sum(float d) {
    auto moved = [](float x, auto ctrl) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true)); };
    d += moved(d, std::integral_constant<int, 0xb1>());                          // lanes 1 0 3 2
    d += moved(d, std::integral_constant<int, 0x4e>());                          // lanes 2 3 0 1
    if constexpr (LPK >= 8) d += moved(d, std::integral_constant<int, 0x141>());  // 7 6 .. 0
    if constexpr (LPK >= 16) d += moved(d, std::integral_constant<int, 0x140>()); // 15 14 .. 0
    if constexpr (LPK >= 32) d += __shfl_xor(d, 16, 64);
    return d;
}

// One workgroup: R rows of a (sequence, cached head) pair against one split of the keys.  LPK lanes share a key, eight components each; a wavefront
// takes 64 / LPK keys at a time, and every such group of lanes carries a running maximum and sum of its own, which meet at the end.
template <typename T, int LPK, int R>
__global__ void __launch_bounds__(kWaves * 64, R == 4 ? (sizeof(T) == 2 ? 3 : 2) : R == 2 && sizeof(T) == 4 ? 3 : 4) attend_kernel(Attend a) {
    constexpr bool kAhead = R == 1 && sizeof(T) == 2;
    constexpr int KPW = 64 / LPK, STEP = kWaves * KPW * kUnroll;
    __shared__ const T* keys[kTable];
    __shared__ const T* values[kTable];
    __shared__ float part[kWaves][R][LPK * kE + 2];
    const Cache& c = a.c;
    const int G = c.N_h / c.N_kv;
    const int split = blockIdx.x, chunk = (int)a.by_kv(blockIdx.y), j = blockIdx.y - chunk * c.N_kv, b = blockIdx.z;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, sub = lane % LPK, grp = lane / LPK;
    const int r0 = chunk * R, n_new = new_tokens(c, b);
    const int rows = min(R, n_new * G - r0);
    if (rows <= 0) return;
    const int start = c.start[b];
    const Divide by_G = a.by_G;
    const Range g = range_of(a, start, (int)by_G((uint32_t)r0), (int)by_G((uint32_t)(r0 + rows - 1)), STEP);
    const bool alone = g.per >= g.hi - g.lo;           // one split holds all keys
    if (split > 0 && (int64_t)split * g.per >= g.hi - g.lo) return;
    const int lo = g.lo + split * g.per, hi = lo + min(g.per, g.hi - lo);
    if (lo >= hi && !(alone && split == 0)) return;

    // the pages' addresses, kTable at a time
    int first_page = 0, k1 = lo;
    bool gone = false;                                 // a page is not there
    auto look_up = [&](int k0) {
        first_page = (int)c.by_P((uint32_t)k0);
        k1 = (int)min((int64_t)hi, (first_page + kTable) * (int64_t)c.P);
        const int n_here = (int)(c.by_P((uint32_t)(k1 - 1)) - first_page) + 1;
        __syncthreads();
        bool missing = false;
        for (int i = tid; i < n_here; i += kWaves * 64) {
            const int page = c.pages[(int64_t)b * c.max_pages + first_page + i];
            const bool ok = page >= 0 && page < c.n_pages;
            const int64_t off = (int64_t)j * c.P * c.h;
            keys[i] = ok ? global_as<const T>(c.K[page]) + off : nullptr;
            values[i] = ok ? global_as<const T>(c.V[page]) + off : nullptr;
            missing = missing || !ok;
        }
        gone = __syncthreads_or(missing);
    };
    if (lo < hi) look_up(lo);

    const bool live = sub * kE < c.h;
    float q[R][kE], acc[R][kE], mx[R], sum[R];
    int upto[R], from[R], at_pos[R];                   // positions that a row sees, its own (where it has none: a valid one)
    const T* at_row[R];
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int row = r0 + min(r, rows - 1), s = (int)by_G((uint32_t)row);
        const int64_t p = (int64_t)start + s;
        const bool there = r < rows && p >= 0 && (!c.rot || p < c.rot_n);
        upto[r] = there ? clamped(p) : -1;
        from[r] = c.window > 0 ? clamped(p - c.window) : -1;
        at_pos[r] = (int)max((int64_t)0, min(p, (int64_t)c.rot_n - 1));
        at_row[r] = row_at<const T>(c.z, (j * G + row - s * G) * c.h, s, b);
    }
    turned<T, R>(c, at_row, live ? sub * kE : 0, at_pos, q);
#pragma unroll
    for (int r = 0; r < R; r++) {
        mx[r] = kNegInf;
        sum[r] = 0.f;
#pragma unroll
        for (int i = 0; i < kE; i++) {
            q[r][i] = live && upto[r] >= 0 ? q[r][i] * a.scale : 0.f;
            acc[r][i] = 0.f;
        }
    }

    int least_upto = INT32_MAX, most_from = -1;
#pragma unroll
    for (int r = 0; r < R; r++)
        if (r < rows) {
            least_upto = min(least_upto, upto[r]);
            most_from = max(most_from, from[r]);
        }
    for (int k0 = lo; k0 < hi;) {
        if (k0 > lo) look_up(k0);
        // A step's keys and values; with one row of bf16, the next step's are on their way while this one's are worked on (64 sequences of up to 4096 90 -> 84 us;
        // elsewhere the registers would cost wavefronts: four rows of 131072 keys 115 -> 126).
        struct Step {
            Eight<T> kk[kUnroll], vv[kUnroll];
            int pos[kUnroll];
        };
        auto fetch = [&](int k, Step& st) {
#pragma unroll
            for (int u = 0; u < kUnroll; u++) {
                const int p = k + (u * kWaves + wv) * KPW + grp;
                st.kk[u].zero();
                st.vv[u].zero();
                st.pos[u] = -1;
                if (p < k1) {
                    const uint32_t pg = c.by_P((uint32_t)p), slot = (uint32_t)p - pg * c.P;
                    const T* kp = keys[pg - (uint32_t)first_page];
                    if (kp) {
                        st.pos[u] = p;
                        if (live) {
                            const uint32_t at = slot * (uint32_t)c.h + sub * kE;
                            st.kk[u].load(in_global(kp) + at);
                            st.vv[u].load(in_global(values[pg - (uint32_t)first_page]) + at);
                        }
                    }
                }
            }
        };
        Step now, ahead;
        if (kAhead) fetch(k0, ahead);
        for (int k = k0; k < k1; k += STEP) {
            if (kAhead) {
                now = ahead;
                if (k + STEP < k1) fetch(k + STEP, ahead);
            } else {
                fetch(k, now);
            }
            const auto& kk = now.kk;
            const auto& vv = now.vv;
            const auto& pos = now.pos;
            // Every row sees every key of the step: nothing to mask.  (Four rows: both forms together take more registers than three wavefronts have, 148 -> 155 us.)
            const bool plain = R < 4 && !gone && k + STEP <= k1 && k + STEP - 1 <= least_upto && k > most_from;
            float score[kUnroll][R];
#pragma unroll
            for (int u = 0; u < kUnroll; u++) {
                float f[kE];
                kk[u].get(f);
#pragma unroll
                for (int r = 0; r < R; r++) {
                    float d = 0.f;
#pragma unroll
                    for (int i = 0; i < kE; i++) d = fmaf(f[i], q[r][i], d);
                    d = lanes_sum<LPK>(d);
                    score[u][r] = d;
                }
            }
            if (!plain) {
#pragma unroll
                for (int u = 0; u < kUnroll; u++)
#pragma unroll
                    for (int r = 0; r < R; r++) score[u][r] = pos[u] >= 0 && pos[u] <= upto[r] && pos[u] > from[r] ? score[u][r] : kNegInf;
            }
#pragma unroll
            for (int r = 0; r < R; r++) {
                float m = mx[r];
#pragma unroll
                for (int u = 0; u < kUnroll; u++) m = fmaxf(m, score[u][r]);
                const float base = m == kNegInf ? 0.f : m;
                const float fall = exp2f(mx[r] - base);
                mx[r] = m;
                sum[r] *= fall;
#pragma unroll
                for (int i = 0; i < kE; i++) acc[r][i] *= fall;
#pragma unroll
                for (int u = 0; u < kUnroll; u++) {
                    score[u][r] = exp2f(score[u][r] - base);
                    sum[r] += score[u][r];
                }
            }
#pragma unroll
            for (int u = 0; u < kUnroll; u++) {
                float f[kE];
                vv[u].get(f);
                if (plain) {
#pragma unroll
                    for (int r = 0; r < R; r++)
#pragma unroll
                        for (int i = 0; i < kE; i++) acc[r][i] = fmaf(score[u][r], f[i], acc[r][i]);
                } else {
                    // (a weight of zero is no mask in front of an infinity)
#pragma unroll
                    for (int r = 0; r < R; r++) {
                        const bool sees = pos[u] >= 0 && pos[u] <= upto[r] && pos[u] > from[r];
#pragma unroll
                        for (int i = 0; i < kE; i++) acc[r][i] = sees ? fmaf(score[u][r], f[i], acc[r][i]) : acc[r][i];
                    }
                }
            }
        }
        k0 = k1;
    }

    // the lane groups of a wavefront meet, then the wavefronts
#pragma unroll
    for (int r = 0; r < R; r++) {
#pragma unroll
        for (int o = LPK; o < 64; o <<= 1) {
            const float m2 = __shfl_xor(mx[r], o, 64), m = fmaxf(mx[r], m2), base = m == kNegInf ? 0.f : m;
            const float f1 = exp2f(mx[r] - base), f2 = exp2f(m2 - base);
            sum[r] = sum[r] * f1 + __shfl_xor(sum[r], o, 64) * f2;
#pragma unroll
            for (int i = 0; i < kE; i++) acc[r][i] = acc[r][i] * f1 + __shfl_xor(acc[r][i], o, 64) * f2;
            mx[r] = m;
        }
        if (grp == 0) {
#pragma unroll
            for (int i = 0; i < kE; i++) part[wv][r][sub * kE + i] = acc[r][i];
            if (sub == 0) {
                part[wv][r][LPK * kE] = mx[r];
                part[wv][r][LPK * kE + 1] = sum[r];
            }
        }
    }
    __syncthreads();
    for (int r = wv; r < rows; r += kWaves) {
        float m = kNegInf;
#pragma unroll
        for (int w = 0; w < kWaves; w++) m = fmaxf(m, part[w][r][LPK * kE]);
        const float base = m == kNegInf ? 0.f : m;
        float f[kWaves], s = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; w++) {
            f[w] = exp2f(part[w][r][LPK * kE] - base);
            s += f[w] * part[w][r][LPK * kE + 1];
        }
        const int tok = (int)by_G((uint32_t)(r0 + r)), head = j * G + r0 + r - tok * G;
        if (grp == 0 && live) {
            float x[kE];
#pragma unroll
            for (int i = 0; i < kE; i++) {
                x[i] = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; w++) x[i] += f[w] * part[w][r][sub * kE + i];
            }
            if (alone) {
#pragma unroll
                for (int i = 0; i < kE; i++) x[i] = s == 0.f ? 0.f : x[i] / s;
                put(row_at<T>(a.out, head * c.h, tok, b) + sub * kE, x);
            } else {
                float* o = a.partial + ((((int64_t)b * c.z.n1 + tok) * c.N_h + head) * a.splits + split) * (c.h + 2);
#pragma unroll
                for (int i = 0; i < kE; i++) o[sub * kE + i] = x[i];
                if (sub == 0) {
                    o[c.h] = m;
                    o[c.h + 1] = s;
                }
            }
        }
    }
}

// ---------------------------------------------------------------- many rows: on the matrix cores
// The workgroup owns 128 rows, 32 to a wavefront, and streams blocks of 64 keys and values through LDS, the next one on its way to registers while the
// products run.  Products and statistics as in the fused attention: scores are a 32 x 32 accumulator, lane = row, whose layout is that of the
// operand of the product with the values.
//   A turned query and the weights have more bits than bf16: each is kept in two bf16 parts, and the scores (of turned queries) and the results are two products.
//   So what a row gets is as near to fp32 weights as on the vector units, and only the result is rounded to bf16 (2^-16 of a weight is lost, half a step of bf16 is 2^-8).
//   Masked weights are zeros, but a zero times an infinity is none: in blocks that some row sees in part, values that are no numbers are
//   taken out (`odd`), and given afterwards to the rows that see them.
// A wavefront without rows only brings keys and values: with few rows, bound by memory, it still beats the vector units (cut_of says where).
constexpr int kTileTable = 256;
template <class X>
struct TileShape {
    static constexpr int kKeys = 64;                          // keys of a block
    static constexpr int kRowVecs = X::H / X::kPer;
    static constexpr int kVec = kKeys * kRowVecs / 256;       // vectors of a thread, of the keys and of the values
    static constexpr int kRows = 128;
    // workgroups of a unit, by registers: what is on its way to them decides
    static constexpr int kResident = sizeof(typename X::T) == 4 ? (X::H == 128 ? 1 : 2) : X::H == 128 ? 2 : 3;
};

// this lane's row, as the products take it; its second part where it is turned
template <class X>
__device__ __forceinline__ void load_query(const Cache& c, int h, const typename X::T* row, int hh, int p, bool there, typename X::Own& q, typename X::Own& rest) {
    if constexpr (sizeof(typename X::T) == 4) {
#pragma unroll
        for (int s = 0; s < X::H / 16; s++) {
            float x[kE] = {};
            if (there && (X::H / 2) * hh + 8 * s < h) turned<float>(c, row, (X::H / 2) * hh + 8 * s, p, x);
#pragma unroll
            for (int i = 0; i < kE; i++) q.v[8 * s + i] = x[i];
        }
    } else {
#pragma unroll
        for (int s = 0; s < X::H / 16; s++) {
            float x[kE] = {};
            if (there && 16 * s + 8 * hh < h) turned<bf16_t>(c, row, 16 * s + 8 * hh, p, x);
#pragma unroll
            for (int i = 0; i < kE; i++) {
                q.v[s][i] = (__bf16)x[i];
                rest.v[s][i] = (__bf16)(x[i] - (float)q.v[s][i]);
            }
        }
    }
}

__device__ __forceinline__ bool no_number(uint32_t b) { return (b & 0x7f800000u) == 0x7f800000u; }

// the elements of a vector that are no numbers, as zeros; whether there was one
__device__ __forceinline__ bool take_out(float4& v) {
    float* f = &v.x;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const bool bad = no_number(__float_as_uint(f[i]));
        f[i] = bad ? 0.f : f[i];
        odd = odd || bad;
    }
    return odd;
}
__device__ __forceinline__ bool take_out(uint4& v) {
    uint32_t* w = &v.x;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const bool lo = no_number(w[i] << 16), hi = no_number(w[i] & 0xffff0000u);
        w[i] &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
        odd = odd || lo || hi;
    }
    return odd;
}

// TURN: queries are turned.  FULL: heads of H components; else of fewer, zeros behind them.
template <class X, bool TURN, bool FULL>
__global__ void __launch_bounds__(256, TileShape<X>::kResident) attend_tile_kernel(Attend a) {
    using T = typename X::T;
    using S = TileShape<X>;
    constexpr int H = X::H, LDK = X::LD, LDV = X::LD_COLS, KEYS = S::kKeys;
    __shared__ __attribute__((aligned(16))) char lds[KEYS * (LDK + LDV) * sizeof(T)];
    __shared__ const T* keys[kTileTable];
    __shared__ const T* values[kTileTable];
    __shared__ int odd_block;
    T* const Ks = reinterpret_cast<T*>(lds);
    T* const Vs = Ks + KEYS * LDK;
    const Cache& c = a.c;
    const int G = c.N_h / c.N_kv, h = FULL ? H : c.h;
    const int split = blockIdx.x, j = blockIdx.y % c.N_kv, b = blockIdx.z;
    // the last rows see the most keys: they go first
    const int chunk = a.chunks - 1 - (int)blockIdx.y / c.N_kv;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, hh = lane >> 5, ln = lane & 31;
    const int r0 = chunk * S::kRows, n_new = new_tokens(c, b);
    const int rows = min(S::kRows, n_new * G - r0);
    if (rows <= 0) return;
    const int start = c.start[b];
    const Range g = range_of(a, start, r0 / G, (r0 + rows - 1) / G, KEYS);
    const bool alone = g.per >= g.hi - g.lo;
    if (split > 0 && (int64_t)split * g.per >= g.hi - g.lo) return;
    const int lo = g.lo + split * g.per, hi = lo + min(g.per, g.hi - lo);
    if (lo >= hi && !(alone && split == 0)) return;

    // this lane's row, and what this wavefront's rows see at least and at most
    const int first = 32 * w, own = first + ln;
    const int tok = (r0 + own) / G, head = j * G + (r0 + own) % G;
    const int64_t pos = (int64_t)start + tok;
    const bool there = own < rows && pos >= 0 && (!c.rot || pos < c.rot_n);
    const int upto = there ? clamped(pos) : -1, from = c.window > 0 ? clamped(pos - c.window) : -1;
    // (clamped too: a first position below 0 sees nothing, and then nothing is seen by all)
    const int w_first = clamped((int64_t)start + (r0 + first) / G), w_last = clamped((int64_t)start + (r0 + min(first + 31, rows - 1)) / G);
    const bool w_any = first < rows;
    typename X::Own q, rest;
    load_query<X>(c, h, there ? row_at<const T>(c.z, head * h, tok, b) : nullptr, hh, (int)pos, there, q, rest);

    f32x16 O[H / 32];
#pragma unroll
    for (int rb = 0; rb < H / 32; rb++) O[rb] = zero16();
    float m = kNegInf, lsum = 0.f;

    for (int k0 = lo; k0 < hi;) {
        // the pages' addresses, kTileTable at a time
        const int first_page = (int)c.by_P((uint32_t)k0);
        const int k1 = (int)min((int64_t)hi, (first_page + kTileTable) * (int64_t)c.P);
        const int n_here = (int)c.by_P((uint32_t)(k1 - 1)) - first_page + 1;
        __syncthreads();
        bool gone = false;
        for (int i = tid; i < n_here; i += 256) {
            const int page = c.pages[(int64_t)b * c.max_pages + first_page + i];
            const bool ok = page >= 0 && page < c.n_pages;
            const int64_t off = (int64_t)j * c.P * h;
            keys[i] = ok ? global_as<const T>(c.K[page]) + off : nullptr;
            values[i] = ok ? global_as<const T>(c.V[page]) + off : nullptr;
            gone = gone || !ok;
        }
        const bool all_there = !__syncthreads_or(gone);

        // block [k, k + KEYS) into registers, zeros beyond k1 and where no page is
        typename X::Vec kr[S::kVec], vr[S::kVec];
        auto fetch = [&](int k) {
#pragma unroll
            for (int i = 0; i < S::kVec; i++) {
                const int idx = tid + 256 * i, row = idx / S::kRowVecs, cv = idx % S::kRowVecs;
                kr[i] = vr[i] = X::zero_vec();
                if (k + row < k1) {
                    const uint32_t p = (uint32_t)(k + row), pg = c.by_P(p), slot = p - pg * c.P, at = pg - (uint32_t)first_page;
                    if (const T* kp = keys[at]) {
                        const uint32_t off = slot * (uint32_t)h + (FULL ? cv * X::kPer : min(cv * X::kPer, h - X::kPer));
                        kr[i] = *reinterpret_cast<const typename X::Vec*>(in_global(kp) + off);
                        vr[i] = *reinterpret_cast<const typename X::Vec*>(in_global(values[at]) + off);
                    }
                }
            }
        };
        // whether every row of the workgroup sees all of the block
        const int wg_first = clamped((int64_t)start + r0 / G), wg_last = clamped((int64_t)start + (r0 + rows - 1) / G);
        auto whole = [&](int k) { return k + KEYS - 1 <= wg_first && (c.window == 0 || k > wg_last - c.window); };
        auto stash = [&](int k) {
            const bool clean = !whole(k);
            bool odd = false;
#pragma unroll
            for (int i = 0; i < S::kVec; i++) {
                const int idx = tid + 256 * i, row = idx / S::kRowVecs, cv = idx % S::kRowVecs;
                if (clean && take_out(vr[i])) odd = true;
                if (!FULL && cv * X::kPer >= h) kr[i] = X::zero_vec();
                X::template put<LDK>(Ks, row, cv, kr[i]);
                X::template put<LDV>(Vs, row, cv, vr[i]);
            }
            if (odd) odd_block = 1;
        };
        // pages begin on large powers of two, and workgroups that walk theirs in step would all ask the same memory channels: each begins elsewhere
        const int blocks = (int)((k1 - k0 + KEYS - 1) / KEYS), turn = (int)((5u * split + 3u * j) % (uint32_t)blocks);
        auto block = [&](int i) { return k0 + KEYS * (i + turn < blocks ? i + turn : i + turn - blocks); };
        fetch(block(0));
        if (tid == 0) odd_block = 0;
        __syncthreads();
        stash(block(0));
        __syncthreads();
        for (int i = 0; i < blocks; i++) {
            const int k = block(i);
            const bool more = i + 1 < blocks;
            if (more) fetch(block(i + 1));
            const bool odd = odd_block != 0;
#pragma unroll
            for (int part = 0; part < 2; part++) {
                const int kb = k + 32 * part;
                if (!w_any || kb >= k1 || kb > w_last || (c.window > 0 && kb + 31 <= w_first - c.window)) continue;
                f32x16 s = X::template rows_times_own<LDK>(Ks, part, ln, hh, q);
                if constexpr (sizeof(T) == 2 && TURN) s = X::template rows_times_own<LDK>(Ks, part, ln, hh, rest, s);
                uint32_t seen = 0xffffu;
                if (!(all_there && kb + 32 <= k1 && kb + 31 <= w_first && (c.window == 0 || kb > w_last - c.window))) {
                    const int end = min(upto + 1, k1);
                    seen = 0;
#pragma unroll
                    for (int r = 0; r < 16; r++) {
                        const int kk = kb + acc_row(r, hh);
                        bool sees = kk < end && kk > from;
                        if (!all_there && sees) sees = keys[c.by_P((uint32_t)kk) - (uint32_t)first_page] != nullptr;
                        seen |= sees ? 1u << r : 0u;
                        s[r] = sees ? s[r] : kNegInf;
                    }
                }
                float mx = kNegInf;
#pragma unroll
                for (int r = 0; r < 16; r++) mx = fmaxf(mx, s[r]);
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                const float m_new = fmaxf(m, mx);
                const float shift = m_new == kNegInf ? 0.f : m_new * a.scale;
                const float alpha = m == m_new ? 1.f : __builtin_amdgcn_exp2f(m * a.scale - shift);
                m = m_new;
                float rowsum = 0.f;
#pragma unroll
                for (int r = 0; r < 16; r++) {
                    s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale, -shift));
                    rowsum += s[r];
                }
                lsum = lsum * alpha + rowsum;
                if (__any(alpha != 1.f)) {
#pragma unroll
                    for (int rb = 0; rb < H / 32; rb++)
#pragma unroll
                        for (int r = 0; r < 16; r++) O[rb][r] *= alpha;
                }
                typename X::Packed pk;
                X::pack(s, pk);
                if constexpr (sizeof(T) == 2) {
                    typename X::Packed low;
                    X::pack_rest(s, pk, low);
                    X::template cols_times_acc<LDV>(O, Vs, part, lane, pk, &low);
                } else {
                    X::template cols_times_acc<LDV>(O, Vs, part, lane, pk);
                }
                if (odd) {
                    // the values that were taken out, to the rows that see their keys
#pragma unroll 1
                    for (int kk = 0; kk < 32; kk++) {
                        const int p = kb + kk;
                        const T* vp = p < k1 ? values[c.by_P((uint32_t)p) - (uint32_t)first_page] : nullptr;
                        if (!vp) continue;
                        const T* v = in_global(vp) + (int64_t)((uint32_t)p - c.by_P((uint32_t)p) * c.P) * h;
                        // the weight of key kk lies in the half that acc_row puts it in
                        const int r = 4 * (kk / 8) + kk % 4, half = (kk / 4) % 2;
                        float wt = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; i++) wt = i == r ? s[i] : wt;
                        uint32_t bits = (seen >> r) & 1u;
                        const float wt2 = __shfl_xor(wt, 32, 64);
                        const uint32_t bits2 = (uint32_t)__shfl_xor((int)bits, 32, 64);
                        wt = hh == half ? wt : wt2;
                        bits = hh == half ? bits : bits2;
#pragma unroll
                        for (int rb = 0; rb < H / 32; rb++)
#pragma unroll
                            for (int i = 0; i < 16; i++) {
                                float x[1];
                                const bool in = FULL || 32 * rb + 8 * (i / 4) < h;   // (eights of components are there or not)
                                ldv<1>(v + (in ? 32 * rb + 8 * (i / 4) : 0) + (4 * hh + i % 4), x);
                                if (in && bits && no_number(__float_as_uint(x[0]))) O[rb][i] += wt * x[0];
                            }
                    }
                }
            }
            __syncthreads();
            if (more) {
                if (tid == 0) odd_block = 0;
                __syncthreads();
                stash(block(i + 1));
            }
            __syncthreads();
        }
        k0 = k1;
    }
    lsum += __shfl_xor(lsum, 32, 64);
    if (!there) {                                             // (a row without a query: it has added up what there was)
        m = kNegInf;
        lsum = 0.f;
#pragma unroll
        for (int rb = 0; rb < H / 32; rb++) O[rb] = zero16();
    }
    if (own >= rows) return;
    if (alone) {
        const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
        T* o = row_at<T>(a.out, head * h, tok, b);
#pragma unroll
        for (int rb = 0; rb < H / 32; rb++)
#pragma unroll
            for (int k = 0; k < 4; k++)
                if (FULL || 32 * rb + 8 * k < h) X::store4(o + 32 * rb + 8 * k + 4 * hh, O[rb][4 * k] * inv, O[rb][4 * k + 1] * inv, O[rb][4 * k + 2] * inv, O[rb][4 * k + 3] * inv);
    } else {
        float* o = a.partial + ((((int64_t)b * c.z.n1 + tok) * c.N_h + head) * a.splits + split) * (h + 2);
#pragma unroll
        for (int rb = 0; rb < H / 32; rb++)
#pragma unroll
            for (int i = 0; i < 16; i++)
                if (FULL || 32 * rb + 8 * (i / 4) < h) o[32 * rb + acc_row(i, hh)] = O[rb][i];
        if (hh == 0) {
            o[h] = m * a.scale;
            o[h + 1] = lsum;
        }
    }
}

// The splits of a row meet.  kSpread: a workgroup per row, its four wavefronts take a quarter of the splits each; else a wavefront per row (many rows of few
// splits).  `R`, `step`: how the rows and keys were cut.
template <typename T, bool kSpread>
__global__ void __launch_bounds__(256) join_kernel(Attend a, int R, int step) {
    __shared__ float part[4][256];
    constexpr int D = kSpread ? 4 : 1;
    const Cache& c = a.c;
    const int G = c.N_h / c.N_kv, tid = threadIdx.x, lane = tid & 63, w = tid >> 6, first = kSpread ? w : 0;
    const int row = kSpread ? (int)blockIdx.x : 4 * (int)blockIdx.x + w;       // (token, head) of sequence blockIdx.y
    const int head = row % c.N_h, tok = row / c.N_h, b = blockIdx.y;
    const int n_new = new_tokens(c, b);
    if (tok >= n_new) return;
    const int r0 = (tok * G + head % G) / R * R, rows = min(R, n_new * G - r0);
    const Range g = range_of(a, c.start[b], r0 / G, (r0 + rows - 1) / G, (uint32_t)step);
    if (g.per >= g.hi - g.lo) return;                  // nothing to join
    const int n = (int)((uint32_t)(g.hi - g.lo + g.per - 1) / (uint32_t)g.per), pitch = c.h + 2;
    const float* p = a.partial + (((int64_t)b * c.z.n1 + tok) * c.N_h + head) * a.splits * pitch;
    // a lane knows the maxima and sums of two splits
    static_assert(kMostSplits <= 128, "two to a lane");
    const int l2 = lane + 64;
    const float m1 = lane < n ? p[lane * pitch + c.h] : kNegInf, m2 = l2 < n ? p[l2 * pitch + c.h] : kNegInf;
    const float s1 = lane < n ? p[lane * pitch + c.h + 1] : 0.f, s2 = l2 < n ? p[l2 * pitch + c.h + 1] : 0.f;
    const float m = wave_max(fmaxf(m1, m2)), base = m == kNegInf ? 0.f : m;
    const float f1 = exp2f(m1 - base), f2 = exp2f(m2 - base);
    const float s = wave_sum(f1 * s1 + f2 * s2);
    T* o = row_at<T>(a.out, head * c.h, tok, b);
    for (int i0 = 0; i0 < c.h; i0 += 64) {
        const int i = min(i0 + lane, c.h - 1);
        float x = 0.f;
        for (int k0 = first; k0 < n; k0 += 8 * D) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; k++) v[k] = p[min(k0 + D * k, n - 1) * pitch + i];
#pragma unroll
            for (int k = 0; k < 8; k++) {
                const int at = k0 + D * k;
                x += at < n ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(at < 64 ? f1 : f2), at & 63)) * v[k] : 0.f;
            }
        }
        if constexpr (kSpread) {
            part[w][i0 + lane] = x;
        } else if (i0 + lane < c.h) {
            const float y[1] = {s == 0.f ? 0.f : x / s};
            stv<1>(o + i, y);
        }
    }
    if constexpr (kSpread) {
        __syncthreads();
        if (tid < c.h) {
            const float y[1] = {s == 0.f ? 0.f : (part[0][tid] + part[1][tid] + part[2][tid] + part[3][tid]) / s};
            stv<1>(o + tid, y);
        }
    }
}

// ---------------------------------------------------------------- host side
int32_t launched() { return hipGetLastError() == hipSuccess ? (int32_t)NNT_OK : (int32_t)NNT_EHIP; }

#define TRY(x)                           \
    do {                                 \
        int32_t rc__ = (x);              \
        if (rc__ != NNT_OK) return rc__; \
    } while (0)


Divide divide_by(uint32_t d) {
    // (n < 2^31: with 2^(k - 1) < d <= 2^k the product with ceil(2^(31 + k) / d) is exact enough)
    uint32_t k = 0;
    while ((1ull << k) < d) k++;
    return Divide{(uint32_t)(((1ull << (31 + k)) + d - 1) / d), k - 1, d};
}

Rows rows_of(const nnt_tensor* t) {
    const TiledView v = t->view();
    return Rows{v.tiles, v.shape[0], v.shape[1], v.shape[2], v.base[0], v.base[1], v.base[2], v.grid[0], v.grid[1],
                divide_by((uint32_t)v.base[0]), divide_by((uint32_t)v.base[1]), divide_by((uint32_t)v.base[2])};
}

Cache cache_of(const nnt_cache_cfg* cfg, nnt_tensor* QKV, nnt_tensor* K, nnt_tensor* V) {
    Cache c{};
    c.z = rows_of(QKV);
    c.K = K->d_tiles;
    c.V = V->d_tiles;
    c.pages = cfg->pages;
    c.start = cfg->start;
    c.count = cfg->count;
    if (nnt_tensor* r = cfg->rotation) {
        c.rot = reinterpret_cast<const float* const*>(r->d_tiles);
        c.rot_r = (int32_t)r->shape[0];
        c.rot_n = (int32_t)r->shape[1];
        c.rot_base = (int32_t)r->base[1];
        c.rot_pairs = cfg->rotate == NNT_ROTATE_PAIRS;
        c.rot_whole = c.rot_r % 16 == 0;
        c.by_rot = divide_by((uint32_t)c.rot_base);
    }
    c.h = (int32_t)K->shape[0];
    c.N_h = cfg->N_h;
    c.N_kv = cfg->N_kv;
    c.P = (int32_t)K->base[1];
    c.n_pages = (int32_t)K->ntiles;
    c.max_pages = cfg->max_pages;
    c.window = cfg->window;
    c.by_P = divide_by((uint32_t)c.P);
    return c;
}

// How the rows (queries that share a cached head of a sequence) and keys of a call are cut.
struct Cut {
    int R, lpk, step, chunks, splits;
    bool tile;
};
// Heads of up to 128 components: the matrix cores take three rows or more of bf16 (five where heads of more than 64 are turned, which is a second product for the scores) and 17 of fp32, where zeros fill
// heads up to 64 or 128 five and 33.  Passes of two states one after the other, in us, vector units -> matrix cores:
//   one sequence of 131072 keys of 8 cached heads of 128 and 64 sequences of 2048 of 12 of 64:
//   bf16, 2 rows 97 -> 99 and 67 -> 69, 4 rows 105 -> 99 and 86 -> 70, turned 107 -> 117 and 88 -> 80, 5 rows turned 194 -> 117 and 138 -> 81, 16 rows 387 -> 103 and 252 -> 74;  fp32, 16 rows 660 -> 660 and 321 -> 366, 32 rows 922 -> 660 and 567 -> 368;
//   waited for, turned, 4 rows: 131072 keys 148 -> 138, 8 sequences of 16384 of 8 heads of 128 123 -> 132;
//   filled up, 64 sequences, heads of 96 (4 cached ones, 1500 keys) and of 32 (8, 2048): bf16, 5 rows 63 -> 47 and 45 -> 49, 8 rows 65 -> 47 and 47 -> 49, 32 rows 234 -> 50 and 175 -> 50;
//   12 cached ones, fp32, 16 rows 416 -> 762 and 184 -> 384, 32 rows 779 -> 764 and 330 -> 385, 100 rows 2390 -> 838 and 926 -> 508.
Cut cut_of(const nnt_cache_cfg* cfg, const nnt_tensor* QKV, const nnt_tensor* K) {
    Cut u;
    const int64_t G = cfg->N_h / cfg->N_kv, rows = G * QKV->shape[1], N_b = QKV->shape[2];
    const int64_t h = K->shape[0];
    const bool bf16 = K->dtype == NNT_BF16;
    const bool full = h == 64 || h == 128;
    u.tile = h <= 128 && rows >= (bf16 ? (full && !(cfg->rotation && h > 64) ? 3 : 5) : full ? 17 : 33);
    u.R = u.tile ? 128 : rows >= 3 ? 4 : rows >= 2 ? 2 : 1;       // (three rows as two and one read the keys twice: fp32 heads of 96 255 -> 180)
    u.lpk = h <= 32 ? 4 : h <= 64 ? 8 : h <= 128 ? 16 : 32;
    u.step = u.tile ? 64 : kWaves * (64 / u.lpk) * kUnroll;
    u.chunks = (int)((rows + u.R - 1) / u.R);
    // The keys are split so that the launch fills the chip.  The matrix cores' kernel: with no more workgroups than it holds at a time (bf16, four rows of 131072 keys, 128 components:
    // 512 workgroups 100 us, 768 103, waited for 120 and 151); the vector units': eight to a unit, or four that keep more registers (four rows: 768 174 us, 1024 155).
    const int64_t pairs = (int64_t)u.chunks * cfg->N_kv * N_b;
    const int64_t held = 256 * (bf16 ? (h > 64 ? TileShape<Bf16Traits<128>>::kResident : TileShape<Bf16Traits<64>>::kResident)
                                     : (h > 64 ? TileShape<F32Traits<128>>::kResident : TileShape<F32Traits<64>>::kResident));
    const int64_t wanted = u.tile ? held / pairs : ((u.R == 1 ? 2048 : 1024) + pairs - 1) / pairs;
    // (no more than the longest range of keys has steps)
    const int64_t keys = std::min((int64_t)cfg->max_pages * K->base[1], cfg->window ? (int64_t)cfg->window + QKV->shape[1] : INT64_MAX);
    const int64_t most = (keys + u.step - 1) / u.step;
    u.splits = (int)std::max<int64_t>(1, std::min<int64_t>({wanted, most, kMostSplits}));
    return u;
}

using AppendFn = void (*)(Cache, Divide, Divide);
template <typename T>
AppendFn append_instance(bool halves, bool turn) { return !halves ? append_kernel<T> : turn ? append_halves_kernel<T, true> : append_halves_kernel<T, false>; }
using AttendFn = void (*)(Attend);
template <typename T, int LPK>
AttendFn attend_rows(int R) { return R == 1 ? attend_kernel<T, LPK, 1> : R == 2 ? attend_kernel<T, LPK, 2> : attend_kernel<T, LPK, 4>; }
template <typename T, int H>
AttendFn attend_tile(bool turn, bool full) {
    if constexpr (sizeof(T) == 4) return full ? attend_tile_kernel<F32Traits<H>, false, true> : attend_tile_kernel<F32Traits<H>, false, false>;
    else if (turn) return full ? attend_tile_kernel<Bf16Traits<H>, true, true> : attend_tile_kernel<Bf16Traits<H>, true, false>;
    else return full ? attend_tile_kernel<Bf16Traits<H>, false, true> : attend_tile_kernel<Bf16Traits<H>, false, false>;
}
template <typename T>
AttendFn attend_instance(const Cut& u, int64_t h, bool turn) {
    if (u.tile) return h <= 64 ? attend_tile<T, 64>(turn, h == 64) : attend_tile<T, 128>(turn, h == 128);
    return u.lpk == 4 ? attend_rows<T, 4>(u.R) : u.lpk == 8 ? attend_rows<T, 8>(u.R) : u.lpk == 16 ? attend_rows<T, 16>(u.R) : attend_rows<T, 32>(u.R);
}

}  // namespace

int32_t cache_check(nnt_ctx* ctx, const nnt_cache_cfg* cfg, nnt_tensor* QKV, nnt_tensor* K, nnt_tensor* V, nnt_tensor* B) {
    const std::string who = B ? "nnt_cache_attention" : "nnt_cache_append";
    if (!cfg || !QKV || !K || !V || !cfg->pages || !cfg->start) return fail(ctx, NNT_EINVAL, who + ": null argument");
    if (QKV->ctx != ctx || K->ctx != ctx || V->ctx != ctx || (B && B->ctx != ctx) || (cfg->rotation && cfg->rotation->ctx != ctx))
        return fail(ctx, NNT_EINVAL, who + ": tensor of another context");
    if (cfg->N_h < 1 || cfg->N_kv < 1 || cfg->N_h % cfg->N_kv || cfg->N_h > 65535 || cfg->max_pages < 1 || cfg->window < 0)
        return fail(ctx, NNT_EINVAL, who + ": bad configuration");
    if (K == V || K->ndim != 3 || K->dtype != V->dtype || !same_tiling(K, V)) return fail(ctx, NNT_EINVAL, who + ": K and V must be two tensors of one type, shape and tiling");
    const int64_t h = K->shape[0], P = K->base[1];
    if (h % kE || h > 256 || K->base[0] != h || K->shape[2] != cfg->N_kv || K->base[2] != cfg->N_kv || K->shape[1] % P)
        return fail(ctx, NNT_EINVAL, who + ": the cache must be [h, n_pages * P, N_kv] in tiles (h, P, N_kv), h a multiple of 8 and at most 256");
    if (K->shape[1] > INT32_MAX || (int64_t)cfg->max_pages * P > INT32_MAX - 65536 || P * h * cfg->N_kv > INT32_MAX) return fail(ctx, NNT_EINVAL, who + ": cache too long");
    if (QKV->dtype != K->dtype || (B && B->dtype != K->dtype)) return fail(ctx, NNT_EDTYPE, who + ": the cache has the activations' type");
    if (QKV->ndim != 3 || QKV->shape[0] != ((int64_t)cfg->N_h + 2 * (int64_t)cfg->N_kv) * h || QKV->base[0] % h)
        return fail(ctx, NNT_EINVAL, who + ": QKV must be [(N_h + 2 N_kv) * h, N_s, N_b], its row tiles whole heads");
    if (QKV->shape[1] > (1 << 24) || QKV->shape[2] > 65535) return fail(ctx, NNT_EINVAL, who + ": at most 2^24 tokens of 65535 sequences");
    if (B && (B->ndim != 3 || B->shape[0] != cfg->N_h * h || B->shape[1] != QKV->shape[1] || B->shape[2] != QKV->shape[2] || B->base[0] % h || B == QKV))
        return fail(ctx, NNT_EINVAL, who + ": the result must be [N_h * h, N_s, N_b], its row tiles whole heads");
    if (!QKV->whole_tiles || !K->whole_tiles || !V->whole_tiles || (B && !B->whole_tiles)) return fail(ctx, NNT_EINVAL, who + ": tiles must be present and 16-byte aligned");
    if (const nnt_tensor* r = cfg->rotation) {
        if (r->dtype != NNT_F32 || r->ndim != 2 || r->shape[0] % 2 || r->shape[0] > h || r->base[0] != r->shape[0] || r->shape[1] > INT32_MAX || !r->whole_tiles)
            return fail(ctx, NNT_EINVAL, who + ": the rotation must be fp32 [r, N_pos], r even and at most h, not cut along its first axis");
        if (cfg->rotate != NNT_ROTATE_HALVES && cfg->rotate != NNT_ROTATE_PAIRS) return fail(ctx, NNT_EINVAL, who + ": unknown pairs of the rotation");
    }
    if (!B) return NNT_OK;
    const Cut u = cut_of(cfg, QKV, K);
    if ((int64_t)u.chunks * cfg->N_kv > 65535) return fail(ctx, NNT_EINVAL, who + ": too many tokens of too many heads in one call");
    if (u.splits == 1) return NNT_OK;
    return ensure_stream_scratch(ctx, QKV->shape[1] * QKV->shape[2] * cfg->N_h * u.splits * (h + 2));
}

}  // namespace nnt

using namespace nnt;

int32_t nnt_cache_append(nnt_ctx* ctx, const nnt_cache_cfg* cfg, nnt_tensor* QKV, nnt_tensor* K, nnt_tensor* V) {
    return entry(ctx, [&]() -> int32_t {
        TRY(cache_check(ctx, cfg, QKV, K, V, nullptr));
        const Cache c = cache_of(cfg, QKV, K, V);
        const bool halves = c.h % (2 * kE) == 0 && (!c.rot || (c.rot_whole && !c.rot_pairs && c.rot_r == c.h));
        const int64_t per_head = c.h / kE / (halves ? 2 : 1), per_seq = per_head * c.N_kv * c.z.n1;
        if (per_seq > INT32_MAX - 256) return fail(ctx, NNT_EINVAL, "nnt_cache_append: too many tokens of too many heads in one call");
        const Divide by_token = divide_by((uint32_t)(per_head * c.N_kv)), by_head = divide_by((uint32_t)per_head);
        const dim3 grid((unsigned)((per_seq + 255) / 256), (unsigned)c.z.n2);
        const bool bf16 = K->dtype == NNT_BF16;
        std::vector<Access> acc{K->whole_access(kReadWrite), V->whole_access(kReadWrite), QKV->all(kRead)};
        if (cfg->rotation) acc.push_back(cfg->rotation->all(kRead));
        OpTag tag(ctx, "cache_append", 4.0 * (double)c.N_kv * c.h * c.z.n1 * c.z.n2 * (double)K->elem_size(), true);
        return submit(ctx, acc, [&](hipStream_t st) {
            hipLaunchKernelGGL(bf16 ? append_instance<bf16_t>(halves, c.rot) : append_instance<float>(halves, c.rot), grid, dim3(256), 0, st, c, by_token, by_head);
            return launched();
        });
    });
}

int32_t nnt_cache_attention(nnt_ctx* ctx, const nnt_cache_cfg* cfg, float scale, nnt_tensor* QKV, nnt_tensor* K, nnt_tensor* V, nnt_tensor* B) {
    return entry(ctx, [&]() -> int32_t {
        if (!B || B == K || B == V) return fail(ctx, NNT_EINVAL, "nnt_cache_attention: the result must be a tensor of its own");
        TRY(cache_check(ctx, cfg, QKV, K, V, B));
        if (!(scale > 0.f && scale < 1e30f)) return fail(ctx, NNT_EINVAL, "nnt_cache_attention: scale must be positive");
        const Cut u = cut_of(cfg, QKV, K);
        Attend a{};
        a.c = cache_of(cfg, QKV, K, V);
        a.out = rows_of(B);
        a.scale = scale * kLog2e;
        a.splits = u.splits;
        a.chunks = u.chunks;
        a.by_G = divide_by((uint32_t)(cfg->N_h / cfg->N_kv));
        a.by_kv = divide_by((uint32_t)cfg->N_kv);
        const bool bf16 = K->dtype == NNT_BF16;
        const AttendFn fn = bf16 ? attend_instance<bf16_t>(u, a.c.h, a.c.rot) : attend_instance<float>(u, a.c.h, a.c.rot);
        const dim3 grid((unsigned)u.splits, (unsigned)(u.chunks * a.c.N_kv), (unsigned)a.c.z.n2);
        const int64_t rows = (int64_t)a.c.z.n1 * a.c.z.n2 * a.c.N_h;
        std::vector<Access> acc{B->all(kReadWrite), QKV->all(kRead), K->whole_access(kRead), V->whole_access(kRead)};
        if (cfg->rotation) acc.push_back(cfg->rotation->all(kRead));
        // (the lengths are on the device: the work counted is that of the queries and results, and of caches that are full)
        OpTag tag(ctx, "cache_attention", (2.0 * (double)rows * a.c.h + 2.0 * (double)a.c.max_pages * a.c.P * a.c.N_kv * a.c.h * a.c.z.n2) * (double)K->elem_size(), true);
        return submit(ctx, acc, [&](hipStream_t st) -> int32_t {
            a.partial = stream_scratch_of(ctx);
            hipLaunchKernelGGL(fn, grid, dim3(kWaves * 64), 0, st, a);
            TRY(launched());
            if (u.splits == 1) return NNT_OK;
            const bool spread = u.splits > 8;
            const int64_t per_seq = (int64_t)a.c.z.n1 * a.c.N_h;
            const dim3 jg((unsigned)(spread ? per_seq : (per_seq + 3) / 4), (unsigned)a.c.z.n2);
            const auto join = bf16 ? (spread ? join_kernel<bf16_t, true> : join_kernel<bf16_t, false>) : (spread ? join_kernel<float, true> : join_kernel<float, false>);
            hipLaunchKernelGGL(join, jg, dim3(256), 0, st, a, u.R, u.step);
            return launched();
        }, u.splits == 1 ? 1 : 2);
    });
}
