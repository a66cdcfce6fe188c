// A paged cache of keys and values, and the attention of new tokens over it (rollouts of a trained model, token by token or a
// part of a prompt at a time).
//
//   append     K[page][:, slot, j] = rot_p k_j,  V[page][:, slot, j] = v_j         p = start + s, page = pages[p / P], slot = p % P
//   attention  B = sum_k V[k] P[k],  P = softmax_k(scale K[k] . rot_p q),  k <= p  (and > p - window)
//
// A page is a tile (h, P, N_kv) of the cache's tensors: what one cached head reads of it is contiguous.
#include "device_util.hpp"
#include "internal.hpp"

#include <algorithm>
#include <cmath>

namespace nnt {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr int kE = 8;                       // components per lane

// [rows, N_s, N_b] with the heads side by side along the first axis
struct Rows {
    void* const* tiles;
    int32_t n0, n1, n2, b0, b1, b2, g0, g1;
};
template <typename T>
__device__ __forceinline__ T* row_at(const Rows& r, int row, int s, int b) {
    const int t0 = row / r.b0, t1 = s / r.b1, t2 = b / r.b2;
    const int e0 = min(r.b0, r.n0 - t0 * r.b0), e1 = min(r.b1, r.n1 - t1 * r.b1);
    return global_as<T>(r.tiles[t0 + r.g0 * (t1 + r.g1 * t2)]) + (row - t0 * r.b0) + (int64_t)e0 * ((s - t1 * r.b1) + (int64_t)e1 * (b - t2 * r.b2));
}

// Division of numbers below 2^31 by a fixed one: q = (n * mul) >> 32 >> shift.
struct Divide {
    uint32_t mul, shift, d;
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return d == 1 ? n : __umulhi(n, mul) >> shift; }
};

struct Cache {
    Rows z;                                  // queries, keys, values of the new tokens
    void* const* K;
    void* const* V;
    const int32_t *pages, *start, *count;
    const float* const* rot;                 // tiles of the rotation, NULL: none
    int32_t rot_r, rot_n, rot_base, rot_pairs;
    int32_t h, N_h, N_kv, P, n_pages, max_pages, window;
    Divide by_P;
};

__device__ __forceinline__ int new_tokens(const Cache& c, int b) { return c.count ? min(max(c.count[b], 0), c.z.n1) : c.z.n1; }

// Components i0 .. i0 + 7 of a head's row, turned by the rotation of position p (0 <= p < rot_n).
template <typename T>
__device__ __forceinline__ void turned(const Cache& c, const T* row, int i0, int p, float (&x)[kE]) {
    if constexpr (sizeof(T) == 2) {
        ldv<8>(row + i0, x);
    } else {
        float lo[4], hi[4];
        ldv<4>(row + i0, lo);
        ldv<4>(row + i0 + 4, hi);
#pragma unroll
        for (int i = 0; i < 4; i++) { x[i] = lo[i]; x[i + 4] = hi[i]; }
    }
    if (!c.rot) return;
    const int half = c.rot_r / 2, t = p / c.rot_base;
    const float* cs = in_global(c.rot[t]) + (int64_t)(p - t * c.rot_base) * c.rot_r;
    if (c.rot_pairs) {
#pragma unroll
        for (int i = 0; i < kE; i += 2)
            if (i0 + i < c.rot_r) {
                const float co = cs[(i0 + i) / 2], si = cs[half + (i0 + i) / 2], a = x[i], b = x[i + 1];
                x[i] = a * co - b * si;
                x[i + 1] = a * si + b * co;
            }
    } else {
#pragma unroll
        for (int i = 0; i < kE; i++) {
            const int at = i0 + i;
            if (at >= c.rot_r) continue;
            const bool second = at >= half;
            const int k = second ? at - half : at;
            float other[1];
            ldv<1>(row + (second ? k : at + half), other);
            x[i] = second ? other[0] * cs[half + k] + x[i] * cs[k] : x[i] * cs[k] - other[0] * cs[half + k];
        }
    }
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

// A thread moves eight components of a key and of its value.
template <typename T>
__global__ void __launch_bounds__(256) append_kernel(Cache c) {
    const int per_head = c.h / kE, per_token = per_head * c.N_kv;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int b = blockIdx.y;
    if (at >= (int64_t)per_token * c.z.n1) return;
    const int s = (int)(at / per_token), k = (int)(at - (int64_t)s * per_token), j = k / per_head, i0 = (k - j * per_head) * kE;
    if (s >= new_tokens(c, b)) return;
    const int64_t p = (int64_t)c.start[b] + s;
    if (p < 0 || p >= (int64_t)c.max_pages * c.P || (c.rot && p >= c.rot_n)) return;
    const uint32_t q = c.by_P((uint32_t)p), slot = (uint32_t)p - q * c.P;
    const int page = c.pages[(int64_t)b * c.max_pages + q];
    if (page < 0 || page >= c.n_pages) return;
    const int64_t to = ((int64_t)j * c.P + slot) * c.h + i0;
    float x[kE];
    turned<T>(c, row_at<const T>(c.z, (c.N_h + j) * c.h, s, b), i0, (int)p, x);
    put(global_as<T>(c.K[page]) + to, x);
    // (values leave as they came, whatever their bits)
    const uint4* from = reinterpret_cast<const uint4*>(row_at<const T>(c.z, (c.N_h + c.N_kv + j) * c.h, s, b) + i0);
    uint4* v = reinterpret_cast<uint4*>(global_as<T>(c.V[page]) + to);
    v[0] = from[0];
    if constexpr (sizeof(T) == 4) v[1] = from[1];
}

// ---------------------------------------------------------------- attention
struct Attend {
    Cache c;
    Rows out;
    float scale;              // times log2(e): scores are exponents of two
    int32_t splits;           // workgroups that share the keys of a row, at most
    int32_t chunks;           // row chunks of a (sequence, cached head) pair
    float* partial;           // [row][split][h + 2]: result of a split (not divided), its maximum, its sum
};

constexpr int kWaves = 4;
constexpr int kUnroll = 4;    // keys a lane has on their way at a time
constexpr int kTable = 512;   // pages whose addresses a workgroup keeps at a time

// The keys of a row chunk's split: the positions [lo, hi), of which a split takes `per`.
struct Range {
    int64_t lo, hi, per;
};
// rows r0 .. r0 + R - 1 of a (sequence, cached head) pair: row r is token r / G, query head j G + r % G
__device__ __forceinline__ Range range_of(const Attend& a, int start, int s_first, int s_last, int step) {
    Range g;
    const int64_t end = (int64_t)a.c.max_pages * a.c.P;
    g.hi = min((int64_t)start + s_last + 1, end);
    g.lo = a.c.window > 0 ? max((int64_t)0, (int64_t)start + s_first + 1 - a.c.window) : 0;
    const int64_t n = max((int64_t)0, g.hi - g.lo);
    g.per = (n + a.splits - 1) / a.splits;
    g.per = max((int64_t)step, (g.per + step - 1) / step * step);
    return g;
}

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

// One workgroup: R rows of a (sequence, cached head) pair against one split of the keys.  LPK lanes share a key, eight components each; a wavefront
// takes 64 / LPK keys at a time, and every such group of lanes carries a running maximum and sum of its own, which meet at the end.
template <typename T, int LPK, int R>
__global__ void __launch_bounds__(kWaves * 64) attend_kernel(Attend a) {
    constexpr int KPW = 64 / LPK, STEP = kWaves * KPW * kUnroll;
    __shared__ const T* keys[kTable];
    __shared__ const T* values[kTable];
    __shared__ float part[kWaves][R][LPK * kE + 2];
    const Cache& c = a.c;
    const int G = c.N_h / c.N_kv;
    const int split = blockIdx.x, j = blockIdx.y % c.N_kv, chunk = blockIdx.y / c.N_kv, b = blockIdx.z;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, sub = lane % LPK, grp = lane / LPK;
    const int r0 = chunk * R, n_new = new_tokens(c, b);
    const int rows = min(R, n_new * G - r0);
    if (rows <= 0) return;
    const int start = c.start[b];
    const Range g = range_of(a, start, r0 / G, (r0 + rows - 1) / G, STEP);
    const int64_t lo = g.lo + split * g.per, hi = min(g.hi, lo + g.per);
    const bool alone = g.lo + g.per >= g.hi;           // one split holds all keys
    if (lo >= hi && !(alone && split == 0)) return;

    const bool live = sub * kE < c.h;
    float q[R][kE], acc[R][kE], mx[R], sum[R];
    int64_t upto[R], from[R];                          // positions that a row sees
#pragma unroll
    for (int r = 0; r < R; r++) {
        mx[r] = kNegInf;
        sum[r] = 0.f;
        const int s = (r0 + r) / G;
        const int64_t p = (int64_t)start + s;
        bool there = r < rows && p >= 0 && (!c.rot || p < c.rot_n);
        upto[r] = there ? p : -1;
        from[r] = c.window > 0 ? p - c.window : -1;
#pragma unroll
        for (int i = 0; i < kE; i++) q[r][i] = acc[r][i] = 0.f;
        if (there && live) {
            turned<T>(c, row_at<const T>(c.z, (j * G + (r0 + r) % G) * c.h, s, b), sub * kE, (int)p, q[r]);
#pragma unroll
            for (int i = 0; i < kE; i++) q[r][i] *= a.scale;
        }
    }

    // the pages' addresses, kTable at a time
    for (int64_t k0 = lo; k0 < hi;) {
        const int64_t first_page = k0 / c.P;
        const int64_t k1 = min(hi, (first_page + kTable) * (int64_t)c.P);
        const int n_here = (int)((k1 + c.P - 1) / c.P - first_page);
        __syncthreads();
        for (int i = tid; i < n_here; i += kWaves * 64) {
            const int page = c.pages[(int64_t)b * c.max_pages + first_page + i];
            const bool ok = page >= 0 && page < c.n_pages;
            const int64_t off = (int64_t)j * c.P * c.h;
            keys[i] = ok ? global_as<const T>(c.K[page]) + off : nullptr;
            values[i] = ok ? global_as<const T>(c.V[page]) + off : nullptr;
        }
        __syncthreads();
        for (int64_t k = k0; k < k1; k += STEP) {
            Eight<T> kk[kUnroll], vv[kUnroll];
            int pos[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; u++) {
                const int64_t p = k + (u * kWaves + wv) * KPW + grp;
                kk[u].zero();
                vv[u].zero();
                pos[u] = -1;
                if (p < k1) {
                    const uint32_t pg = c.by_P((uint32_t)p), slot = (uint32_t)p - pg * c.P;
                    const T* kp = keys[pg - (uint32_t)first_page];
                    if (kp) {
                        pos[u] = (int)p;
                        if (live) {
                            const int64_t at = (int64_t)slot * c.h + sub * kE;
                            kk[u].load(in_global(kp) + at);
                            vv[u].load(in_global(values[pg - (uint32_t)first_page]) + at);
                        }
                    }
                }
            }
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
#pragma unroll
                    for (int o = 1; o < LPK; o <<= 1) d += __shfl_xor(d, o, 64);
                    score[u][r] = pos[u] >= 0 && pos[u] <= upto[r] && pos[u] > from[r] ? d : kNegInf;
                }
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
#pragma unroll
                for (int r = 0; r < R; r++) {
                    const bool sees = pos[u] >= 0 && pos[u] <= upto[r] && pos[u] > from[r];
#pragma unroll
                    for (int i = 0; i < kE; i++) acc[r][i] = sees ? fmaf(score[u][r], f[i], acc[r][i]) : acc[r][i];
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
        const int tok = (r0 + r) / G, head = j * G + (r0 + r) % G;
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

// The splits of a row meet: one wavefront per row.  `R`, `step`: how the rows and keys were cut.
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(Attend a, int R, int step) {
    const Cache& c = a.c;
    const int G = c.N_h / c.N_kv, lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)c.z.n2 * c.z.n1 * c.N_h) return;
    const int head = (int)(row % c.N_h), tok = (int)(row / c.N_h % c.z.n1), b = (int)(row / c.N_h / c.z.n1);
    const int n_new = new_tokens(c, b);
    if (tok >= n_new) return;
    const int r0 = (tok * G + head % G) / R * R, rows = min(R, n_new * G - r0);
    const Range g = range_of(a, c.start[b], r0 / G, (r0 + rows - 1) / G, step);
    if (g.lo + g.per >= g.hi) return;                  // nothing to join
    const int n = (int)((g.hi - g.lo + g.per - 1) / g.per);
    const float* p = a.partial + row * a.splits * (c.h + 2);
    float m = kNegInf;
    for (int k = lane; k < n; k += 64) m = fmaxf(m, p[(int64_t)k * (c.h + 2) + c.h]);
    m = wave_max(m);
    const float base = m == kNegInf ? 0.f : m;
    float s = 0.f;
    for (int k = lane; k < n; k += 64) s += exp2f(p[(int64_t)k * (c.h + 2) + c.h] - base) * p[(int64_t)k * (c.h + 2) + c.h + 1];
    s = wave_sum(s);
    T* o = row_at<T>(a.out, head * c.h, tok, b);
    for (int i = lane; i < c.h; i += 64) {
        float x[1] = {0.f};
        for (int k = 0; k < n; k++) x[0] += exp2f(p[(int64_t)k * (c.h + 2) + c.h] - base) * p[(int64_t)k * (c.h + 2) + i];
        x[0] = s == 0.f ? 0.f : x[0] / s;
        stv<1>(o + i, x);
    }
}

// ---------------------------------------------------------------- host side
int32_t launched() { return hipGetLastError() == hipSuccess ? (int32_t)NNT_OK : (int32_t)NNT_EHIP; }

#define TRY(x)                           \
    do {                                 \
        int32_t rc__ = (x);              \
        if (rc__ != NNT_OK) return rc__; \
    } while (0)

constexpr int kMostSplits = 64;

Rows rows_of(const nnt_tensor* t) {
    const TiledView v = t->view();
    return Rows{v.tiles, v.shape[0], v.shape[1], v.shape[2], v.base[0], v.base[1], v.base[2], v.grid[0], v.grid[1]};
}

Divide divide_by(uint32_t d) {
    // (n < 2^31: with 2^(k - 1) < d <= 2^k the product with ceil(2^(31 + k) / d) is exact enough)
    uint32_t k = 0;
    while ((1ull << k) < d) k++;
    return Divide{(uint32_t)(((1ull << (31 + k)) + d - 1) / d), k - 1, d};
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

// How the rows and keys of a call are cut.
struct Cut {
    int R, lpk, step, chunks, splits;
};
Cut cut_of(const nnt_cache_cfg* cfg, const nnt_tensor* QKV, const nnt_tensor* K) {
    Cut u;
    const int64_t G = cfg->N_h / cfg->N_kv, rows = G * QKV->shape[1], N_b = QKV->shape[2];
    u.R = rows >= 4 ? 4 : rows >= 2 ? 2 : 1;
    const int64_t h = K->shape[0];
    u.lpk = h <= 32 ? 4 : h <= 64 ? 8 : h <= 128 ? 16 : 32;
    u.step = kWaves * (64 / u.lpk) * kUnroll;
    u.chunks = (int)((rows + u.R - 1) / u.R);
    // about eight workgroups to a compute unit
    const int64_t pairs = u.chunks * cfg->N_kv * N_b;
    const int64_t most = ((int64_t)cfg->max_pages * K->base[1] + u.step - 1) / u.step;
    u.splits = (int)std::max<int64_t>(1, std::min<int64_t>({(2048 + pairs - 1) / pairs, most, kMostSplits}));
    return u;
}

using AttendFn = void (*)(Attend);
template <typename T, int LPK>
AttendFn attend_rows(int R) { return R == 1 ? attend_kernel<T, LPK, 1> : R == 2 ? attend_kernel<T, LPK, 2> : attend_kernel<T, LPK, 4>; }
template <typename T>
AttendFn attend_instance(const Cut& u) {
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
        const int64_t per_seq = (int64_t)(c.h / kE) * c.N_kv * c.z.n1;
        const dim3 grid((unsigned)((per_seq + 255) / 256), (unsigned)c.z.n2);
        const bool bf16 = K->dtype == NNT_BF16;
        std::vector<Access> acc;
        K->whole_access(kReadWrite, &acc);
        V->whole_access(kReadWrite, &acc);
        acc.push_back(QKV->all(kRead));
        if (cfg->rotation) acc.push_back(cfg->rotation->all(kRead));
        OpTag tag(ctx, "cache_append", 4.0 * (double)c.N_kv * c.h * c.z.n1 * c.z.n2 * (double)K->elem_size(), true);
        TRY(submit(ctx, acc, [&](hipStream_t st) {
            if (bf16) hipLaunchKernelGGL(append_kernel<bf16_t>, grid, dim3(256), 0, st, c);
            else hipLaunchKernelGGL(append_kernel<float>, grid, dim3(256), 0, st, c);
            return launched();
        }));
        K->whole_submitted();
        V->whole_submitted();
        return NNT_OK;
    });
}

int32_t nnt_cache_attention(nnt_ctx* ctx, const nnt_cache_cfg* cfg, float scale, nnt_tensor* QKV, nnt_tensor* K, nnt_tensor* V, nnt_tensor* B) {
    return entry(ctx, [&]() -> int32_t {
        if (!B) return fail(ctx, NNT_EINVAL, "nnt_cache_attention: null argument");
        TRY(cache_check(ctx, cfg, QKV, K, V, B));
        if (!(scale > 0.f && scale < 1e30f)) return fail(ctx, NNT_EINVAL, "nnt_cache_attention: scale must be positive");
        const Cut u = cut_of(cfg, QKV, K);
        Attend a{};
        a.c = cache_of(cfg, QKV, K, V);
        a.out = rows_of(B);
        a.scale = scale * kLog2e;
        a.splits = u.splits;
        a.chunks = u.chunks;
        const bool bf16 = K->dtype == NNT_BF16;
        const AttendFn fn = bf16 ? attend_instance<bf16_t>(u) : attend_instance<float>(u);
        const dim3 grid((unsigned)u.splits, (unsigned)(u.chunks * a.c.N_kv), (unsigned)a.c.z.n2);
        const int64_t rows = (int64_t)a.c.z.n1 * a.c.z.n2 * a.c.N_h;
        std::vector<Access> acc{B->all(kReadWrite), QKV->all(kRead)};
        K->whole_access(kRead, &acc);
        V->whole_access(kRead, &acc);
        if (cfg->rotation) acc.push_back(cfg->rotation->all(kRead));
        // (the lengths are on the device: the work counted is that of the queries and results, and of caches that are full)
        OpTag tag(ctx, "cache_attention", (2.0 * (double)rows * a.c.h + 2.0 * (double)a.c.max_pages * a.c.P * a.c.N_kv * a.c.h * a.c.z.n2) * (double)K->elem_size(), true);
        TRY(submit(ctx, acc, [&](hipStream_t st) -> int32_t {
            a.partial = stream_scratch_of(ctx);
            hipLaunchKernelGGL(fn, grid, dim3(kWaves * 64), 0, st, a);
            TRY(launched());
            if (u.splits == 1) return NNT_OK;
            const dim3 jg((unsigned)((rows + 3) / 4));
            if (bf16) hipLaunchKernelGGL(join_kernel<bf16_t>, jg, dim3(256), 0, st, a, u.R, u.step);
            else hipLaunchKernelGGL(join_kernel<float>, jg, dim3(256), 0, st, a, u.R, u.step);
            return launched();
        }, u.splits == 1 ? 1 : 2));
        K->whole_submitted();
        V->whole_submitted();
        return NNT_OK;
    });
}
