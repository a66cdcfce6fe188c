// Orthogonalisation of matrices by Newton-Schulz products, and the optimiser step that is made of it:
//
//   X_0 = U / (|U|_F + eps),   A = X X^T,   B = b A + c A^2,   X <- a X + B X   (the short side of X first),
//   M <- mu M + G,  U = M or G + mu M,   P <- (1 - lr wd) P - lr s X.
//
// A step costs m^2 n (A is symmetric: half of it) + m^3 (A^2: half) + 2 m^2 n flops, so it is bound by the matrix cores
// for all but the smallest matrices.  The fp32 matrix instructions reach 150 TFLOP/s; the fp16 ones eight times that
// and more.  A value x is therefore kept as two halves, hi = fp16(2^12 x) and lo = fp16(2^12 x - hi), and a product is
// hi hi + hi lo + lo hi with sums in fp32: three instructions of the fast kind in place of one of the slow.  hi + lo hold 22 bits of
// x (the last one that an fp16 number of this scale can have is 2^-36), the term lo lo that is left out is below 2^-22 of the product, so
// results are as far from 64 bits as those of fp32 products to within a small factor.  2^12 keeps both halves of the entries that matter
// away from fp16's smallest numbers and leaves room up to 16; what the iteration's polynomials can reach is checked by the caller.
//
// All operands of the products lie in the workspace as panels: 64 rows x 32 columns of the contraction, hi part and lo part of 4 KB each,
// inside them eight columns of a row next to each other (16 bytes), 64 rows of those, then the next eight columns.  That is the
// image that the products want in LDS, so loads are contiguous, and a matrix instruction's operand is one 16-byte LDS read per lane
// without bank conflicts.  Every product has the contraction along the columns of both operands: A = X X^T and A^2 = A A^T anyway, and B X
// reads X as its transpose, which the step before (or the set-up) has written beside X itself.  Rows and columns are padded with zeros to whole
// tiles; zeros stay zeros through the iteration.
#include "device_util.hpp"
#include "internal.hpp"
#include "raw_vec.hpp"

#include <cmath>

namespace nnt {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kGroupMatrices = 16;        // matrices of one set of launches
constexpr int kNormBlocks = 512;          // most partial sums of a matrix's norm
constexpr float kScale = 4096.f;          // 2^12
constexpr int kPanelBytes = 8192;         // 64 rows x 32 columns, both parts

// A matrix as a tiled tensor of two axes.
struct MatView {
    void* const* tiles;
    int32_t dtype;
};

struct NsMatrix {
    int32_t rows, cols, base0, base1, grid0, grid1;      // the tensors' geometry
    int32_t flip;                                        // X is the transpose (more rows than columns)
    int32_t mp, np;                                      // X's padded extents, mp <= np up to padding
    int32_t first_sym, first_full, first_patch;          // workgroups of the matrices before it, per kind of launch
    int64_t X, XT, A, B, part;                           // bytes from the start of the workspace; X and XT: two buffers each, one behind the other
    MatView G, M, P, LP;                                 // gradient, momentum, parameter (or result), bf16 copy
    float decay, step;                                   // P <- decay P - step X (step < 0: P <- X)
};

struct NsGroup {
    char* space;
    int32_t n, norm_blocks, nesterov;
    float mu;                                            // < 0: no momentum, U = G
    float a, b, c, eps;
    NsMatrix mat[kGroupMatrices];
};

__device__ __forceinline__ float load_of(const MatView& v, int tile, int64_t off) {
    return v.dtype == NNT_F32 ? global_as<const float>(v.tiles[tile])[off] : bf2f(global_as<const bf16_t>(v.tiles[tile])[off]);
}

// ---------------------------------------------------------------- momentum and norm
// Workgroups take chunks of 2048 elements of a tile in turn; each leaves one partial sum of squares in 64 bits (no value of fp32 overflows or
// vanishes in it).
__global__ void __launch_bounds__(256) ns_norm_kernel(NsGroup g) {
    __shared__ double red[4];
    const NsMatrix& q = g.mat[blockIdx.y];
    const int tid = threadIdx.x;
    constexpr int kChunk = 2048;
    const int64_t full = (int64_t)q.base0 * q.base1;
    const int per_tile = (int)((full + kChunk - 1) / kChunk);
    const int64_t chunks = (int64_t)per_tile * q.grid0 * q.grid1;
    double sum = 0.0;
    for (int64_t ch = blockIdx.x; ch < chunks; ch += gridDim.x) {
        const int tile = (int)(ch / per_tile);
        const int t0 = tile % q.grid0, t1 = tile / q.grid0;
        const int64_t numel = (int64_t)min(q.base0, q.rows - t0 * q.base0) * min(q.base1, q.cols - t1 * q.base1);
        const int64_t at = (ch - (int64_t)tile * per_tile) * kChunk;
#pragma unroll
        for (int s = 0; s < 2; s++) {
            const int64_t e = at + (s * 256 + tid) * 4;
            if (e >= numel) continue;
            const int cnt = (int)min((int64_t)4, numel - e);
            float u[4];
            if (q.G.dtype == NNT_F32) {
                RawVec<float> x;
                x.load(global_as<const float>(q.G.tiles[tile]) + e, cnt);
#pragma unroll
                for (int k = 0; k < 4; k++) u[k] = x.at(k);
            } else {
#pragma unroll
                for (int k = 0; k < 4; k++) u[k] = k < cnt ? bf2f(global_as<const bf16_t>(q.G.tiles[tile])[e + k]) : 0.f;
            }
            if (g.mu >= 0.f) {
                float* mp = global_as<float>(q.M.tiles[tile]) + e;
                RawVec<float> m;
                m.load(mp, cnt);
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    v[k] = fmaf(g.mu, m.at(k), u[k]);
                    u[k] = g.nesterov ? fmaf(g.mu, v[k], u[k]) : v[k];
                }
                RawVec<float>::store(mp, v, cnt);
            }
#pragma unroll
            for (int k = 0; k < 4; k++)
                if (k < cnt) sum += (double)u[k] * (double)u[k];
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if ((tid & 63) == 0) red[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) reinterpret_cast<double*>(g.space + q.part)[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

__device__ __forceinline__ int matrix_of(const NsGroup& g, int wg, int32_t NsMatrix::*first) {
    int k = 0;
    while (k + 1 < g.n && wg >= g.mat[k + 1].*first) k++;
    return k;
}

// hi and lo part of a value of the workspace's scale
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// byte offset of the 16 bytes that hold columns k .. k + 7 (k a multiple of 8) of a row in an operand with K columns, hi part
__device__ __forceinline__ int64_t panel_at(int row, int k, int K) {
    return ((int64_t)(row >> 6) * (K >> 5) + (k >> 5)) * kPanelBytes + ((k & 31) >> 3) * 1024 + (row & 63) * 16;
}

// ---------------------------------------------------------------- set-up: X_0 and its transpose
// One workgroup takes 64 x 64 elements: read along the tensor's contiguous axis, turned in LDS, written as panels of both.
__global__ void __launch_bounds__(256) ns_split_kernel(NsGroup g) {
    __shared__ float t[64][65];                          // [i][j]
    __shared__ double red[4];
    const int wg = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const NsMatrix& q = g.mat[matrix_of(g, wg, &NsMatrix::first_patch)];
    const int pm = q.mp >> 6, p = wg - q.first_patch;
    const int i0 = (p % pm) * 64, j0 = (p / pm) * 64;
    const double* part = reinterpret_cast<const double*>(g.space + q.part);
    double sum = 0.0;
    for (int k = tid; k < g.norm_blocks; k += 256) sum += part[k];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) red[wave] = sum;
    __syncthreads();
    const float scale = (float)((double)kScale / (sqrt(red[0] + red[1] + red[2] + red[3]) + (double)g.eps));
    const int r0 = q.flip ? j0 : i0, c0 = q.flip ? i0 : j0;
    const int r = r0 + lane, t0 = r / q.base0, o0 = r - t0 * q.base0, e0 = min(q.base0, q.rows - t0 * q.base0);
#pragma unroll 4
    for (int s = 0; s < 16; s++) {
        const int c = c0 + s * 4 + wave;
        float u = 0.f;
        if (r < q.rows && c < q.cols) {
            const int t1 = c / q.base1;
            const int tile = t0 + q.grid0 * t1;
            const int64_t off = o0 + (int64_t)e0 * (c - t1 * q.base1);
            u = load_of(q.G, tile, off);
            if (g.mu >= 0.f) {
                const float m = global_as<const float>(q.M.tiles[tile])[off];
                u = g.nesterov ? fmaf(g.mu, m, u) : m;
            }
        }
        const int i = q.flip ? s * 4 + wave : lane, j = q.flip ? lane : s * 4 + wave;
        t[i][j] = u * scale;
    }
    __syncthreads();
    // a lane's row, a wavefront's two groups of eight columns, of X and of its transpose
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int k = (wave * 2 + h) * 8;
        f16x8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            _Float16 x, y;
            split(t[lane][k + e], x, y);
            hi[e] = x;
            lo[e] = y;
        }
        char* d = g.space + q.X + panel_at(i0 + lane, j0 + k, q.np);
        *reinterpret_cast<f16x8*>(d) = hi;
        *reinterpret_cast<f16x8*>(d + 4096) = lo;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            _Float16 x, y;
            split(t[k + e][lane], x, y);
            hi[e] = x;
            lo[e] = y;
        }
        d = g.space + q.XT + panel_at(j0 + lane, i0 + k, q.mp);
        *reinterpret_cast<f16x8*>(d) = hi;
        *reinterpret_cast<f16x8*>(d + 4096) = lo;
    }
}

// ---------------------------------------------------------------- products
enum { kGram, kPoly, kStep, kLast };

// What a lane has of the result: one column j, four rows i .. i + 3 at a time, as the second operand's row j and columns i.
__device__ __forceinline__ void apply_result(const NsMatrix& q, const float (&x)[4], int i, int j) {
    const bool copy = q.LP.tiles != nullptr;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int r = q.flip ? j : i + k, c = q.flip ? i + k : j;
        if (r >= q.rows || c >= q.cols) continue;
        const int t0 = r / q.base0, t1 = c / q.base1;
        const int tile = t0 + q.grid0 * t1;
        const int64_t off = (r - t0 * q.base0) + (int64_t)min(q.base0, q.rows - t0 * q.base0) * (c - t1 * q.base1);
        if (q.step < 0.f) {
            if (q.P.dtype == NNT_F32) global_as<float>(q.P.tiles[tile])[off] = x[k];
            else global_as<bf16_t>(q.P.tiles[tile])[off] = f2bf(x[k]);
        } else {
            float* p = global_as<float>(q.P.tiles[tile]) + off;
            const float v = fmaf(-q.step, x[k], q.decay * *p);
            *p = v;
            if (copy) global_as<bf16_t>(q.LP.tiles[tile])[off] = f2bf(v);
        }
    }
}

// One workgroup of four wavefronts computes 2 WT x 2 WT results, each wavefront WT x WT of them.  Of the symmetric results only tiles on
// and above the diagonal are computed, and written twice.
template <int MODE, int WT>
__global__ void __launch_bounds__(256, WT == 64 ? 2 : 4) ns_product_kernel(NsGroup g, int now) {
    constexpr int MT = 2 * WT, MI = WT / 32, RB = MT / 64;      // macro-tile, fragments per side, row blocks
    constexpr int kStage = 2 * RB * kPanelBytes, NL = kStage / 4096;
    constexpr int kPitch = WT + 8;                              // of the turned results, in 32-bit words
    constexpr int kTurn = 4 * WT * kPitch * 4;
    __shared__ __align__(16) char lds[2 * kStage > kTurn ? 2 * kStage : kTurn];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wr = wave & 1, wc = wave >> 1;
    const int wg = blockIdx.x;
    constexpr bool kSym = MODE == kGram || MODE == kPoly;
    const NsMatrix& q = g.mat[matrix_of(g, wg, kSym ? &NsMatrix::first_sym : &NsMatrix::first_full)];
    const int tm = q.mp / MT;
    int ti, tj;
    if constexpr (kSym) {
        const int p = wg - q.first_sym;
        tj = (int)((sqrtf(8.f * (float)p + 1.f) - 1.f) * 0.5f);
        while (tj * (tj + 1) / 2 > p) tj--;
        while ((tj + 1) * (tj + 2) / 2 <= p) tj++;
        ti = p - tj * (tj + 1) / 2;
    } else {
        const int p = wg - q.first_full;
        ti = p % tm;
        tj = p / tm;
    }
    const int64_t xbytes = (int64_t)q.mp * q.np * 4;
    const int K = MODE == kGram ? q.np : q.mp, nk = K >> 5;
    const char* Pb = g.space + (MODE == kGram ? q.X + now * xbytes : MODE == kPoly ? q.A : q.B);
    const char* Qb = g.space + (MODE == kGram ? q.X + now * xbytes : MODE == kPoly ? q.A : q.XT + now * xbytes);
    // 16 bytes per thread and load; load l of a stage lies in row block l / 2 (half l & 1 of its 8 KB), P's blocks first
    const char* src[NL];
#pragma unroll
    for (int l = 0; l < NL; l++) {
        const int blk = l >> 1;
        const char* b = blk < RB ? Pb + (int64_t)(ti * RB + blk) * nk * kPanelBytes : Qb + (int64_t)(tj * RB + blk - RB) * nk * kPanelBytes;
        src[l] = in_global(b) + (l & 1) * 4096 + tid * 16;
    }
    f32x16 acc[MI][MI];
#pragma unroll
    for (int x = 0; x < MI; x++)
#pragma unroll
        for (int y = 0; y < MI; y++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[x][y][r] = 0.f;
    uint4 st[NL];
#pragma unroll
    for (int l = 0; l < NL; l++) st[l] = *reinterpret_cast<const uint4*>(in_global(src[l]));
#pragma unroll
    for (int l = 0; l < NL; l++) *reinterpret_cast<uint4*>(lds + l * 4096 + tid * 16) = st[l];
    __syncthreads();
    const int row_p = WT == 64 ? 0 : wr * 32, row_q = WT == 64 ? 0 : wc * 32;
    const int off_p = (WT == 64 ? wr * kPanelBytes : 0) + (row_p + (lane & 31)) * 16 + (lane >> 5) * 1024;
    const int off_q = RB * kPanelBytes + (WT == 64 ? wc * kPanelBytes : 0) + (row_q + (lane & 31)) * 16 + (lane >> 5) * 1024;
    for (int kb = 0; kb < nk; kb++) {
        const bool more = kb + 1 < nk;
        if (more) {
#pragma unroll
            for (int l = 0; l < NL; l++) st[l] = *reinterpret_cast<const uint4*>(in_global(src[l] + (int64_t)(kb + 1) * kPanelBytes));
        }
        const char* buf = lds + (kb & 1) * kStage;
#pragma unroll
        for (int ks = 0; ks < 2; ks++) {
            f16x8 ph[MI], pl[MI], qh[MI], ql[MI];
#pragma unroll
            for (int x = 0; x < MI; x++) {
                ph[x] = *reinterpret_cast<const f16x8*>(buf + off_p + ks * 2048 + x * 512);
                pl[x] = *reinterpret_cast<const f16x8*>(buf + off_p + ks * 2048 + x * 512 + 4096);
                qh[x] = *reinterpret_cast<const f16x8*>(buf + off_q + ks * 2048 + x * 512);
                ql[x] = *reinterpret_cast<const f16x8*>(buf + off_q + ks * 2048 + x * 512 + 4096);
            }
#pragma unroll
            for (int x = 0; x < MI; x++)
#pragma unroll
                for (int y = 0; y < MI; y++) {
                    acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[x], ql[y], acc[x][y], 0, 0, 0);
                    acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl[x], qh[y], acc[x][y], 0, 0, 0);
                    acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[x], qh[y], acc[x][y], 0, 0, 0);
                }
        }
        if (more) {
            char* nxt = lds + ((kb + 1) & 1) * kStage;
#pragma unroll
            for (int l = 0; l < NL; l++) *reinterpret_cast<uint4*>(nxt + l * 4096 + tid * 16) = st[l];
        }
        __syncthreads();
    }
    // results: this lane has column j0 + 32 y + (lane & 31), rows i0 + 32 x + 8 p + 4 (lane >> 5) + 0 .. 3
    const int i0 = ti * MT + wr * WT, j0 = tj * MT + wc * WT;
    const char* E = g.space + (MODE == kPoly ? q.A : q.XT + now * xbytes);          // the term that is added, laid out like the result
    char* D = g.space + (MODE == kGram ? q.A : MODE == kPoly ? q.B : q.XT + (1 - now) * xbytes);
    const float factor = (MODE == kPoly ? g.c : 1.f) / kScale;      // sums carry the scale twice
    const float add = MODE == kPoly ? g.b : g.a;
    uint32_t* turn = reinterpret_cast<uint32_t*>(lds) + wave * WT * kPitch;
#pragma unroll
    for (int x = 0; x < MI; x++)
#pragma unroll
        for (int y = 0; y < MI; y++)
#pragma unroll
            for (int p = 0; p < 4; p++) {
                const int i = i0 + x * 32 + p * 8, j = j0 + y * 32 + (lane & 31);
                const int64_t at = panel_at(j, i, q.mp) + (lane >> 5) * 8;
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; k++) v[k] = acc[x][y][p * 4 + k] * factor;
                if constexpr (MODE != kGram) {
                    const f16x4 eh = *reinterpret_cast<const f16x4*>(E + at), el = *reinterpret_cast<const f16x4*>(E + at + 4096);
#pragma unroll
                    for (int k = 0; k < 4; k++) v[k] = fmaf(add, (float)eh[k] + (float)el[k], v[k]);
                }
                if constexpr (MODE == kLast) {
#pragma unroll
                    for (int k = 0; k < 4; k++) v[k] *= 1.f / kScale;
                    apply_result(q, v, i + (lane >> 5) * 4, j);
                } else {
                    f16x4 hi, lo;
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        _Float16 h, l;
                        split(v[k], h, l);
                        hi[k] = h;
                        lo[k] = l;
                        turn[(x * 32 + p * 8 + (lane >> 5) * 4 + k) * kPitch + y * 32 + (lane & 31)] =
                            (uint32_t)__builtin_bit_cast(uint16_t, h) | ((uint32_t)__builtin_bit_cast(uint16_t, l) << 16);
                    }
                    *reinterpret_cast<f16x4*>(D + at) = hi;
                    *reinterpret_cast<f16x4*>(D + at + 4096) = lo;
                }
            }
    if constexpr (MODE != kLast) {
        if (kSym && ti == tj) return;
        // the same with rows and columns exchanged: each wavefront turns its own part
        char* Dt = kSym ? D : g.space + q.X + (1 - now) * xbytes;
        const int Kt = kSym ? q.mp : q.np;
#pragma unroll
        for (int s = 0; s < WT * WT / 8 / 64; s++) {
            const int idx = s * 64 + lane, row = idx % WT, k = idx / WT * 8;
            const uint4 u = *reinterpret_cast<const uint4*>(turn + row * kPitch + k), w = *reinterpret_cast<const uint4*>(turn + row * kPitch + k + 4);
            const uint4 hi = make_uint4((u.x & 0xffff) | (u.y << 16), (u.z & 0xffff) | (u.w << 16), (w.x & 0xffff) | (w.y << 16), (w.z & 0xffff) | (w.w << 16));
            const uint4 lo = make_uint4((u.x >> 16) | (u.y & 0xffff0000u), (u.z >> 16) | (u.w & 0xffff0000u), (w.x >> 16) | (w.y & 0xffff0000u),
                                        (w.z >> 16) | (w.w & 0xffff0000u));
            char* d = Dt + panel_at(i0 + row, j0 + k, Kt);
            *reinterpret_cast<uint4*>(d) = hi;
            *reinterpret_cast<uint4*>(d + 4096) = lo;
        }
    }
}

// ---------------------------------------------------------------- host side
int32_t launched() { return hipGetLastError() == hipSuccess ? (int32_t)NNT_OK : (int32_t)NNT_EHIP; }

// Whether the iteration stays where the workspace's numbers can hold it: singular values start in [0, 1]; followed on a grid, they, their squares' polynomial
// and its parts have to stay below 8 (2^12 times 16 is fp16's largest number).
bool in_range(const nnt_newton_schulz_cfg& c) {
    if (!std::isfinite(c.a) || !std::isfinite(c.b) || !std::isfinite(c.c) || !(c.eps > 0.0) || !std::isfinite(c.eps) || c.steps < 1 || c.steps > 64) return false;
    constexpr int n = 4096;
    for (int k = 0; k <= n; k++) {
        double s = (double)k / n;
        for (int t = 0; t < c.steps; t++) {
            const double l = s * s, p = c.b * l + c.c * l * l;
            if (!(l <= 8.0) || !(std::fabs(p) <= 8.0)) return false;
            s = std::fabs(s * (c.a + p));
            if (!(s <= 8.0)) return false;
        }
    }
    return true;
}

bool whole_matrix(const nnt_ctx* ctx, const nnt_tensor* t) {
    if (!t || t->ctx != ctx || t->ndim != 2) return false;
    for (void* p : t->tiles)
        if (!p) return false;
    return true;
}

struct Task {
    nnt_tensor *G, *M, *P, *LP;
    float decay, step;
};

template <int WT>
void launch_product(int mode, const NsGroup& g, int now, unsigned wgs, hipStream_t st) {
    switch (mode) {
        case kGram: hipLaunchKernelGGL((ns_product_kernel<kGram, WT>), dim3(wgs), dim3(256), 0, st, g, now); break;
        case kPoly: hipLaunchKernelGGL((ns_product_kernel<kPoly, WT>), dim3(wgs), dim3(256), 0, st, g, now); break;
        case kStep: hipLaunchKernelGGL((ns_product_kernel<kStep, WT>), dim3(wgs), dim3(256), 0, st, g, now); break;
        default: hipLaunchKernelGGL((ns_product_kernel<kLast, WT>), dim3(wgs), dim3(256), 0, st, g, now); break;
    }
}

// Orthogonalises the matrices of `tasks` and applies the results, as many of them in one set of launches as it takes to fill the
// chip.  mu < 0: no momentum.
int32_t newton_schulz(nnt_ctx* ctx, const char* label, const nnt_newton_schulz_cfg& cfg, float mu, int nesterov, const std::vector<Task>& tasks) {
    size_t first = 0;
    while (first < tasks.size()) {
        // macro-tiles of 128 x 128 as soon as they fill the chip
        const size_t most = std::min(tasks.size() - first, (size_t)kGroupMatrices);
        auto count = [&](size_t k, int mt) {
            const nnt_tensor* t = tasks[first + k].G;
            return (t->shape[0] + mt - 1) / mt * ((t->shape[1] + mt - 1) / mt);
        };
        size_t n = 0;
        int64_t wide = 0;
        while (n < most && wide < 1024) wide += count(n++, 128);
        const int wt = wide >= 256 ? 64 : 32, mt = 2 * wt;
        NsGroup g{};
        g.n = (int32_t)n;
        g.nesterov = nesterov;
        g.mu = mu;
        g.a = (float)cfg.a;
        g.b = (float)cfg.b;
        g.c = (float)cfg.c;
        g.eps = (float)cfg.eps;
        int64_t bytes = 0, sym = 0, full = 0, patch = 0, chunks = 0;
        double work = 0.0;
        std::vector<Access> acc;
        for (size_t k = 0; k < n; k++) {
            const Task& t = tasks[first + k];
            NsMatrix& q = g.mat[k];
            q.rows = (int32_t)t.G->shape[0];
            q.cols = (int32_t)t.G->shape[1];
            q.base0 = (int32_t)t.G->base[0];
            q.base1 = (int32_t)t.G->base[1];
            q.grid0 = (int32_t)t.G->grid[0];
            q.grid1 = (int32_t)t.G->grid[1];
            q.flip = q.rows > q.cols;
            q.mp = (std::min(q.rows, q.cols) + mt - 1) / mt * mt;
            q.np = (std::max(q.rows, q.cols) + mt - 1) / mt * mt;
            q.first_sym = (int32_t)sym;
            q.first_full = (int32_t)full;
            q.first_patch = (int32_t)patch;
            const int64_t tm = q.mp / mt, tn = q.np / mt;
            sym += tm * (tm + 1) / 2;
            full += tm * tn;
            patch += (int64_t)(q.mp / 64) * (q.np / 64);
            chunks = std::max(chunks, ((int64_t)q.base0 * q.base1 + 2047) / 2048 * q.grid0 * q.grid1);
            const int64_t x = (int64_t)q.mp * q.np * 4, a = (int64_t)q.mp * q.mp * 4;
            q.X = bytes;
            q.XT = q.X + 2 * x;
            q.A = q.XT + 2 * x;
            q.B = q.A + a;
            q.part = q.B + a;
            bytes = q.part + kNormBlocks * 8;
            q.G = MatView{t.G->d_tiles, t.G->dtype};
            q.P = MatView{t.P->d_tiles, t.P->dtype};
            if (t.M) q.M = MatView{t.M->d_tiles, NNT_F32};
            if (t.LP) q.LP = MatView{t.LP->d_tiles, NNT_BF16};
            q.decay = t.decay;
            q.step = t.step;
            const double m = std::min(q.rows, q.cols), l = std::max(q.rows, q.cols);
            work += cfg.steps * (3.0 * m * m * l + m * m * m);
            acc.push_back(t.G->all(kRead));
            acc.push_back(t.P->all(t.step < 0.f ? kWrite : kReadWrite));
            if (t.M) acc.push_back(t.M->all(kReadWrite));
            if (t.LP) acc.push_back(t.LP->all(kWrite));
        }
        if (full > INT32_MAX || patch > INT32_MAX) return fail(ctx, NNT_EINVAL, std::string(label) + ": matrix too large");
        g.norm_blocks = (int32_t)std::min<int64_t>(chunks, kNormBlocks);
        const int32_t rc = ensure_matrix_scratch(ctx, bytes);
        if (rc != NNT_OK) return rc;
        g.space = reinterpret_cast<char*>(ctx->matrix_scratch);
        acc.push_back(Access{&ctx->matrix_dep, 1, kReadWrite});
        const int steps = cfg.steps;
        OpTag tag(ctx, label, work, false);
        const int32_t sc = submit(ctx, acc, [=](hipStream_t st) {
            hipLaunchKernelGGL(ns_norm_kernel, dim3((unsigned)g.norm_blocks, (unsigned)g.n), dim3(256), 0, st, g);
            hipLaunchKernelGGL(ns_split_kernel, dim3((unsigned)patch), dim3(256), 0, st, g);
            for (int s = 0; s < steps; s++) {
                for (int mode : {(int)kGram, (int)kPoly, s + 1 < steps ? (int)kStep : (int)kLast}) {
                    const unsigned wgs = (unsigned)(mode == kGram || mode == kPoly ? sym : full);
                    if (wt == 64) launch_product<64>(mode, g, s & 1, wgs, st);
                    else launch_product<32>(mode, g, s & 1, wgs, st);
                }
            }
            return launched();
        }, 2 + 3 * steps);
        if (sc != NNT_OK) return sc;
        first += n;
    }
    return NNT_OK;
}

}  // namespace
}  // namespace nnt

using namespace nnt;

int32_t nnt_orthogonalize(nnt_ctx* ctx, const nnt_newton_schulz_cfg* cfg, int32_t n, nnt_tensor* const* G, nnt_tensor* const* O) {
    return entry(ctx, [&]() -> int32_t {
        if (!cfg || n < 1 || !G || !O) return fail(ctx, NNT_EINVAL, "nnt_orthogonalize: bad argument");
        if (!in_range(*cfg)) return fail(ctx, NNT_EINVAL, "nnt_orthogonalize: bad configuration, or an iteration that leaves its range");
        std::vector<Task> tasks;
        for (int k = 0; k < n; k++) {
            if (!whole_matrix(ctx, G[k]) || !whole_matrix(ctx, O[k]) || !same_tiling(G[k], O[k]))
                return fail(ctx, NNT_EINVAL, "nnt_orthogonalize: G and O must be matrices of this context, tiled alike, all tiles present");
            for (int l = 0; l < n; l++)
                if ((l != k && O[l] == O[k]) || (l > k && G[l] == O[k])) return fail(ctx, NNT_EINVAL, "nnt_orthogonalize: a result is given twice or is a later input");
            tasks.push_back(Task{G[k], nullptr, O[k], nullptr, 0.f, -1.f});
        }
        return newton_schulz(ctx, "orthogonalize", *cfg, -1.f, 0, tasks);
    });
}

int32_t nnt_muon_step(nnt_ctx* ctx, const nnt_muon_cfg* cfg, int32_t n, nnt_tensor* const* G, nnt_tensor* const* P, nnt_tensor* const* M,
                      nnt_tensor* const* P_lowp) {
    return entry(ctx, [&]() -> int32_t {
        if (!cfg || n < 1 || !G || !P || !M) return fail(ctx, NNT_EINVAL, "nnt_muon_step: bad argument");
        if (!(cfg->lr >= 0.0 && cfg->lr < 1e30) || !(cfg->momentum >= 0.0 && cfg->momentum < 1.0) || !std::isfinite(cfg->weight_decay) ||
            cfg->scale < NNT_MUON_SCALE_NONE || cfg->scale > NNT_MUON_SCALE_RMS || !in_range(cfg->iteration))
            return fail(ctx, NNT_EINVAL, "nnt_muon_step: bad configuration, or an iteration that leaves its range");
        std::vector<Task> tasks;
        for (int k = 0; k < n; k++) {
            nnt_tensor* lp = P_lowp ? P_lowp[k] : nullptr;
            for (nnt_tensor* t : {G[k], P[k], M[k]})
                if (!whole_matrix(ctx, t) || t->dtype != NNT_F32 || !same_tiling(t, G[k]))
                    return fail(ctx, NNT_EINVAL, "nnt_muon_step: G, P, M must be fp32 matrices of this context, tiled alike, all tiles present");
            if (lp && (!whole_matrix(ctx, lp) || lp->dtype != NNT_BF16 || !same_tiling(lp, G[k])))
                return fail(ctx, NNT_EINVAL, "nnt_muon_step: the copy must be a bf16 matrix tiled like the parameter, all tiles present");
            if (G[k] == P[k] || G[k] == M[k] || P[k] == M[k]) return fail(ctx, NNT_EINVAL, "nnt_muon_step: one tensor in two roles");
            for (int l = 0; l < n; l++)
                if (l != k && (P[l] == P[k] || M[l] == M[k] || P[l] == M[k] || P[l] == G[k] || M[l] == G[k] || (lp && P_lowp[l] == lp)))
                    return fail(ctx, NNT_EINVAL, "nnt_muon_step: one tensor in two roles");
            const double rows = (double)P[k]->shape[0], cols = (double)P[k]->shape[1];
            const double s = cfg->scale == NNT_MUON_SCALE_ASPECT ? std::sqrt(std::max(1.0, rows / cols))
                             : cfg->scale == NNT_MUON_SCALE_RMS ? 0.2 * std::sqrt(std::max(rows, cols)) : 1.0;
            tasks.push_back(Task{G[k], M[k], P[k], lp, (float)(1.0 - cfg->lr * cfg->weight_decay), (float)(cfg->lr * s)});
        }
        return newton_schulz(ctx, "muon", cfg->iteration, (float)cfg->momentum, cfg->nesterov != 0, tasks);
    });
}
