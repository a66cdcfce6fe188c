// Orthogonalisation of matrices by Newton-Schulz products, and the optimiser step that is made of it:
//
//   X_0 = U / (|U|_F + eps),   A = X X^T,   B = b A + c A^2,   X <- a X + B X   (the short side of X first),
//   M <- mu M + G,  U = M or G + mu M,   P <- (1 - lr wd) P - lr s X.
//
// A step costs m^2 n (A is symmetric: half of it) + m^3 (A^2: half) + 2 m^2 n flops, so it is bound by the matrix cores
// for all but the smallest matrices.  The fp32 matrix instructions reach 150 TFLOP/s; the fp16 ones eight times that
// and more.  A value x is therefore kept as two halves, hi = fp16(2^14 x) and lo = fp16(2^14 x - hi), and a product is
// hi hi + hi lo + lo hi with sums in fp32: three instructions of the fast kind in place of one of the slow.  hi + lo hold 22 bits of
// x, but none below 2^-38, the last one that an fp16 number of this scale can have; the term lo lo that is left out is below 2^-22 of the product.  X stays below
// 2.83; polynomials in A are kept at a scale of 2^12, which leaves room up to 16: what the iteration can reach is checked by the caller.
//
// fp32 products keep every entry of X to 24 bits of its own size, and what is small beside its row's or column's neighbours counts: the iteration brings it up to them, by a
// factor of `a` a step.  So here rows and columns have powers of two of their own.  X is there three times: in fp32 (E), which the next X is made of; with rows as 2^e_i x_ij for
// A = X X^T, to which a column much smaller than the others contributes nothing that counts; and as its transpose with columns as 2^f_j x_ij for B X, to which a small row contributes
// nothing that counts.  Rows and columns are at most of length 1 then wherever e_i or f_j > 0.  Both come from the lengths in X_0 and fall by what a step can make a row or
// column grow, max |a + b s^2 + c s^4|, until they are 0 (X <- p(X X^T) X: a row or column grows by no more than its singular directions do).  With D = diag(2^e_i) the square products
// keep to it without a factor inside the sums:
//   (D X)(D X)^T = D A D;  stored as  D A = (D A D) D^-1, so that  (D A)(D A)^T = D A^2 D  and so on for all polynomials in A, which commute;
//   (D B)(X diag(2^f_j)) = D (B X) diag(2^f_j).
// What is stored stays below 16: |x_i (.) X^T| <= max s |.| for rows of length 1, and |b + c s^2| s <= 13.6 where |b s^2 + c s^4| <= 8 on [0, 1].  B's diagonal is kept out of it: a + B_ii, in
// fp32, is what X's row i is multiplied by (most of the step once X has arrived, where B is near a multiple of the identity).
// Rows of 1e-8 of the others, 512 x 2560, five steps: the worst of them 5e-6 of its length off, with fp32 products 8e-6, with one scale for all of X 4e-1.
//
// All operands of the products lie in the workspace as panels: 64 rows x 16 columns of the contraction, hi part and lo part of 2 KB each,
// inside them eight columns of a row next to each other (16 bytes), 64 rows of those, then the next eight columns.  That is the
// image that the products want in LDS, so loads go straight there in runs of 4 KB, and a matrix instruction's operand is one 16-byte LDS
// read per lane without bank conflicts.  Every product has the contraction along the columns of both operands: A = X X^T and A^2 = A A^T anyway, and B X
// reads X as its transpose.  D A and D B are not symmetric, but their sums are: tiles on and above
// the diagonal are computed, and scaled twice.  E lies as the results do in registers, by blocks of 32 x 32.  Rows and columns are padded with zeros to whole tiles; zeros stay zeros
// through the iteration.
#include "device_util.hpp"
#include "gemm_dl_common.hpp"
#include "internal.hpp"
#include "raw_vec.hpp"

#include <algorithm>
#include <cmath>

namespace nnt {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kGroupMatrices = 16;        // matrices of one set of launches
constexpr float kScale = 4096.f;          // of square matrices, 2^12
constexpr float kScaleX = 16384.f;        // of X, whose entries stay below 2.83: 2^14
constexpr float kGramFactor = kScale / kScaleX / kScaleX;
constexpr int kShift = 12, kShiftX = 14;  // the same as powers of two
constexpr int kPanelBytes = 4096;         // 64 rows x 16 columns, both parts
constexpr int kPartBytes = 2048;

// A matrix as a tiled tensor of two axes.
struct MatView {
    void* const* tiles;
    int32_t dtype;
};

struct NsMatrix {
    int32_t rows, cols, base0, base1, grid0, grid1;      // the tensors' geometry
    int32_t flip;                                        // X is the transpose (more rows than columns)
    int32_t mp, np;                                      // X's extents, mp <= np, padded to whole panels of 64 rows
    int32_t splits;                                      // of the long side by the workgroups that add up squares
    int64_t X, XT, E, A;                                 // bytes from the start of the workspace; XT: two buffers, one behind the other; A: see NsOp
    int64_t squares, part, largest;                      // sums of squares by split and row of X, the same of 64 rows at a time; largest entries by 64 (X the transpose: 16) rows and column
    int64_t exponents, columns, coefficients;            // e_i and f_j of the first step; a + B_ii
    MatView G, M, P, LP;                                 // gradient, momentum, parameter (or result), bf16 copy
    float decay, step;                                   // P <- decay P - step X (step < 0: P <- X)
};

// The matrices' sizes, an argument of every launch.
struct NsSizes {
    int32_t n;
    uint32_t blocks[kGroupMatrices];                     // mp / 64 and np / 64, 16 bits each
};

// Written to the start of the workspace by the first launch, so that the others have short arguments (a launch with all 2.6 KB of it takes the host
// 0.6 us longer).
struct NsGroup {
    char* space;
    int32_t n, nesterov, growth;                         // growth: log2 of what a step can make a row grow by, in 1/256
    float mu;                                            // < 0: no momentum, U = G
    float a, b, c;
    double eps;
    int64_t partial;                                     // parts of A's tiles, bytes from the start of the workspace
    NsMatrix mat[kGroupMatrices];
};

static_assert(sizeof(NsGroup) <= 4096 && sizeof(NsGroup) % 4 == 0, "an argument, copied by words");

// 16 columns, from column c0 on, of a row of a matrix: t0, o0, e0 are its tile, its place in it and the tile's height; 0 where there is none
template <typename T>
__device__ __forceinline__ void read_columns_as(const NsMatrix& q, void* const* tiles, bool there, int t0, int o0, int e0, int c0, float (&v)[16]) {
    int t1 = c0 / q.base1, c1 = c0 - t1 * q.base1;
    const T* p = there && c0 < q.cols ? global_as<const T>(tiles[t0 + q.grid0 * t1]) + o0 + (int64_t)e0 * c1 : nullptr;
#pragma unroll
    for (int s = 0; s < 16; s++) {
        v[s] = 0.f;
        if (there && c0 + s < q.cols) {
            if constexpr (sizeof(T) == 4) v[s] = *p;
            else v[s] = bf2f(*p);
        }
        p += e0;
        if (++c1 == q.base1) {                           // (the tiles' pointers are looked up once each)
            c1 = 0;
            t1++;
            if (there && c0 + s + 1 < q.cols) p = global_as<const T>(tiles[t0 + q.grid0 * t1]) + o0;
        }
    }
}
__device__ __forceinline__ void read_columns(const NsMatrix& q, const MatView& w, bool there, int t0, int o0, int e0, int c0, float (&v)[16]) {
    if (w.dtype == NNT_F32) read_columns_as<float>(q, w.tiles, there, t0, o0, e0, c0, v);
    else read_columns_as<bf16_t>(q, w.tiles, there, t0, o0, e0, c0, v);
}

// ... to where read_columns finds them
__device__ __forceinline__ void write_columns(const NsMatrix& q, void* const* tiles, bool there, int t0, int o0, int e0, int c0, const float (&v)[16]) {
    int t1 = c0 / q.base1, c1 = c0 - t1 * q.base1;
    float* p = there && c0 < q.cols ? global_as<float>(tiles[t0 + q.grid0 * t1]) + o0 + (int64_t)e0 * c1 : nullptr;
#pragma unroll
    for (int s = 0; s < 16; s++) {
        if (there && c0 + s < q.cols) *p = v[s];
        p += e0;
        if (++c1 == q.base1) {
            c1 = 0;
            t1++;
            if (there && c0 + s + 1 < q.cols) p = global_as<float>(tiles[t0 + q.grid0 * t1]) + o0;
        }
    }
}

// ---------------------------------------------------------------- momentum and norms
// Sums over the wavefront of 16 values each: the lane's own of the sums, number sum16_index(lane).  Halves are exchanged while there is more than one value left,
// 17 exchanges for all of them.
__device__ __forceinline__ int sum16_index(int lane) { return lane >> 2; }
template <int HALF>
__device__ __forceinline__ void sum_halves(double (&v)[16], int lane) {
    const bool up = lane & (HALF * 4);
#pragma unroll
    for (int k = 0; k < HALF; k++) {
        const double keep = up ? v[k + HALF] : v[k], give = up ? v[k] : v[k + HALF];
        v[k] = keep + __shfl_xor(give, HALF * 4, 64);
    }
}
__device__ __forceinline__ double sum16(double (&v)[16], int lane) {
    sum_halves<8>(v, lane);
    sum_halves<4>(v, lane);
    sum_halves<2>(v, lane);
    sum_halves<1>(v, lane);
    v[0] += __shfl_xor(v[0], 2, 64);
    return v[0] + __shfl_xor(v[0], 1, 64);
}

// The upper half of an absolute value's bits, rounded up.
__device__ __forceinline__ uint32_t upper_half(float v) { return (__float_as_uint(fabsf(v)) + 0xffffu) >> 16; }
__device__ __forceinline__ float from_upper_half(uint32_t h) { return __uint_as_float(h << 16); }
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t larger_halves(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// The same as sum16 for the upper halves of the largest absolute values, two at a time: lane 8 k has number k in its lower half and number k + 8 in its upper half.
__device__ __forceinline__ uint32_t largest16(const float (&u)[16], int lane) {
    uint32_t v[8];
#pragma unroll
    for (int k = 0; k < 8; k++) v[k] = upper_half(u[k]) | (upper_half(u[k + 8]) << 16);
#pragma unroll
    for (int half = 4; half > 0; half >>= 1) {
        const bool up = lane & (half * 8);
#pragma unroll
        for (int k = 0; k < half; k++) {
            const uint32_t keep = up ? v[k + half] : v[k], give = up ? v[k] : v[k + half];
            v[k] = larger_halves(keep, __shfl_xor(give, half * 8, 64));
        }
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) v[0] = larger_halves(v[0], __shfl_xor(v[0], o, 64));
    return v[0];
}
// and within a lane
__device__ __forceinline__ float largest_of(const float (&u)[16]) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < 16; k++) v = fmaxf(v, fabsf(u[k]));
    return v;
}

// A workgroup takes 64 rows of X and a part of its columns, 128 at a time: a lane a row of the tensor and a wavefront 16 columns of it.  Squares are added up in 64
// bits (no value of fp32 overflows or vanishes in it), by row of X and over the 64 rows; of X's columns the largest entries are left.  Bound by memory: 8192 x 8192 with momentum, 180 us for 805 MB (139 along the tiles
// in 16-byte vectors, which cannot add up rows).
constexpr int kNormWaves = 8, kNormSpan = 16 * kNormWaves;
template <bool FLIP>
__device__ __forceinline__ void norm_part(const NsGroup& g, const NsMatrix& q, int rb, int part, double (*red)[64]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint16_t* largest = reinterpret_cast<uint16_t*>(g.space + q.largest);
    double sum[FLIP ? 16 : 1];
#pragma unroll
    for (int s = 0; s < (FLIP ? 16 : 1); s++) sum[s] = 0.0;
#pragma unroll 1
    for (int l0 = part * kNormSpan; l0 < q.np; l0 += q.splits * kNormSpan) {
        const int r = (FLIP ? l0 + (wave >> 2) * 64 : rb * 64) + lane, c0 = FLIP ? rb * 64 + (wave & 3) * 16 : l0 + wave * 16;
        const int t0 = min(r, q.rows - 1) / q.base0, o0 = r - t0 * q.base0, e0 = min(q.base0, q.rows - t0 * q.base0);
        const bool there = r < q.rows;
        float u[16];
        read_columns(q, q.G, there, t0, o0, e0, c0, u);
        if (g.mu >= 0.f) {
            float m[16];
            read_columns(q, q.M, there, t0, o0, e0, c0, m);
#pragma unroll
            for (int s = 0; s < 16; s++) {
                m[s] = fmaf(g.mu, m[s], u[s]);
                u[s] = g.nesterov ? fmaf(g.mu, m[s], u[s]) : m[s];
            }
            write_columns(q, q.M.tiles, there, t0, o0, e0, c0, m);
        }
#pragma unroll
        for (int s = 0; s < 16; s++) sum[FLIP ? s : 0] += (double)u[s] * (double)u[s];
        if constexpr (FLIP) {
            if (r < q.np) largest[(int64_t)(rb * 4 + (wave & 3)) * q.np + r] = (uint16_t)upper_half(largest_of(u));
        } else {
            const uint32_t x = largest16(u, lane);
            if (c0 < q.np && (lane & 7) == 0) {
                uint16_t* d = largest + (int64_t)rb * q.np + c0 + (lane >> 3);
                d[0] = (uint16_t)x;
                d[8] = (uint16_t)(x >> 16);
            }
        }
    }
    if constexpr (FLIP) {
        const double x = sum16(sum, lane);
        if ((lane & 3) == 0) red[wave >> 2][(wave & 3) * 16 + sum16_index(lane)] = x;
    } else {
        red[wave][lane] = sum[0];
    }
}

__global__ void __launch_bounds__(64 * kNormWaves, 6) ns_norm_kernel(NsGroup g) {
    __shared__ double red[kNormWaves][64];
    // the launches behind this one read the group from the workspace
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (unsigned k = threadIdx.x; k < sizeof(NsGroup) / 4; k += 64 * kNormWaves) reinterpret_cast<uint32_t*>(g.space)[k] = reinterpret_cast<const uint32_t*>(&g)[k];
    const NsMatrix& q = g.mat[blockIdx.y];
    const int row_blocks = q.mp >> 6, tid = threadIdx.x;
    if ((int)blockIdx.x >= row_blocks * q.splits) return;
    const int rb = blockIdx.x % row_blocks, part = blockIdx.x / row_blocks;
    if (q.flip) norm_part<true>(g, q, rb, part, red);
    else norm_part<false>(g, q, rb, part, red);
    __syncthreads();
    if (tid < 64) {
        double t = 0.0;
        for (int w = 0; w < (q.flip ? kNormWaves / 4 : kNormWaves); w++) t += red[w][tid];
        reinterpret_cast<double*>(g.space + q.squares)[(int64_t)part * q.mp + rb * 64 + tid] = t;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o, 64);
        if (tid == 0) reinterpret_cast<double*>(g.space + q.part)[blockIdx.x] = t;
    }
}

// e of a row or column of at most the given length in a matrix of the given length: that of X_0 times 2^e is at most 1 long.  0 for those without a length (zeros, no numbers).
// No more than 120: fp32 rounds at 2^-149, and what has shrunk as far as that need not shrink any further (0.6 times the last bit is the last bit).
constexpr int kMostExponent = 120;
__device__ __forceinline__ int exponent_of(double length, double of) {
    const double x = length / of;
    if (!(x > 0.0) || x > 1.0) return 0;
    int k;
    (void)frexp(x, &k);
    return min(max(0, -k), kMostExponent);
}

// Set-up of a workgroup of four wavefronts: the matrix's length, and the exponents of the 64 rows of X from row i0 on and of the 64 columns from column j0 on.
struct SetUp {
    double total[4], squares[4][64];
    int largest[4][64];
    int row[64], column[64];
};
__device__ __forceinline__ void largest_of_columns(const NsGroup& g, const NsMatrix& q, int j0, SetUp& w) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint16_t* largest = reinterpret_cast<const uint16_t*>(g.space + q.largest) + j0 + lane;
    int most = 0;
#pragma unroll 8
    for (int k = wave; k < (q.flip ? q.mp >> 4 : q.mp >> 6); k += 4) most = max(most, (int)largest[(int64_t)k * q.np]);
    w.largest[wave][lane] = most;
}
__device__ __forceinline__ void column_exponents(const NsGroup& g, const NsMatrix& q, int j0, bool keep, double length, SetUp& w) {
    const int lane = threadIdx.x & 63;
    const int most = max(max(w.largest[0][lane], w.largest[1][lane]), max(w.largest[2][lane], w.largest[3][lane]));
    const int f = exponent_of((double)from_upper_half((uint32_t)most) * sqrt((double)q.mp), length);
    w.column[lane] = f;
    if (keep) reinterpret_cast<int*>(g.space + q.columns)[j0 + lane] = f;
}
// j0 < 0: rows only
__device__ __forceinline__ double length_and_exponents(const NsGroup& g, const NsMatrix& q, int i0, int j0, bool keep_rows, bool keep_columns, SetUp& w) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const double *part = reinterpret_cast<const double*>(g.space + q.part), *squares = reinterpret_cast<const double*>(g.space + q.squares);
    double sum = 0.0, row = 0.0;
    for (int k = tid; k < (q.mp >> 6) * q.splits; k += 256) sum += part[k];
#pragma unroll 8
    for (int k = wave; k < q.splits; k += 4) row += squares[(int64_t)k * q.mp + i0 + lane];
    if (j0 >= 0) largest_of_columns(g, q, j0, w);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) w.total[wave] = sum;
    w.squares[wave][lane] = row;
    __syncthreads();
    const double length = sqrt(w.total[0] + w.total[1] + w.total[2] + w.total[3]) + g.eps;
    if (wave == 0) {
        const int e = exponent_of(sqrt(w.squares[0][lane] + w.squares[1][lane] + w.squares[2][lane] + w.squares[3][lane]), length);
        w.row[lane] = e;
        if (keep_rows) reinterpret_cast<int*>(g.space + q.exponents)[i0 + lane] = e;
    }
    if (wave == 1 && j0 >= 0) column_exponents(g, q, j0, keep_columns, length, w);
    return length;                                       // (w.row and w.column are there behind the next barrier)
}

// What `steps` steps can make a row or column grow by, as a power of two; its exponent behind that.
__host__ __device__ inline int grown_by(int growth, int steps) { return (growth * steps + 255) >> 8; }
__device__ __forceinline__ int exponent_at(int first, int grown) { return min(max(first - grown, 0), kMostExponent); }

// The matrix of a workgroup of a launch over tiles of BM x BM results of all matrices (SYM: those on and above the diagonal of
// square results); `wg` becomes its number among the matrix's own.
template <bool SYM, int BM>
__device__ __forceinline__ int matrix_of(const NsSizes& g, int& wg) {
    constexpr int u = BM / 64;
    int k = 0, total = 0, before = 0;
#pragma unroll
    for (int m = 0; m < kGroupMatrices - 1; m++) {
        if (m + 1 < g.n) {
            const int tm = ((int)(g.blocks[m] & 0xffffu) + u - 1) / u, tn = ((int)(g.blocks[m] >> 16) + u - 1) / u;
            total += SYM ? tm * (tm + 1) / 2 : tm * tn;
            if (wg >= total) {
                k = m + 1;
                before = total;
            }
        }
    }
    wg -= before;
    return k;
}

// hi and lo part of a value of the workspace's scale.  The value is made definite first: as the result of a product the compiler rounds it straight
// to fp16 in one place and by way of fp32 in another, and where the two differ, one value in some ten thousand, hi + lo is off by 2^-11.
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
    asm("" : "+v"(v));
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// byte offset in E of a lane's results p .. of the block of 32 x 32 at row i and column j: rows i + 8 p + 4 (lane >> 5) + 0 .. 3, column j + (lane & 31)
__device__ __forceinline__ int64_t block_at(int i, int j, int mp) { return ((int64_t)(j >> 5) * (mp >> 5) + (i >> 5)) * 4096 + (threadIdx.x & 63) * 16; }

// byte offset of the 16 bytes that hold columns k .. k + 7 (k a multiple of 8) of a row in an operand with K columns, hi part
__device__ __forceinline__ int64_t panel_at(int row, int k, int K) {
    return ((int64_t)(row >> 6) * (K >> 4) + (k >> 4)) * kPanelBytes + ((k & 15) >> 3) * 1024 + (row & 63) * 16;
}

// x / length times a power of two, for any length above 0 (in 64 bits: the sum of the partial sums' root and eps): a factor between 1 and 2 and a power of two, since the
// quotient alone can lie outside of fp32.
struct Scale {
    float factor;
    int exponent;
    __device__ __forceinline__ explicit Scale(double length) {
        factor = (float)(1.0 / frexp(length, &exponent));
        exponent = -exponent;
    }
    __device__ __forceinline__ float operator()(float x, int more) const { return ldexpf(x, exponent + more) * factor; }
};

// ---------------------------------------------------------------- set-up: X_0 in its three forms
// One workgroup takes 64 x 64 elements: read along the tensor's contiguous axis, turned in LDS, written as panels of X and of its transpose and in fp32.  Bound by memory: 8192 x 8192
// with momentum, 310 us for 1342 MB; all forms are written here because turning X for the first product with it would cost a pass of its own.
__global__ void __launch_bounds__(256, 8) ns_split_kernel(const NsGroup* __restrict__ group, NsSizes sizes) {
    const NsGroup& g = *group;
    __shared__ float t[64][65];                          // [i][j]
    __shared__ SetUp setup;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int p = blockIdx.x;
    const NsMatrix& q = g.mat[matrix_of<false, 64>(sizes, p)];
    const int pm = q.mp >> 6;
    const int i0 = (p % pm) * 64, j0 = (p / pm) * 64;
    // this lane's row of the tensor, and the wavefront's 16 columns; all loads are started before the norm is put together
    const int r0 = q.flip ? j0 : i0, c0 = __builtin_amdgcn_readfirstlane((q.flip ? i0 : j0) + wave * 16);
    const int r = r0 + lane, t0 = min(r, q.rows - 1) / q.base0, o0 = r - t0 * q.base0, e0 = min(q.base0, q.rows - t0 * q.base0);
    float u[16], m[16];
    read_columns(q, q.G, r < q.rows, t0, o0, e0, c0, u);
    if (g.mu >= 0.f) read_columns(q, q.M, r < q.rows, t0, o0, e0, c0, m);
    const Scale scaled(length_and_exponents(g, q, i0, j0, j0 == 0, i0 == 0, setup));
#pragma unroll
    for (int s = 0; s < 16; s++) {
        float x = u[s];
        if (g.mu >= 0.f) x = g.nesterov ? fmaf(g.mu, m[s], x) : m[s];
        const int c = wave * 16 + s;
        if (q.flip) t[c][lane] = x;
        else t[lane][c] = x;
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
            split(scaled(t[lane][k + e], kShiftX + setup.row[lane]), x, y);
            hi[e] = x;
            lo[e] = y;
        }
        char* d = g.space + q.X + panel_at(i0 + lane, j0 + k, q.np);
        *reinterpret_cast<f16x8*>(d) = hi;
        *reinterpret_cast<f16x8*>(d + kPartBytes) = lo;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            _Float16 x, y;
            split(scaled(t[k + e][lane], kShiftX + setup.column[lane]), x, y);
            hi[e] = x;
            lo[e] = y;
        }
        d = g.space + q.XT + panel_at(j0 + lane, i0 + k, q.mp);
        *reinterpret_cast<f16x8*>(d) = hi;
        *reinterpret_cast<f16x8*>(d + kPartBytes) = lo;
    }
    // a wavefront's block of 32 x 32
    const int wi = (wave & 1) * 32, wj = (wave >> 1) * 32;
    float4* E = reinterpret_cast<float4*>(g.space + q.E + block_at(i0 + wi, j0 + wj, q.mp));
#pragma unroll
    for (int b = 0; b < 4; b++) {
        const int i = wi + b * 8 + (lane >> 5) * 4, j = wj + (lane & 31);
        E[b * 64] = make_float4(scaled(t[i][j], 0), scaled(t[i + 1][j], 0), scaled(t[i + 2][j], 0), scaled(t[i + 3][j], 0));
    }
}

// ---------------------------------------------------------------- products
enum { kGram, kPoly, kPair, kStep, kLast };

// What a product of square matrices, or one with X, is made of.  The group's matrices have up to four square buffers each (0: A), that hold D p of a polynomial
// p in A without a constant term.  The `last` one of a step is what X is multiplied by: its diagonal goes into the coefficients, with `base` added.
//   kPoly  buffer d = mul (buffer p)(buffer q) + add (buffer e)
//   kPair  the same with two terms, add (buffer p) + add (buffer q), at a scale of 2^10 (it reaches some 32)
//   kStep  X = (buffer p) X + coefficients X;  kLast  the same, applied.  2^shift: the sums' scales
// Rows and columns of X have grown by up to 2^from before, and by 2^to behind it.
struct NsOp {
    int32_t p, q, e, d, last, from, to, shift;
    float mul, add, base;
};
constexpr int kPairShift = 2;             // 2^12 / 2^10

// One result's place in the tensor, found from its row and column of X.
__device__ __forceinline__ void apply_one(const NsMatrix& q, float x, int i, int j) {
    const int r = q.flip ? j : i, c = q.flip ? i : j;
    if (r >= q.rows || c >= q.cols) return;
    const int t0 = r / q.base0, t1 = c / q.base1, tile = t0 + q.grid0 * t1;
    const int64_t off = (r - t0 * q.base0) + (int64_t)min(q.base0, q.rows - t0 * q.base0) * (c - t1 * q.base1);
    if (q.step < 0.f) {
        if (q.P.dtype == NNT_F32) global_as<float>(q.P.tiles[tile])[off] = x;
        else global_as<bf16_t>(q.P.tiles[tile])[off] = f2bf(x);
        return;
    }
    float* p = global_as<float>(q.P.tiles[tile]) + off;
    const float v = fmaf(-q.step, x, q.decay * *p);
    *p = v;
    if (q.LP.tiles) global_as<bf16_t>(q.LP.tiles[tile])[off] = f2bf(v);
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));

// P <- decay P - step x, or P <- x, of a lane's results of a block: rows i + 8 p + 0 .. 3 of X, column j.  Four of them lie in one tile, next to each other or
// (X the transpose) a column apart, except where a tile or the matrix ends among them.  All reads are started before the first write.
__device__ __forceinline__ void apply_results(const NsMatrix& q, const float (&x)[4][4], int i, int j) {
    if (j >= (q.flip ? q.rows : q.cols)) return;
    const int extent = q.flip ? q.cols : q.rows, base_i = q.flip ? q.base1 : q.base0, base_j = q.flip ? q.base0 : q.base1;
    const int tj = j / base_j, oj = j - tj * base_j;
    const bool update = q.step >= 0.f, fp32 = q.P.dtype == NNT_F32;
    int tile[4];
    int64_t off[4];
    int64_t stride[4];
    bool even[4];
    RawVec<float> old[4];
#pragma unroll
    for (int p = 0; p < 4; p++) {
        const int ip = i + p * 8, ti = ip / base_i, oi = ip - ti * base_i;
        even[p] = ip + 4 <= extent && oi + 4 <= base_i;
        tile[p] = q.flip ? tj + q.grid0 * ti : ti + q.grid0 * tj;
        const int e0 = q.flip ? min(q.base0, q.rows - tj * q.base0) : min(q.base0, q.rows - ti * q.base0);
        off[p] = q.flip ? oj + (int64_t)e0 * oi : oi + (int64_t)e0 * oj;
        stride[p] = q.flip ? e0 : 1;
        if (update && even[p]) {
            const float* src = global_as<const float>(q.P.tiles[tile[p]]) + off[p];
            if (q.flip) {
#pragma unroll
                for (int k = 0; k < 4; k++) old[p].set(k, src[k * stride[p]]);
            } else {
                old[p].load(src, 4);
            }
        }
    }
#pragma unroll
    for (int p = 0; p < 4; p++) {
        if (!even[p]) {
#pragma unroll
            for (int k = 0; k < 4; k++) apply_one(q, x[p][k], i + p * 8 + k, j);
            continue;
        }
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; k++) v[k] = update ? fmaf(-q.step, x[p][k], q.decay * old[p].at(k)) : x[p][k];
        if (fp32) {
            float* d = global_as<float>(q.P.tiles[tile[p]]) + off[p];
            if (q.flip) {
#pragma unroll
                for (int k = 0; k < 4; k++) d[k * stride[p]] = v[k];
            } else {
                RawVec<float>::store(d, v, 4);
            }
        }
        if (!fp32 || q.LP.tiles) {
            bf16_t* d = global_as<bf16_t>((fp32 ? q.LP : q.P).tiles[tile[p]]) + off[p];
            if (q.flip) {
#pragma unroll
                for (int k = 0; k < 4; k++) d[k * stride[p]] = f2bf(v[k]);
            } else {
                u32x2 y;
                y[0] = (uint32_t)f2bf(v[0]) | ((uint32_t)f2bf(v[1]) << 16);
                y[1] = (uint32_t)f2bf(v[2]) | ((uint32_t)f2bf(v[3]) << 16);
                *reinterpret_cast<u32x2*>(d) = y;
            }
        }
    }
}

constexpr int turn_pitch(int FN) { return 32 * FN + 8; }         // in 32-bit words

// The result path of a wavefront for square matrices: FM x FN blocks of 32 x 32 from row i0 and column j0 on.  er, ec: the exponents of its rows and columns, from LDS.  `turn`: LDS
// for 32 rows, in which the sums change places.
template <int MODE, int FM, int FN>
__device__ __forceinline__ void store_square(const NsGroup& g, const NsMatrix& q, const f32x16 (&acc)[FM][FN], int i0, int j0, bool diagonal, const NsOp& op,
                                             const int* er, const int* ec, uint32_t* turn) {
    // results: this lane has column j0 + 32 y + (lane & 31), rows i0 + 32 x + 8 p + 4 (lane >> 5) + 0 .. 3
    constexpr int kPitch = turn_pitch(FN), kTerms = MODE == kGram ? 0 : MODE == kPair ? 2 : 1;
    const int lane = threadIdx.x & 63;
    const int64_t square = (int64_t)q.mp * q.mp * 4;
    // the terms that are added, laid out like the result
    const char* E[2] = {g.space + q.A + (MODE == kPoly ? op.e : op.p) * square, g.space + q.A + op.q * square};
    char* D = g.space + q.A + (MODE == kGram ? 0 : op.d * square);
    const float factor = MODE == kGram ? kGramFactor : op.mul / kScale;      // sums carry both factors' scales
    const float add = op.add;
    const bool fetches = kTerms > 0 && add != 0.f, last = MODE == kPair || (MODE == kPoly && op.last);
    constexpr int kDown = MODE == kPair ? kPairShift : 0;
    // what is added is fetched one block of 32 rows ahead: behind the stores that the compiler cannot tell apart from it every load would wait (two terms: no registers for that)
    constexpr int kAhead = kTerms == 1;
    f16x4 e[1 + kAhead][kTerms ? kTerms : 1][FN][4][2];
    f16x8 et[kTerms ? kTerms : 1][2 * FN][2];                          // the same with rows and columns exchanged
    // (blocks behind the last row block are not there)
    const int rows = q.mp;
    auto fetch = [&](int x) {
        if (i0 + x * 32 >= rows) return;
#pragma unroll
        for (int t = 0; t < kTerms; t++)
#pragma unroll
            for (int y = 0; y < FN; y++) {
                if (j0 + y * 32 >= rows) continue;
#pragma unroll
                for (int p = 0; p < 4; p++) {
                    const char* at = E[t] + panel_at(j0 + y * 32 + (lane & 31), i0 + x * 32 + p * 8, q.mp) + (lane >> 5) * 8;
                    e[x & kAhead][t][y][p][0] = *reinterpret_cast<const f16x4*>(at);
                    e[x & kAhead][t][y][p][1] = *reinterpret_cast<const f16x4*>(at + kPartBytes);
                }
            }
    };
    // (a lane's eight columns of `turn`, see below)
    const int turned_row = lane & 31, turned_col = (lane >> 5) * 8;
    auto fetch_turned = [&](int x) {
#pragma unroll
        for (int t = 0; t < kTerms; t++)
#pragma unroll
            for (int s = 0; s < 2 * FN; s++) {
                if (j0 + s / 2 * 32 >= rows) continue;
                const char* at = E[t] + panel_at(i0 + x * 32 + turned_row, j0 + s * 16 + turned_col, q.mp);
                et[t][s][0] = *reinterpret_cast<const f16x8*>(at);
                et[t][s][1] = *reinterpret_cast<const f16x8*>(at + kPartBytes);
            }
    };
    if (fetches && kAhead) fetch(0);
#pragma unroll
    for (int x = 0; x < FM; x++) {
        if (fetches && x + kAhead < FM) fetch(x + kAhead);
        if (i0 + x * 32 >= rows) continue;
        if (fetches && !diagonal) fetch_turned(x);
#pragma unroll
        for (int y = 0; y < FN; y++) {
            if (j0 + y * 32 >= rows) continue;
            const int i = i0 + x * 32 + (lane >> 5) * 4, j = j0 + y * 32 + (lane & 31);
            float v[4][4];
#pragma unroll
            for (int p = 0; p < 4; p++) {
                const int4 ei = *reinterpret_cast<const int4*>(er + x * 32 + p * 8 + (lane >> 5) * 4);
                const int ek[4] = {ei.x, ei.y, ei.z, ei.w};
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const float w = acc[x][y][p * 4 + k] * factor;
                    if (!diagonal) turn[(p * 8 + (lane >> 5) * 4 + k) * kPitch + y * 32 + (lane & 31)] = __float_as_uint(w);
                    v[p][k] = ldexpf(w, -ek[k]);
                    if (fetches)
#pragma unroll
                        for (int t = 0; t < kTerms; t++) v[p][k] = fmaf(add, (float)e[x & kAhead][t][y][p][0][k] + (float)e[x & kAhead][t][y][p][1][k], v[p][k]);
                }
            }
            if (MODE != kGram && last && diagonal) {
#pragma unroll
                for (int p = 0; p < 4; p++)
#pragma unroll
                    for (int k = 0; k < 4; k++)
                        if (i + p * 8 + k == j) {
                            reinterpret_cast<float*>(g.space + q.coefficients)[j] = op.base + ldexpf(v[p][k], -er[x * 32 + p * 8 + (lane >> 5) * 4 + k] - kShift);
                            v[p][k] = 0.f;
                        }
            }
#pragma unroll
            for (int p = 0; p < 4; p++) {
                f16x4 hi, lo;
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    _Float16 h, l;
                    split(kDown ? v[p][k] * (1.f / (1 << kDown)) : v[p][k], h, l);
                    hi[k] = h;
                    lo[k] = l;
                }
                char* d = D + panel_at(j, i0 + x * 32 + p * 8, q.mp) + (lane >> 5) * 8;
                *reinterpret_cast<f16x4*>(d) = hi;
                *reinterpret_cast<f16x4*>(d + kPartBytes) = lo;
            }
        }
        if (!diagonal) {
            // 32 rows of the wavefront's own sums, eight columns to a lane
#pragma unroll
            for (int s = 0; s < 2 * FN; s++) {
                if (j0 + s / 2 * 32 >= rows) continue;
                const int k = s * 16 + turned_col;
                const uint4 u = *reinterpret_cast<const uint4*>(turn + turned_row * kPitch + k), w = *reinterpret_cast<const uint4*>(turn + turned_row * kPitch + k + 4);
                const uint32_t sums[8] = {u.x, u.y, u.z, u.w, w.x, w.y, w.z, w.w};
                const int4 ea = *reinterpret_cast<const int4*>(ec + k), eb = *reinterpret_cast<const int4*>(ec + k + 4);
                const int ek[8] = {ea.x, ea.y, ea.z, ea.w, eb.x, eb.y, eb.z, eb.w};
                f16x8 hi, lo;
#pragma unroll
                for (int m = 0; m < 8; m++) {
                    float r = ldexpf(__uint_as_float(sums[m]), -ek[m]);
                    if (fetches)
#pragma unroll
                        for (int t = 0; t < kTerms; t++) r = fmaf(add, (float)et[t][s][0][m] + (float)et[t][s][1][m], r);
                    _Float16 h, l;
                    split(kDown ? r * (1.f / (1 << kDown)) : r, h, l);
                    hi[m] = h;
                    lo[m] = l;
                }
                char* d = D + panel_at(i0 + x * 32 + turned_row, j0 + k, q.mp);
                *reinterpret_cast<f16x8*>(d) = hi;
                *reinterpret_cast<f16x8*>(d + kPartBytes) = lo;
            }
        }
    }
}

// The same for X: fp32 results from X's form in fp32, from which the two others are made.  er, ec: the first exponents of X's rows and columns; cf: the rows' coefficients.
template <int MODE, int FM, int FN>
__device__ __forceinline__ void store_step(const NsGroup& g, const NsMatrix& q, const f32x16 (&acc)[FM][FN], int i0, int j0, int now, const NsOp& op,
                                           const int* er, const int* ec, const float* cf, uint32_t* turn) {
    constexpr int kPitch = turn_pitch(FN);
    const int lane = threadIdx.x & 63;
    char *XT = g.space + q.XT + (1 - now) * ((int64_t)q.mp * q.np * 4), *X = g.space + q.X;
    char* E = g.space + q.E;
    float4 e[2][FN][4];
    const int rows = q.mp, cols = q.np;
    auto fetch = [&](int x) {
        if (i0 + x * 32 >= rows) return;
#pragma unroll
        for (int y = 0; y < FN; y++) {
            if (j0 + y * 32 >= cols) continue;
            const float4* at = reinterpret_cast<const float4*>(E + block_at(i0 + x * 32, j0 + y * 32, q.mp));
#pragma unroll
            for (int p = 0; p < 4; p++) e[x & 1][y][p] = at[p * 64];
        }
    };
    fetch(0);
#pragma unroll
    for (int x = 0; x < FM; x++) {
        if (x + 1 < FM) fetch(x + 1);
        if (i0 + x * 32 >= rows) continue;
#pragma unroll
        for (int y = 0; y < FN; y++) {
            if (j0 + y * 32 >= cols) continue;
            const int i = i0 + x * 32, j = j0 + y * 32 + (lane & 31), column = ec[y * 32 + (lane & 31)], f = exponent_at(column, op.from);
            float v[4][4];
#pragma unroll
            for (int p = 0; p < 4; p++) {
                const int at = x * 32 + p * 8 + (lane >> 5) * 4;
                const int4 first = *reinterpret_cast<const int4*>(er + at);
                const float4 c = *reinterpret_cast<const float4*>(cf + at), old = e[x & 1][y][p];
                const int down = op.shift - f;
                v[p][0] = fmaf(c.x, old.x, ldexpf(acc[x][y][p * 4], down - exponent_at(first.x, op.from)));
                v[p][1] = fmaf(c.y, old.y, ldexpf(acc[x][y][p * 4 + 1], down - exponent_at(first.y, op.from)));
                v[p][2] = fmaf(c.z, old.z, ldexpf(acc[x][y][p * 4 + 2], down - exponent_at(first.z, op.from)));
                v[p][3] = fmaf(c.w, old.w, ldexpf(acc[x][y][p * 4 + 3], down - exponent_at(first.w, op.from)));
            }
            if constexpr (MODE == kLast) {
                apply_results(q, v, i + (lane >> 5) * 4, j);
            } else {
                const int up = kShiftX + exponent_at(column, op.to);
                float4* to = reinterpret_cast<float4*>(E + block_at(i, j0 + y * 32, q.mp));
#pragma unroll
                for (int p = 0; p < 4; p++) {
                    f16x4 hi, lo;
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        _Float16 h, l;
                        split(ldexpf(v[p][k], up), h, l);
                        hi[k] = h;
                        lo[k] = l;
                        turn[(p * 8 + (lane >> 5) * 4 + k) * kPitch + y * 32 + (lane & 31)] = __float_as_uint(v[p][k]);
                    }
                    to[p * 64] = make_float4(v[p][0], v[p][1], v[p][2], v[p][3]);
                    char* d = XT + panel_at(j, i + p * 8, q.mp) + (lane >> 5) * 8;
                    *reinterpret_cast<f16x4*>(d) = hi;
                    *reinterpret_cast<f16x4*>(d + kPartBytes) = lo;
                }
            }
        }
        if constexpr (MODE == kStep) {
            // 32 rows of the wavefront's own results, eight columns to a lane
            const int row = lane & 31, up = kShiftX + exponent_at(er[x * 32 + row], op.to);
#pragma unroll
            for (int s = 0; s < 2 * FN; s++) {
                if (j0 + s / 2 * 32 >= cols) continue;
                const int k = (s * 2 + (lane >> 5)) * 8;
                const uint4 u = *reinterpret_cast<const uint4*>(turn + row * kPitch + k), w = *reinterpret_cast<const uint4*>(turn + row * kPitch + k + 4);
                const uint32_t x8[8] = {u.x, u.y, u.z, u.w, w.x, w.y, w.z, w.w};
                f16x8 hi, lo;
#pragma unroll
                for (int m = 0; m < 8; m++) {
                    _Float16 h, l;
                    split(ldexpf(__uint_as_float(x8[m]), up), h, l);
                    hi[m] = h;
                    lo[m] = l;
                }
                char* d = X + panel_at(i0 + x * 32 + row, j0 + k, q.np);
                *reinterpret_cast<f16x8*>(d) = hi;
                *reinterpret_cast<f16x8*>(d + kPartBytes) = lo;
            }
        }
    }
}

// A macro-tile: WR x WC wavefronts of FM x FN results of 32 x 32 each, ST stages of KS panels (16 KS columns of the contraction) in LDS.
template <int FM_, int FN_, int WR_, int WC_, int KS_, int ST_>
struct Shape {
    static constexpr int FM = FM_, FN = FN_, WR = WR_, WC = WC_, KS = KS_, ST = ST_, kWaves = WR * WC;
    static constexpr int BM = 32 * FM * WR, BN = 32 * FN * WC;
    static constexpr int kStage = (BM + BN) / 64 * KS * kPanelBytes, kLoads = kStage / 1024 / kWaves;
    static constexpr int kTurn = 32 * turn_pitch(FN) * 4;
    static constexpr int kLds = ST * kStage > kWaves * kTurn ? ST * kStage : kWaves * kTurn;
    static_assert(BM == BN && kLoads * kWaves * 1024 == kStage && 4 * KS % kLoads == 0, "symmetric results need square tiles, a wavefront's loads one row block");
    static_assert((ST - 1) * kLoads < 64, "loads in flight are counted in six bits");
};
using Large = Shape<4, 2, 2, 4, 1, 4>;       // one workgroup per compute unit
using Middle = Shape<2, 2, 2, 2, 1, 4>;      // two
using Small = Shape<1, 1, 2, 2, 1, 6>;       // three

template <int OFFSET>
__device__ __forceinline__ void read_fragment(f16x8& f, uint32_t addr) {
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f) : "v"(addr), "n"(OFFSET));
}

// what uses these stays behind the wait in front of this
__device__ __forceinline__ void hold(f16x8& a, f16x8& b) { asm volatile("" : "+v"(a), "+v"(b)); }

// Tiles of a launch in an order in which neighbours share operands: eight rows of tiles at a time, column by column.  Of a symmetric result the
// tiles on and above the diagonal.
template <bool SYM>
__device__ __forceinline__ void tile_of(int p, int tm, int tn, int& ti, int& tj) {
    for (int r0 = 0;; r0 += 8) {
        const int rows = min(8, tm - r0);
        if constexpr (SYM) {
            const int corner = rows * (rows + 1) / 2, count = corner + rows * (tn - r0 - rows);
            if (p < count) {
                if (p >= corner) {
                    tj = r0 + rows + (p - corner) / rows;
                    ti = r0 + (p - corner) % rows;
                } else {
                    int c = 0;
                    while ((c + 1) * (c + 2) / 2 <= p) c++;
                    tj = r0 + c;
                    ti = r0 + p - c * (c + 1) / 2;
                }
                return;
            }
            p -= count;
        } else {
            const int count = rows * tn;
            if (p < count) {
                tj = p / rows;
                ti = r0 + p % rows;
                return;
            }
            p -= count;
        }
    }
}

// One workgroup computes a macro-tile.  Of the symmetric results only tiles on and above the diagonal are computed, and written twice.
//
// Stages of 16 columns go from memory straight into LDS, ST of them, so that loads have ST - 1 steps to land; the fragments of the next step
// are read under the matrix instructions of the present one, into the other of two register sets.  At the top of a step every wavefront waits for
// its fragments and for its own loads of the next step; the barrier behind that makes the next stage complete for everybody and the present one, whose
// fragments all have, free for the loads of step + ST.  LDS reads and their waits are spelled out: the compiler would wait for all loads in flight.
//
// What bounds it: 8192 x 8192, B X on 256 x 256: 2.44 ms, 1350 TFLOP/s of fp16 (a plain fp16 product of the installed library: 1180), by the clock that the power limit
// leaves (1.55 GHz, the matrix cores busy for 81 % of the cycles).  Twelve of 768 x 768 on 128 x 128: 48 us, 680 TFLOP/s of fp16, half of it in the loop and half in
// the launch, the filling of the stages and the results' way out.  777 x 1111 on 64 x 64: 11 us, of which the loop takes 7, as long as it takes to
// fetch 8 KB a step at 32 bytes per clock.
template <int MODE, typename S>
__global__ void __launch_bounds__(64 * S::kWaves, 2) ns_product_kernel(const NsGroup* __restrict__ group, NsSizes sizes, NsOp op, int now, int splits) {
    const NsGroup& g = *group;
    constexpr int FM = S::FM, FN = S::FN, ST = S::ST;
    constexpr bool kSym = MODE == kGram || MODE == kPoly || MODE == kPair;
    __shared__ __align__(1024) char lds[S::kLds];
    __shared__ __align__(16) int ex[S::BM + S::BN];
    __shared__ __align__(16) float cf[kSym ? 4 : S::BM];
    static_assert(S::BM + S::BN <= 64 * S::kWaves, "a thread fetches one exponent");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave % S::WR, wc = wave / S::WR;
    // workgroups go to the eight dies in turn: each die gets one run of the tiles
    int wg = blockIdx.x;
    {
        const int total = gridDim.x, per = total / 8, rest = total % 8, die = wg % 8;
        wg = die * per + min(die, rest) + wg / 8;
    }
    // A's contraction may be cut: the tiles of one part lie side by side, so that a die finds most of what they share in its own cache
    int part = 0;
    if constexpr (MODE == kGram) {
        const int tiles = gridDim.x / splits;
        part = wg / tiles;
        wg -= part * tiles;
    }
    const int tile = wg;                                         // of all matrices
    const NsMatrix& q = g.mat[matrix_of<kSym, S::BM>(sizes, wg)];
    const int tm = (q.mp + S::BM - 1) / S::BM;
    int ti, tj;
    tile_of<kSym>(wg, tm, kSym ? tm : (q.np + S::BN - 1) / S::BN, ti, tj);
    ti = __builtin_amdgcn_readfirstlane(ti);
    tj = __builtin_amdgcn_readfirstlane(tj);
    const int64_t xbytes = (int64_t)q.mp * q.np * 4;
    const int nk = (MODE == kGram ? q.np : q.mp) >> 4;           // panels along the contraction, a multiple of 4
    const int64_t square = (int64_t)q.mp * q.mp * 4;
    const char* Pb = g.space + (MODE == kGram ? q.X : q.A + op.p * square);
    const char* Qb = g.space + (MODE == kGram ? q.X : kSym ? q.A + op.q * square : q.XT + now * xbytes);

    // a thread's row or column (older than the loads that are counted below, which they can only make wait longer)
    const int mine = tid < S::BM ? min(ti * S::BM + tid, q.mp - 1) : min(tj * S::BN + tid - S::BM, (kSym ? q.mp : q.np) - 1);
    const int exponent = reinterpret_cast<const int*>(g.space + (kSym || tid < S::BM ? q.exponents : q.columns))[mine];
    float coefficient = 0.f;
    if constexpr (!kSym) coefficient = reinterpret_cast<const float*>(g.space + q.coefficients)[min(mine, q.mp - 1)];

    // a wavefront loads a part of one row block's panels per step
    const char* src;
    {
        constexpr int kRB = S::BM / 64;
        const int blk = wave * S::kLoads / (4 * S::KS), sub = wave * S::kLoads % (4 * S::KS);
        // (a tile may end behind the last row block: that one is loaded again, its results are not stored)
        const int row = blk < kRB ? min(ti * kRB + blk, (q.mp >> 6) - 1) : min(tj * kRB + blk - kRB, ((kSym ? q.mp : q.np) >> 6) - 1);
        src = (blk < kRB ? Pb : Qb) + (int64_t)row * nk * kPanelBytes + sub * 1024;
    }
    int steps = nk / S::KS;
    if constexpr (MODE == kGram) {
        const int from = (int)((int64_t)steps * part / splits);
        steps = (int)((int64_t)steps * (part + 1) / splits) - from;
        src += (int64_t)from * S::KS * kPanelBytes;
        if (steps == 0 && from > 0) src -= S::KS * kPanelBytes;      // (more parts than steps: fetches one that it does not use)
    }
    int left = steps;                                            // steps whose loads have not been started
    auto load_one = [&](int stage, int l) {
        __builtin_amdgcn_global_load_lds((glb_void_ptr)(src + l * 1024 + lane * 16), (lds_void_ptr)(lds + stage * S::kStage + (wave * S::kLoads + l) * 1024), 16, 0, 0);
    };
    // (loads are started in every step, so that the count in flight is the same at every wait: the last steps fetch the last one again)
    auto advance = [&]() {
        if (--left > 0) src += S::KS * kPanelBytes;
    };
    f32x16 acc[FM][FN];
#pragma unroll
    for (int x = 0; x < FM; x++)
#pragma unroll
        for (int y = 0; y < FN; y++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[x][y][r] = 0.f;

    constexpr int KS = S::KS, kFrags = KS * 2 * (FM + FN), kMfma = KS * 3 * FM * FN, kBlock = KS * kPanelBytes;
    f16x8 pf[2][KS][FM][2], qf[2][KS][FN][2];
    const uint32_t lane_at = lds_offset(lds) + (lane & 31) * 16 + (lane >> 5) * 1024;
    const uint32_t p_at = lane_at + (FM == 1 ? wr * 512 : wr * (FM / 2) * kBlock);
    const uint32_t q_at = lane_at + S::BM / 64 * kBlock + (FN == 1 ? wc * 512 : wc * (FN / 2) * kBlock);
    // fragment I of a stage; of a panel the hi parts first, which are multiplied first
    auto frag_one = [&](auto I, int set, uint32_t stage) {
        constexpr int i = decltype(I)::value, ks = i / (2 * (FM + FN)), part = i / (FM + FN) % 2, k = i % (FM + FN);
        constexpr int at = ks * kPanelBytes + part * kPartBytes;
        if constexpr (k < FN) read_fragment<(k >> 1) * kBlock + (k & 1) * 512 + at>(qf[set][ks][k][part], q_at + stage);
        else read_fragment<((k - FN) >> 1) * kBlock + ((k - FN) & 1) * 512 + at>(pf[set][ks][k - FN][part], p_at + stage);
    };
    auto wait_frags = [&](int set) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int ks = 0; ks < KS; ks++) {
#pragma unroll
            for (int k = 0; k < FM; k++) hold(pf[set][ks][k][0], pf[set][ks][k][1]);
#pragma unroll
            for (int k = 0; k < FN; k++) hold(qf[set][ks][k][0], qf[set][ks][k][1]);
        }
    };
    int stage = 0;                                               // of the present step
    auto step = [&](int set) {
        wait_frags(set);
        __builtin_amdgcn_s_waitcnt(wait_vm((ST - 2) * S::kLoads));
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        const int next = stage + 1 == ST ? 0 : stage + 1;
        const uint32_t next_at = (uint32_t)(next * S::kStage);
        static_for<kMfma>([&](auto Q) {
            constexpr int m = decltype(Q)::value, ks = m / (3 * FM * FN), term = m / (FM * FN) % 3, x = m % (FM * FN) / FN, y = m % FN;
            // hi hi, hi lo, lo hi
            acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pf[set][ks][x][term == 2], qf[set][ks][y][term == 1], acc[x][y], 0, 0, 0);
            static_for<kFrags + S::kLoads>([&](auto I) {
                constexpr int i = decltype(I)::value;
                constexpr int slot = i < kFrags ? i * kMfma / 2 / kFrags : (i - kFrags) * kMfma / S::kLoads;
                if constexpr (slot == m) {
                    if constexpr (i < kFrags) frag_one(I, set ^ 1, next_at);
                    else load_one(stage, i - kFrags);
                }
            });
            __builtin_amdgcn_sched_barrier(0);
        });
        advance();
        stage = next;
    };
#pragma unroll
    for (int s = 0; s < ST; s++) {
#pragma unroll
        for (int l = 0; l < S::kLoads; l++) load_one(s, l);
        advance();
    }
    __builtin_amdgcn_s_waitcnt(wait_vm((ST - 1) * S::kLoads));
    asm volatile("s_barrier" ::: "memory");
    static_for<kFrags>([&](auto I) { frag_one(I, 0, 0u); });
    for (int k = 0; k < steps; k += 2) {
        step(0);
        if (MODE != kGram || k + 1 < steps) step(1);             // (whole contractions have an even number of steps)
    }
    // nothing may still be on its way into fragment registers or LDS (the last step has read a stage that nobody needs)
    wait_frags(0);
    wait_frags(1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    asm volatile("s_barrier" ::: "memory");

    if constexpr (MODE == kGram) {
        if (splits > 1) {
            // partial sums leave as they lie in registers
            float4* d = reinterpret_cast<float4*>(g.space + g.partial) + ((int64_t)(tile * splits + part) * S::kWaves + wave) * (FM * FN * 256) + lane;
#pragma unroll
            for (int x = 0; x < FM; x++)
#pragma unroll
                for (int y = 0; y < FN; y++)
#pragma unroll
                    for (int v = 0; v < 4; v++) d[((x * FN + y) * 4 + v) * 64] = make_float4(acc[x][y][4 * v], acc[x][y][4 * v + 1], acc[x][y][4 * v + 2], acc[x][y][4 * v + 3]);
            return;
        }
    }
    if (tid < S::BM + S::BN) ex[tid] = kSym ? exponent_at(exponent, op.from) : exponent;
    if (!kSym && tid < S::BM) cf[tid] = coefficient;
    __syncthreads();
    const int ri = wr * 32 * FM, cj = wc * 32 * FN;
    uint32_t* turn = reinterpret_cast<uint32_t*>(lds + wave * S::kTurn);
    if constexpr (kSym) store_square<MODE, FM, FN>(g, q, acc, ti * S::BM + ri, tj * S::BN + cj, ti == tj, op, ex + ri, ex + S::BM + cj, turn);
    else store_step<MODE, FM, FN>(g, q, acc, ti * S::BM + ri, tj * S::BN + cj, now, op, ex + ri, ex + S::BM + cj, cf + ri, turn);
}

// Adds up the parts of A's tiles, in their order: a wavefront takes one block of 32 x 32.
template <typename S>
__global__ void __launch_bounds__(256) ns_combine_kernel(const NsGroup* __restrict__ group, NsSizes sizes, NsOp op, int splits) {
    const NsGroup& g = *group;
    __shared__ __align__(16) uint32_t turn[4 * 32 * turn_pitch(1)];
    __shared__ __align__(16) int ex[4][64];                 // of a wavefront's 32 rows and 32 columns
    constexpr int kBlocks = S::kWaves * S::FM * S::FN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = blockIdx.x / (kBlocks / 4), blk = blockIdx.x % (kBlocks / 4) * 4 + wave;
    int wg = tile;
    const NsMatrix& q = g.mat[matrix_of<true, S::BM>(sizes, wg)];
    const int tm = (q.mp + S::BM - 1) / S::BM;
    int ti, tj;
    tile_of<true>(wg, tm, tm, ti, tj);
    const float4* d = reinterpret_cast<const float4*>(g.space + g.partial) + ((int64_t)tile * splits * kBlocks + blk) * 256 + lane;
    float4 t[4];
#pragma unroll
    for (int v = 0; v < 4; v++) t[v] = d[v * 64];
#pragma unroll 4
    for (int part = 1; part < splits; part++) {
#pragma unroll
        for (int v = 0; v < 4; v++) {
            const float4 u = d[(int64_t)part * kBlocks * 256 + v * 64];
            t[v].x += u.x;
            t[v].y += u.y;
            t[v].z += u.z;
            t[v].w += u.w;
        }
    }
    f32x16 acc[1][1];
#pragma unroll
    for (int v = 0; v < 4; v++) {
        acc[0][0][4 * v] = t[v].x;
        acc[0][0][4 * v + 1] = t[v].y;
        acc[0][0][4 * v + 2] = t[v].z;
        acc[0][0][4 * v + 3] = t[v].w;
    }
    const int w = blk / (S::FM * S::FN), x = blk / S::FN % S::FM, y = blk % S::FN;
    const int i0 = ti * S::BM + (w % S::WR * S::FM + x) * 32, j0 = tj * S::BN + (w / S::WR * S::FN + y) * 32;
    ex[wave][lane] = exponent_at(reinterpret_cast<const int*>(g.space + q.exponents)[min((lane < 32 ? i0 : j0 - 32) + lane, q.mp - 1)], op.from);
    __syncthreads();
    store_square<kGram, 1, 1>(g, q, acc, i0, j0, ti == tj, op, ex[wave], ex[wave] + 32, turn + wave * 32 * turn_pitch(1));
}

// ---------------------------------------------------------------- matrices with a side of at most 64
// Here a launch is longer than what it computes, so a whole iteration is one launch.  A workgroup holds some of X's column blocks of 64; it adds up the
// parts of A that the workgroups have left (its own and the others'), computes B (64 x 64, every workgroup the same), its blocks of X and their
// part of the next A.  X is kept as its transpose and in fp32.  The first launch takes U in place of B X, the last one leaves the results.  64 x 320: 7 us a
// launch, 49 in all (some 75 with the products above); it is the launches that bound it, and within one the parts' way through memory.
enum { kFirst, kMiddle, kFinal };

// how many workgroups share a matrix of nt column blocks: each adds up as many parts (0.2 us) as there are, and takes nt / parts blocks (1.5 us) in turn
__host__ __device__ inline int narrow_parts(int nt) { return nt <= 16 ? nt : nt <= 64 ? 16 : 32; }
constexpr int kNarrowBlocks = 256;                       // longer matrices take the products above

constexpr int kImage = 4 * kPanelBytes;                  // 64 x 64: four panels
__device__ __forceinline__ int image_at(int row, int k) { return (k >> 4) * kPanelBytes + ((k & 15) >> 3) * 1024 + row * 16 + (k & 7) * 2; }

// A wavefront's block of 32 x 32 of the product of two images: rows r0 of the first, rows c0 of the second, over all 64 columns.
template <typename LoadQ>
__device__ __forceinline__ void multiply(const char* image, int r0, LoadQ&& second, f32x16& acc) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int ks = 0; ks < 4; ks++) {
        const char* p = image + ks * kPanelBytes + (lane >> 5) * 1024 + (r0 + (lane & 31)) * 16;
        const f16x8 ph = *reinterpret_cast<const f16x8*>(p), pl = *reinterpret_cast<const f16x8*>(p + kPartBytes);
        f16x8 qh, ql;
        second(ks, qh, ql);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, qh, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph, ql, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl, qh, acc, 0, 0, 0);
    }
}
__device__ __forceinline__ void multiply(const char* image, int r0, const char* second, int c0, f32x16& acc) {
    const int lane = threadIdx.x & 63;
    multiply(image, r0, [&](int ks, f16x8& qh, f16x8& ql) {
        const char* p = second + ks * kPanelBytes + (lane >> 5) * 1024 + (c0 + (lane & 31)) * 16;
        qh = *reinterpret_cast<const f16x8*>(p);
        ql = *reinterpret_cast<const f16x8*>(p + kPartBytes);
    }, acc);
}

// A lane's results of a block of 64 x 64: rows i + 8 p + 0 .. 3, column j.
// The exponents of a lane's rows i .. i + 3, from LDS, where rows have grown by 2^grown.
struct RowExponents {
    const int* first;
    int grown;
    __device__ __forceinline__ void at(int i, int (&e)[4]) const {
        const int4 f = *reinterpret_cast<const int4*>(first + i);
        e[0] = exponent_at(f.x, grown);
        e[1] = exponent_at(f.y, grown);
        e[2] = exponent_at(f.z, grown);
        e[3] = exponent_at(f.w, grown);
    }
};
// A symmetric block D p D as the image of D p: four rows of a column are four columns of a row.  `coefficients`: where the diagonal goes, with `base` added (B).
__device__ __forceinline__ void store_symmetric(char* dst, const float (&x)[4][4], const RowExponents& rows, int i, int j, float* coefficients = nullptr, float base = 0.f) {
#pragma unroll
    for (int p = 0; p < 4; p++) {
        int e[4];
        rows.at(i + p * 8, e);
        f16x4 hi, lo;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            float w = ldexpf(x[p][k], -e[k]);
            if (coefficients && i + p * 8 + k == j) {
                coefficients[j] = base + ldexpf(w, -e[k] - kShift);
                w = 0.f;
            }
            _Float16 h, l;
            split(w, h, l);
            hi[k] = h;
            lo[k] = l;
        }
        char* d = dst + image_at(j, i + p * 8);
        *reinterpret_cast<f16x4*>(d) = hi;
        *reinterpret_cast<f16x4*>(d + kPartBytes) = lo;
    }
}
// X's block as its transpose, with its column's exponent f, and as it is, with its rows' exponents.
__device__ __forceinline__ void store_both(char* XT, char* X, const float (&x)[4][4], const RowExponents& rows, int f, int i, int j) {
#pragma unroll
    for (int p = 0; p < 4; p++) {
        int e[4];
        rows.at(i + p * 8, e);
        f16x4 hi, lo;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            _Float16 h, l;
            split(ldexpf(x[p][k], kShiftX + e[k]), h, l);
            char* d = X + image_at(i + p * 8 + k, j);
            *reinterpret_cast<_Float16*>(d) = h;
            *reinterpret_cast<_Float16*>(d + kPartBytes) = l;
            split(ldexpf(x[p][k], kShiftX + f), h, l);
            hi[k] = h;
            lo[k] = l;
        }
        char* d = XT + image_at(j, i + p * 8);
        *reinterpret_cast<f16x4*>(d) = hi;
        *reinterpret_cast<f16x4*>(d + kPartBytes) = lo;
    }
}
// x <- coefficients x + B X of X's block, f: the exponent of this lane's column
__device__ __forceinline__ void step_block(const char* B, const char* XT, int wr, int wc, int i, const float* coefficients, const RowExponents& rows, int f, float (&x)[4][4]) {
    f32x16 acc;
#pragma unroll
    for (int k = 0; k < 16; k++) acc[k] = 0.f;
    multiply(B, wr * 32, XT, wc * 32, acc);
#pragma unroll
    for (int p = 0; p < 4; p++) {
        const float4 c = *reinterpret_cast<const float4*>(coefficients + i + p * 8);
        int e[4];
        rows.at(i + p * 8, e);
        x[p][0] = fmaf(c.x, x[p][0], ldexpf(acc[p * 4], -kShift - kShiftX - f - e[0]));
        x[p][1] = fmaf(c.y, x[p][1], ldexpf(acc[p * 4 + 1], -kShift - kShiftX - f - e[1]));
        x[p][2] = fmaf(c.z, x[p][2], ldexpf(acc[p * 4 + 2], -kShift - kShiftX - f - e[2]));
        x[p][3] = fmaf(c.w, x[p][3], ldexpf(acc[p * 4 + 3], -kShift - kShiftX - f - e[3]));
    }
}

template <int PHASE>
__global__ void __launch_bounds__(256) ns_narrow_kernel(const NsGroup* __restrict__ group, NsSizes sizes, int step) {
    const NsGroup& g = *group;
    __shared__ __align__(16) char image[3][kImage];      // A (set-up: U in fp32), B, X's block with its rows along the contraction
    __shared__ __align__(16) SetUp setup;
    __shared__ __align__(16) float coefficients[64];
    const int now = step & 1;                            // the sums' buffer of this step
    const int nt = sizes.blocks[blockIdx.y] >> 16, parts = narrow_parts(nt), part = blockIdx.x;
    if (part >= parts) return;
    const NsMatrix& q = g.mat[blockIdx.y];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave & 1, wc = wave >> 1;
    float4* sums = reinterpret_cast<float4*>(g.space + q.A);             // two buffers of `parts` images of 64 x 64 in fp32, as they lie in registers
    auto sum_at = [&](int buffer, int p, int v) { return (((int64_t)buffer * parts + p) * 4 + wave) * 256 + v * 64 + lane; };
    const int i = wr * 32 + (lane >> 5) * 4, j = wc * 32 + (lane & 31);    // this lane's results: rows i + 8 p + 0 .. 3, column j of a block
    double length = 1.0;
    const RowExponents rows{setup.row, grown_by(g.growth, step)};
    if constexpr (PHASE == kFirst) {
        length = length_and_exponents(g, q, 0, -1, part == 0, false, setup);
    } else {
        if (tid < 64) setup.row[tid] = reinterpret_cast<const int*>(g.space + q.exponents)[tid];
        float4 t[4];
#pragma unroll
        for (int v = 0; v < 4; v++) t[v] = sums[sum_at(now, 0, v)];
#pragma unroll 4
        for (int p = 1; p < parts; p++) {
#pragma unroll
            for (int v = 0; v < 4; v++) {
                const float4 u = sums[sum_at(now, p, v)];
                t[v].x += u.x;
                t[v].y += u.y;
                t[v].z += u.z;
                t[v].w += u.w;
            }
        }
        float a[4][4];
#pragma unroll
        for (int p = 0; p < 4; p++) {
            a[p][0] = t[p].x * kGramFactor;
            a[p][1] = t[p].y * kGramFactor;
            a[p][2] = t[p].z * kGramFactor;
            a[p][3] = t[p].w * kGramFactor;
        }
        __syncthreads();
        store_symmetric(image[0], a, rows, i, j);
        __syncthreads();
        f32x16 acc;
#pragma unroll
        for (int k = 0; k < 16; k++) acc[k] = 0.f;
        multiply(image[0], wr * 32, image[0], wc * 32, acc);
#pragma unroll
        for (int p = 0; p < 4; p++)
#pragma unroll
            for (int k = 0; k < 4; k++) a[p][k] = fmaf(g.b, a[p][k], acc[p * 4 + k] * (g.c / kScale));
        store_symmetric(image[1], a, rows, i, j, coefficients, g.a);
        __syncthreads();
    }
    f32x16 gram;
#pragma unroll
    for (int k = 0; k < 16; k++) gram[k] = 0.f;
    for (int t = part * nt / parts; t < (part + 1) * nt / parts; t++) {
        char* XT = in_global(g.space + q.XT + (int64_t)t * kImage);
        float4* E = reinterpret_cast<float4*>(in_global(g.space + q.E + block_at(wr * 32, t * 64 + wc * 32, 64)));
        float x[4][4];
        if constexpr (PHASE == kFirst) {
            float (*u)[65] = reinterpret_cast<float (*)[65]>(image[0]);      // [i][j] (16640 bytes: reaches into the second image, which is free)
            const int r0 = q.flip ? t * 64 : 0, c0 = (q.flip ? 0 : t * 64) + wave * 16;
            const int r = r0 + lane, t0 = min(r, q.rows - 1) / q.base0, o0 = r - t0 * q.base0, e0 = min(q.base0, q.rows - t0 * q.base0);
            float y[16], m[16];
            read_columns(q, q.G, r < q.rows, t0, o0, e0, c0, y);
            if (g.mu >= 0.f) read_columns(q, q.M, r < q.rows, t0, o0, e0, c0, m);
            largest_of_columns(g, q, t * 64, setup);
            const Scale scaled(length);
#pragma unroll
            for (int s = 0; s < 16; s++) {
                if (g.mu >= 0.f) y[s] = g.nesterov ? fmaf(g.mu, m[s], y[s]) : m[s];
                if (q.flip) u[wave * 16 + s][lane] = scaled(y[s], 0);
                else u[lane][wave * 16 + s] = scaled(y[s], 0);
            }
            __syncthreads();
            if (wave == 0) column_exponents(g, q, t * 64, true, length, setup);
            __syncthreads();
#pragma unroll
            for (int p = 0; p < 4; p++) {
#pragma unroll
                for (int k = 0; k < 4; k++) x[p][k] = u[i + p * 8 + k][j];
                E[p * 64] = make_float4(x[p][0], x[p][1], x[p][2], x[p][3]);
            }
            store_both(XT, image[2], x, rows, setup.column[j], i, j);
        } else {
            const int column = reinterpret_cast<const int*>(g.space + q.columns)[t * 64 + j];
#pragma unroll
            for (int p = 0; p < 4; p++) {
                const float4 y = E[p * 64];
                x[p][0] = y.x;
                x[p][1] = y.y;
                x[p][2] = y.z;
                x[p][3] = y.w;
            }
            step_block(image[1], XT, wr, wc, i, coefficients, rows, exponent_at(column, rows.grown), x);
            if constexpr (PHASE == kFinal) {
                apply_results(q, x, i, t * 64 + j);
                continue;
            }
#pragma unroll
            for (int p = 0; p < 4; p++) E[p * 64] = make_float4(x[p][0], x[p][1], x[p][2], x[p][3]);
            __syncthreads();                             // everybody has read X's block, which is overwritten, and is done with the last one's image
            const RowExponents next{setup.row, grown_by(g.growth, step + 1)};
            store_both(XT, image[2], x, next, exponent_at(column, next.grown), i, j);
        }
        __syncthreads();
        multiply(image[2], wr * 32, image[2], wc * 32, gram);
        if constexpr (PHASE == kFirst) __syncthreads();  // (before the next block's U and image)
    }
    if constexpr (PHASE != kFinal) {
        const int next = PHASE == kFirst ? now : 1 - now;
#pragma unroll
        for (int v = 0; v < 4; v++) sums[sum_at(next, part, v)] = make_float4(gram[4 * v], gram[4 * v + 1], gram[4 * v + 2], gram[4 * v + 3]);
    }
}

// ---------------------------------------------------------------- matrices of at most 64 x 256
// One workgroup holds all of X in LDS and does everything in one launch: momentum, norm, the steps, the results.  Four wavefronts to a column block of 64; the first four
// put A together and compute B for all.  64 x 64 25 us (33 with a launch per step), 64 x 256 44 (49), and the rest of the chip is free meanwhile: passes over the four
// matrices of a block of 64 that need not wait for one another take 28 us each (47).  What bounds it is LDS, 3 us a step and 1.2 for each further block.  (X computed
// twice, as its transpose too, in place of the two-byte writes: 40 us, but the two drift apart, errors a quarter larger.)
constexpr int kHeldBlocks = 4;

__global__ void __launch_bounds__(256 * kHeldBlocks) ns_held_kernel(NsGroup g, int steps) {
    __shared__ __align__(16) char images[2 * kHeldBlocks + 1][kImage];       // X's transpose and X by block; A, then B
    __shared__ double red[4 * kHeldBlocks][64];          // sums of squares of X's rows
    __shared__ __align__(16) int exponent[64];
    __shared__ __align__(16) float coefficients[64];
    __shared__ float largest[kHeldBlocks][4][64];        // of X's columns
    const NsMatrix& q = g.mat[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane((tid >> 6) & 3), t = __builtin_amdgcn_readfirstlane(tid >> 8);
    const int wr = wave & 1, wc = wave >> 1, nt = q.np >> 6;
    const int i = wr * 32 + (lane >> 5) * 4, j = wc * 32 + (lane & 31);
    const bool mine = t < nt;                            // (the launch has as many wavefronts as its longest matrix wants)
    char *XT = images[t], *X = images[kHeldBlocks + t], *S = images[2 * kHeldBlocks];
    float x[4][4];                                       // X in fp32, from step to step
    int column;                                          // the first exponent of this lane's column
    {
        const int r0 = q.flip ? t * 64 : 0, c0 = (q.flip ? 0 : t * 64) + wave * 16;
        const int r = r0 + lane, t0 = min(r, q.rows - 1) / q.base0, o0 = r - t0 * q.base0, e0 = min(q.base0, q.rows - t0 * q.base0);
        const bool there = mine && r < q.rows;
        float u[16];
        read_columns(q, q.G, there, t0, o0, e0, c0, u);
        if (g.mu >= 0.f) {
            float m[16];
            read_columns(q, q.M, there, t0, o0, e0, c0, m);
#pragma unroll
            for (int s = 0; s < 16; s++) {
                m[s] = fmaf(g.mu, m[s], u[s]);
                u[s] = g.nesterov ? fmaf(g.mu, m[s], u[s]) : m[s];
            }
            write_columns(q, q.M.tiles, there, t0, o0, e0, c0, m);
        }
        // a lane has a row of X and 16 columns of it, or (X the transpose) a column and 16 rows
        double square[16];
#pragma unroll
        for (int s = 0; s < 16; s++) square[s] = (double)u[s] * (double)u[s];
        if (q.flip) {
            const double x = sum16(square, lane);
            if ((lane & 3) == 0) red[t][wave * 16 + sum16_index(lane)] = x;
            largest[t][wave][lane] = largest_of(u);
        } else {
#pragma unroll
            for (int s = 1; s < 16; s++) square[0] += square[s];
            red[tid >> 6][lane] = square[0];
            const uint32_t x = largest16(u, lane);
            if ((lane & 7) == 0) {
                largest[t][0][wave * 16 + (lane >> 3)] = from_upper_half(x & 0xffffu);
                largest[t][0][wave * 16 + 8 + (lane >> 3)] = from_upper_half(x >> 16);
            }
        }
        __syncthreads();
        double row = 0.0;
        for (int w = 0; w < (q.flip ? nt : 4 * nt); w++) row += red[w][lane];
        double sum = row;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        const double length = sqrt(sum) + g.eps;         // (every wavefront by itself, in the same order)
        if (tid < 64) exponent[lane] = exponent_of(sqrt(row), length);
        const float most = q.flip ? fmaxf(fmaxf(largest[t][0][j], largest[t][1][j]), fmaxf(largest[t][2][j], largest[t][3][j])) : largest[t][0][j];
        column = exponent_of((double)most * 8.0, length);
        // through LDS to this lane's results: column c of X's block is 64 floats, in an order in which neither way has many conflicts
        const Scale scaled(length);
        float* turn = reinterpret_cast<float*>(X);
        auto at = [](int row, int c) { return c * 64 + (row ^ ((c & 15) << 2)); };
#pragma unroll
        for (int s = 0; s < 16; s++) turn[q.flip ? at(wave * 16 + s, lane) : at(lane, wave * 16 + s)] = scaled(u[s], 0);
        __syncthreads();
#pragma unroll
        for (int p = 0; p < 4; p++) {
            const float4 y = *reinterpret_cast<const float4*>(turn + at(i + p * 8, j));
            x[p][0] = y.x;
            x[p][1] = y.y;
            x[p][2] = y.z;
            x[p][3] = y.w;
        }
    }
    RowExponents rows{exponent, 0};
    __syncthreads();
    if (mine) store_both(XT, X, x, rows, column, i, j);
    for (int step = 0;; step++) {
        __syncthreads();
        f32x16 acc;
#pragma unroll
        for (int k = 0; k < 16; k++) acc[k] = 0.f;
        if (mine) multiply(X, wr * 32, X, wc * 32, acc);
        __syncthreads();                                 // X's image has been read: the blocks' parts of A take its place
        auto part_at = [&](int block, int v) { return reinterpret_cast<float4*>(images[kHeldBlocks + block]) + (wave * 4 + v) * 64 + lane; };
        if (mine && t > 0)
#pragma unroll
            for (int v = 0; v < 4; v++) *part_at(t, v) = make_float4(acc[4 * v], acc[4 * v + 1], acc[4 * v + 2], acc[4 * v + 3]);
        __syncthreads();
        float a[4][4];
        if (t == 0) {
            for (int b = 1; b < nt; b++)
#pragma unroll
                for (int v = 0; v < 4; v++) {
                    const float4 y = *part_at(b, v);
                    acc[4 * v] += y.x;
                    acc[4 * v + 1] += y.y;
                    acc[4 * v + 2] += y.z;
                    acc[4 * v + 3] += y.w;
                }
#pragma unroll
            for (int p = 0; p < 4; p++)
#pragma unroll
                for (int k = 0; k < 4; k++) a[p][k] = acc[p * 4 + k] * kGramFactor;
            store_symmetric(S, a, rows, i, j);
        }
        __syncthreads();
        if (t == 0) {
#pragma unroll
            for (int k = 0; k < 16; k++) acc[k] = 0.f;
            multiply(S, wr * 32, S, wc * 32, acc);
#pragma unroll
            for (int p = 0; p < 4; p++)
#pragma unroll
                for (int k = 0; k < 4; k++) a[p][k] = fmaf(g.b, a[p][k], acc[p * 4 + k] * (g.c / kScale));
        }
        __syncthreads();                                 // A has been read
        if (t == 0) store_symmetric(S, a, rows, i, j, coefficients, g.a);
        __syncthreads();
        if (mine) step_block(S, XT, wr, wc, i, coefficients, rows, exponent_at(column, rows.grown), x);
        if (step + 1 == steps) {
            if (mine) apply_results(q, x, i, t * 64 + j);
            return;
        }
        rows.grown = grown_by(g.growth, step + 1);
        __syncthreads();                                 // X's transpose has been read
        if (mine) store_both(XT, X, x, rows, exponent_at(column, rows.grown), i, j);
    }
}

// ---------------------------------------------------------------- host side
int32_t launched() { return hipGetLastError() == hipSuccess ? (int32_t)NNT_OK : (int32_t)NNT_EHIP; }

// The largest |c1 x + c2 x^2| between 0 and x = top.
double most_of_square(double c1, double c2, double top) {
    double most = std::fabs(c1 * top + c2 * top * top);
    if (c2 != 0.0) {
        const double x = -c1 / (2.0 * c2);
        if (x > 0.0 && x < top) most = std::max(most, std::fabs(c1 * x + c2 * x * x));
    }
    return most;
}
// Whether the iteration stays where the workspace's numbers can hold it (2^12 times 16 is fp16's largest number): singular values start in [0, 1]; with their
// bound followed from step to step, they, their squares and b s^2 + c s^4 have to stay below 8.  *reach: the largest of the bounds; *before: the largest that a step starts from.
bool in_range(const nnt_newton_schulz_cfg& c, double* reach = nullptr, double* before = nullptr) {
    if (!std::isfinite(c.a) || !std::isfinite(c.b) || !std::isfinite(c.c) || !(c.eps > 0.0) || !std::isfinite(c.eps) || c.steps < 1 || c.steps > 64) return false;
    double top = 1.0, far = 1.0, start = 1.0;
    for (int t = 0; t < c.steps; t++) {
        const double l = top * top;
        start = std::max(start, top);
        if (!(most_of_square(c.b, c.c, l) <= 8.0)) return false;
        // f(s) = a s + b s^3 + c s^5 is largest at the end or where a + 3 b s^2 + 5 c s^4 = 0
        auto f = [&](double x) { return std::fabs(std::sqrt(x) * (c.a + c.b * x + c.c * x * x)); };
        double most = f(l);
        const double p = 3.0 * c.b, q = 5.0 * c.c, d = p * p - 4.0 * q * c.a;
        if (q == 0.0) {
            if (p != 0.0 && -c.a / p > 0.0 && -c.a / p < l) most = std::max(most, f(-c.a / p));
        } else if (d >= 0.0) {
            for (double x : {(-p + std::sqrt(d)) / (2.0 * q), (-p - std::sqrt(d)) / (2.0 * q)})
                if (x > 0.0 && x < l) most = std::max(most, f(x));
        }
        if (!(most <= 8.0) || !(most * most <= 8.0)) return false;
        top = most;
        far = std::max(far, top);
    }
    if (reach) *reach = far;
    if (before) *before = start;
    return true;
}

// What a step can make a row grow by, the largest |a + b s^2 + c s^4|, as its logarithm in 1/256 (rounded up; rows that shrink are followed for 16 binary places a step).
int growth_of(const nnt_newton_schulz_cfg& c) {
    double before = 1.0;
    (void)in_range(c, nullptr, &before);
    const double l = before * before, x = c.c != 0.0 ? -c.b / (2.0 * c.c) : 0.0;
    double most = std::max(std::fabs(c.a), std::fabs(c.a + c.b * l + c.c * l * l));
    if (x > 0.0 && x < l) most = std::max(most, std::fabs(c.a + c.b * x + c.c * x * x));
    return (int)std::ceil(256.0 * std::max(std::log2(most), -16.0) + 0.01);
}

// Whether two steps can be taken at once.  The buffers hold polynomials in A = X X^T without a constant term, p(s^2) = s^2 r(s^2), as D p, whose entries reach |r| s in a row
// of length 1 and |p| in one that keeps its length; the last one, P_1 P_0 without its constant term, the same at a quarter of the scale.  r has degree 11 in s^2 at most:
// between two of 257 places it rises by less than 4 % of its largest value (|r''| <= 11^2 (11^2 - 1) / 3 (2 / l)^2 of it), s by what the next place has; the margin is 6 %.
bool pairs_in_range(const nnt_newton_schulz_cfg& c) {
    double reach = 1.0;
    if (!in_range(c, &reach)) return false;
    double most = 0.0, last = 0.0;
    for (int i = 0; i <= 256; i++) {
        const double l = reach * reach * i / 256.0, next = reach * reach * (i + 1) / 256.0, at = std::max(std::sqrt(next), next);
        const double p0 = c.a + c.b * l + c.c * l * l, r0 = c.b + c.c * l, r1 = p0 * p0 * (c.b + c.c * l * p0 * p0);
        for (double r : {r0, p0, p0 * p0, r1}) most = std::max(most, at * std::fabs(r));
        last = std::max(last, at * std::fabs(r1 * l * r0 + c.a * (r0 + r1)));
    }
    return most < 15.0 && last < 60.0;
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

template <typename S>
void launch_product(int mode, const NsGroup* g, const NsSizes& sizes, const NsOp& op, int now, unsigned tiles, int splits, hipStream_t st) {
    const dim3 grid(tiles * (unsigned)splits), block(64 * S::kWaves);
    switch (mode) {
        case kGram:
            hipLaunchKernelGGL((ns_product_kernel<kGram, S>), grid, block, 0, st, g, sizes, op, now, splits);
            if constexpr (S::BM <= 128)
                if (splits > 1) hipLaunchKernelGGL((ns_combine_kernel<S>), dim3(tiles * (S::kWaves * S::FM * S::FN / 4)), dim3(256), 0, st, g, sizes, op, splits);
            break;
        case kPoly: hipLaunchKernelGGL((ns_product_kernel<kPoly, S>), grid, block, 0, st, g, sizes, op, now, 1); break;
        case kStep: hipLaunchKernelGGL((ns_product_kernel<kStep, S>), grid, block, 0, st, g, sizes, op, now, 1); break;
        default:
            // (two terms to add, or the results' way into the tensors' tiles, do not fit the registers of the large shape)
            if constexpr (S::BM <= 128) {
                if (mode == kPair) hipLaunchKernelGGL((ns_product_kernel<kPair, S>), grid, block, 0, st, g, sizes, op, now, 1);
                else hipLaunchKernelGGL((ns_product_kernel<kLast, S>), grid, block, 0, st, g, sizes, op, now, 1);
            }
            break;
    }
}

// How a product of a group is launched.
struct Launch {
    int shape = 0, splits = 1;           // shape: 0 small, 1 middle, 2 large
    unsigned tiles = 0;
    double time = 0.0;                   // of the model below, in microseconds
};
struct Item {
    int mode;
    NsOp op;
    int now;
};

// The products of an iteration of `steps` steps.  Two steps can be taken at once: with A_1 = P_0 A_0 P_0, P = a I + b A + c A^2, the second one's polynomial comes
// from square products alone, and X <- (P_1 P_0) X once: one product of X with itself and one with X (3 m^2 n flops) less for three square ones
// (3 m^3) more.  A is recomputed from X after that, so what A_1 loses of the small singular values is not handed on.
std::vector<Item> plan(const nnt_newton_schulz_cfg& c, int growth, bool pairs) {
    const float A = (float)c.a, B = (float)c.b, C = (float)c.c;
    std::vector<Item> out;
    int now = 0;
    for (int left = c.steps; left > 0;) {
        const bool two = pairs && left >= 2;
        const int from = grown_by(growth, c.steps - left);
        auto poly = [&](int mode, int p, int q, int e, int d, int last, float mul, float add, float base) {
            out.push_back(Item{mode, NsOp{p, q, e, d, last, from, from, 0, mul, add, base}, now});
        };
        out.push_back(Item{kGram, NsOp{0, 0, 0, 0, 0, from, from, 0, 1.f, 0.f, 0.f}, now});
        if (two) {
            poly(kPoly, 0, 0, 0, 1, 0, C, B, 0.f);           // B_0 = P_0 - a I
            poly(kPoly, 1, 0, 0, 2, 0, 1.f, A, 0.f);         // P_0 A_0
            poly(kPoly, 1, 2, 2, 3, 0, 1.f, A, 0.f);         // A_1 = P_0 (P_0 A_0)
            poly(kPoly, 3, 3, 3, 2, 0, C, B, 0.f);           // B_1 = P_1 - a I
            poly(kPair, 2, 1, 0, 0, 1, 1.f, A, A * A);       // P_1 P_0 = B_1 B_0 + a B_1 + a B_0 + a^2 I
        } else {
            poly(kPoly, 0, 0, 0, 1, 1, C, B, A);
        }
        left -= two ? 2 : 1;
        out.push_back(Item{left ? kStep : kLast, NsOp{two ? 0 : 1, 0, 0, 0, 0, from, grown_by(growth, c.steps - left), -kShift - kShiftX + (two ? kPairShift : 0), 1.f, 0.f, 0.f}, now});
        now = 1 - now;
    }
    return out;
}

// The fastest launch of a product by a model of its time: a compute unit takes `lone` microseconds per panel of 16 columns for the only tile that it
// holds, `full` for each of several, and a launch a fixed time besides and the time of its results' way to memory (5 TB/s).  (Measured; a tile of 64 x 64 alone is bound by the 32 bytes per clock that a
// unit fetches, large ones by the clock that the power limit leaves.)  A product whose contraction is long and whose tiles are few is cut along the contraction.
Launch choose(const NsSizes& g, int mode) {
    static const struct { int blocks; double lone, full, fixed; } kShapes[3] = {{1, 0.107, 0.12, 2.6}, {2, 0.25, 0.339, 4.0}, {4, 0.8, 1.18, 7.0}};
    constexpr double kCombine = 4.0;
    const bool sym = mode == kGram || mode == kPoly || mode == kPair;
    Launch best;
    double best_time = 0.0;
    for (int s = 0; s < (mode == kLast || mode == kPair ? 2 : 3); s++) {
        const int u = kShapes[s].blocks;
        int64_t tiles = 0, panels = 0, longest = 0;
        double bytes = 0.0;                                                            // of the result path
        for (int k = 0; k < g.n; k++) {
            const int64_t mb = g.blocks[k] & 0xffffu, nb = g.blocks[k] >> 16, tm = (mb + u - 1) / u, tn = (nb + u - 1) / u;
            const int64_t t = sym ? tm * (tm + 1) / 2 : tm * tn, c = 4 * (mode == kGram ? nb : mb);
            tiles += t;
            panels += t * c;
            longest = std::max(longest, c);
            bytes += 4096.0 * mb * (mode == kGram ? 4 * mb : mode == kPoly ? 6 * mb : mode == kPair ? 8 * mb : mode == kStep ? 16 * nb : 16 * nb);
        }
        for (int splits = 1; splits <= 64; splits *= 2) {
            if (splits > 1 && (mode != kGram || s == 2 || tiles * splits > 512 || longest / splits < 8)) break;
            const double each = (double)panels / tiles / splits;                       // panels of a workgroup, on average
            const double per = std::ceil(tiles * splits / 256.0);
            double time = per > 1.0 ? per * each * kShapes[s].full : (double)longest / splits * kShapes[s].lone;
            time += kShapes[s].fixed + bytes / 5e6 + (splits > 1 ? kCombine + 0.1 * splits : 0.0);
            if (best.tiles == 0 || time < best_time) {
                best_time = best.time = time;
                best.shape = s;
                best.splits = splits;
                best.tiles = (unsigned)tiles;
            }
        }
    }
    return best;
}

// How a matrix is worked on.
enum { kProducts, kNarrow, kHeld };
int kind_of(int64_t m, int64_t l) { return m > 64 || l > 64 * kNarrowBlocks ? kProducts : l > 64 * kHeldBlocks ? kNarrow : kHeld; }

// Sets of up to this size take the two halves of the workspace in turn, so that two of them run side by side: a launch's beginning and end, and the units that
// it leaves idle, are the other's (sets of a step on 12 blocks of 768 wide 4.8 -> 4.0 ms, 777 x 1111 185 -> 115 us each; more than two at a time, four sets of a
// block of 1600 10.0 -> 10.7 ms).  Larger ones fill the chip (two of 4096 x 4096 7.97 ms either way) and take all of it.
constexpr int64_t kHalfBytes = (int64_t)512 << 20;

// One set of launches: as many matrices as it takes to fill the chip.
struct Set {
    NsGroup g{};
    NsSizes sizes{};
    int kind = 0;                        // kProducts, kNarrow, kHeld
    Launch launch[5];                    // by mode
    std::vector<Item> items;
    int parts = 0;
    unsigned norm_blocks = 0;
    int64_t patch = 0, bytes = 0;        // 64 x 64 blocks of all matrices; workspace
    double work = 0.0;
    std::vector<Access> acc;
    bool whole() const { return bytes > kHalfBytes; }
};

// Puts tasks from number *first on into a set.
int32_t make_set(nnt_ctx* ctx, const char* label, const nnt_newton_schulz_cfg& cfg, float mu, int nesterov, const std::vector<Task>& tasks, int kind, size_t* first, Set* out) {
    Set& w = *out;
    NsGroup& g = w.g;
    g.nesterov = nesterov;
    g.mu = mu;
    g.a = (float)cfg.a;
    g.b = (float)cfg.b;
    g.c = (float)cfg.c;
    g.eps = cfg.eps;
    g.growth = growth_of(cfg);
    const bool narrow = kind == kNarrow;
    w.kind = kind;
    int64_t bytes = (sizeof(NsGroup) + 255) / 256 * 256, shortest = INT64_MAX;
    std::vector<const nnt_tensor*> taken;                // inputs of this set
    while (*first < tasks.size() && g.n < kGroupMatrices && w.patch < 4096) {
        const Task& t = tasks[*first];
        // (a workgroup that holds its matrix does not wait for the others to have read theirs)
        if (kind == kHeld && std::any_of(taken.begin(), taken.end(), [&](const nnt_tensor* G) { return G == t.P; })) break;
        taken.push_back(t.G);
        ++*first;
        const int64_t rows = t.G->shape[0], cols = t.G->shape[1], m = std::min(rows, cols), l = std::max(rows, cols);
        const int64_t mb = (m + 63) / 64, nb = (l + 63) / 64;
        if (nb > 0xffff || mb * nb > (1 << 24)) return fail(ctx, NNT_EINVAL, std::string(label) + ": matrix too large");
        w.sizes.blocks[g.n] = (uint32_t)mb | ((uint32_t)nb << 16);
        NsMatrix& q = g.mat[g.n++];
        q.rows = (int32_t)rows;
        q.cols = (int32_t)cols;
        q.base0 = (int32_t)t.G->base[0];
        q.base1 = (int32_t)t.G->base[1];
        q.grid0 = (int32_t)t.G->grid[0];
        q.grid1 = (int32_t)t.G->grid[1];
        q.flip = rows > cols;
        q.mp = (int32_t)(mb * 64);
        q.np = (int32_t)(nb * 64);
        w.patch += mb * nb;
        shortest = std::min(shortest, m);
        if (kind != kProducts) w.parts = std::max(w.parts, narrow ? narrow_parts((int)nb) : (int)nb);
        // squares are added up by as many workgroups as fill the chip; the set-up reads one sum per row and part
        const int64_t rounds = (q.np + kNormSpan - 1) / kNormSpan;
        q.splits = (int32_t)std::min({rounds, std::max<int64_t>(1, 1024 / mb), std::max<int64_t>(32, std::min<int64_t>(rounds / 32, 128))});
        w.norm_blocks = std::max(w.norm_blocks, (unsigned)(mb * q.splits));
        // X once, its transpose twice, X in fp32, and four square buffers; narrow matrices: the transpose and fp32, and two times A in parts
        const int64_t x = (int64_t)q.mp * q.np * 4, a = (int64_t)q.mp * q.mp * 4;
        q.X = bytes;
        q.XT = narrow ? bytes : q.X + x;
        q.E = narrow ? q.XT + x : q.XT + 2 * x;
        q.A = q.E + x;
        q.squares = q.A + (narrow ? (int64_t)narrow_parts((int)nb) * 64 * 64 * 4 * 2 : 4 * a);
        q.part = q.squares + (int64_t)q.splits * q.mp * 8;
        q.exponents = q.part + mb * q.splits * 8;
        q.columns = q.exponents + q.mp * 4;
        q.coefficients = q.columns + (int64_t)q.np * 4;
        q.largest = q.coefficients + q.mp * 4;
        bytes = (q.largest + mb * (q.flip ? 4 : 1) * q.np * 2 + 255) / 256 * 256;
        q.G = MatView{t.G->d_tiles, t.G->dtype};
        q.P = MatView{t.P->d_tiles, t.P->dtype};
        if (t.M) q.M = MatView{t.M->d_tiles, NNT_F32};
        if (t.LP) q.LP = MatView{t.LP->d_tiles, NNT_BF16};
        q.decay = t.decay;
        q.step = t.step;
        w.work += cfg.steps * (3.0 * m * m * l + (double)m * m * m);
        w.acc.push_back(t.G->all(kRead));
        w.acc.push_back(t.P->all(t.step < 0.f ? kWrite : kReadWrite));
        if (t.M) w.acc.push_back(t.M->all(kReadWrite));
        if (t.LP) w.acc.push_back(t.LP->all(kWrite));
    }
    w.sizes.n = g.n;
    if (kind == kHeld) return NNT_OK;                    // (needs no workspace)
    g.partial = bytes;
    if (kind == kProducts) {
        for (int mode : {(int)kGram, (int)kPoly, (int)kPair, (int)kStep, (int)kLast}) w.launch[mode] = choose(w.sizes, mode);
        const Launch& gram = w.launch[kGram];
        if (gram.splits > 1) bytes += (int64_t)gram.tiles * gram.splits * (gram.shape == 0 ? Small::BM * Small::BM : Middle::BM * Middle::BM) * 4;
        // (The model is a tenth and more off either way: two steps at once have to promise that much.  Below 256 rows they gain less, 128 x 6272 120 us instead of 128, and
        // their errors are larger than those of fp32 products, 128 x 1000 2.9e-6 after five steps instead of 1.7e-6.)
        w.items = plan(cfg, g.growth, shortest >= 256 && 1.15 * 3.0 * w.launch[kPoly].time < gram.time + w.launch[kStep].time && pairs_in_range(cfg));
    }
    w.bytes = bytes;
    return NNT_OK;
}

int32_t submit_set(nnt_ctx* ctx, const char* label, int steps, Set& w) {
    NsGroup g = w.g;
    if (w.kind != kHeld) {
        const bool alone = w.whole() || ctx->matrix_halves == 1;
        const int half = alone ? 0 : ctx->matrix_turn++ & 1;
        for (int k = 0; k < 2; k++)
            if (k == half || alone) w.acc.push_back(Access{&ctx->matrix_dep[k], 1, kReadWrite});
        g.space = ctx->matrix_scratch + half * ctx->matrix_half;
    }
    const NsGroup* there = reinterpret_cast<const NsGroup*>(g.space);
    OpTag tag(ctx, label, w.work, false);
    if (w.kind == kHeld)
        return submit(ctx, w.acc, [&](hipStream_t st) {
            hipLaunchKernelGGL(ns_held_kernel, dim3((unsigned)g.n), dim3(256u * w.parts), 0, st, g, steps);
            return launched();
        });
    const int grams = (int)std::count_if(w.items.begin(), w.items.end(), [](const Item& t) { return t.mode == kGram; });      // each with a launch that adds up its parts, if it is cut
    return submit(ctx, w.acc, [&](hipStream_t st) {
        hipLaunchKernelGGL(ns_norm_kernel, dim3(w.norm_blocks, (unsigned)g.n), dim3(64 * kNormWaves), 0, st, g);
        if (w.kind == kNarrow) {
            const dim3 grid((unsigned)w.parts, (unsigned)g.n), block(256);
            hipLaunchKernelGGL((ns_narrow_kernel<kFirst>), grid, block, 0, st, there, w.sizes, 0);
            for (int s = 0; s + 1 < steps; s++) hipLaunchKernelGGL((ns_narrow_kernel<kMiddle>), grid, block, 0, st, there, w.sizes, s);
            hipLaunchKernelGGL((ns_narrow_kernel<kFinal>), grid, block, 0, st, there, w.sizes, steps - 1);
            return launched();
        }
        hipLaunchKernelGGL(ns_split_kernel, dim3((unsigned)w.patch), dim3(256), 0, st, there, w.sizes);
        for (const Item& t : w.items) {
            const Launch& l = w.launch[t.mode];
            if (l.shape == 2) launch_product<Large>(t.mode, there, w.sizes, t.op, t.now, l.tiles, l.splits, st);
            else if (l.shape == 1) launch_product<Middle>(t.mode, there, w.sizes, t.op, t.now, l.tiles, l.splits, st);
            else launch_product<Small>(t.mode, there, w.sizes, t.op, t.now, l.tiles, l.splits, st);
        }
        return launched();
    }, w.kind == kNarrow ? 2 + steps : 2 + (int)w.items.size() + (w.launch[kGram].splits > 1 ? grams : 0));
}

// Orthogonalises the matrices of `tasks` and applies the results.  mu < 0: no momentum.  Nothing is launched before all sets are known to fit.
int32_t newton_schulz(nnt_ctx* ctx, const char* label, const nnt_newton_schulz_cfg& cfg, float mu, int nesterov, const std::vector<Task>& tasks) {
    std::vector<Task> kind[3];
    for (const Task& t : tasks) {
        const int64_t m = std::min(t.G->shape[0], t.G->shape[1]), l = std::max(t.G->shape[0], t.G->shape[1]);
        kind[kind_of(m, l)].push_back(t);
    }
    std::vector<Set> sets;
    int64_t half = 0, whole = 0;
    for (int k = 0; k < 3; k++)
        for (size_t first = 0; first < kind[k].size();) {
            sets.emplace_back();
            const int32_t rc = make_set(ctx, label, cfg, mu, nesterov, kind[k], k, &first, &sets.back());
            if (rc != NNT_OK) return rc;
            int64_t& most = sets.back().whole() ? whole : half;
            most = std::max(most, sets.back().bytes);
        }
    int32_t rc = ensure_matrix_scratch(ctx, half, whole);
    for (size_t k = 0; rc == NNT_OK && k < sets.size(); k++) rc = submit_set(ctx, label, cfg.steps, sets[k]);
    return rc;
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
