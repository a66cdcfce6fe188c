// Tiles of attention on the matrix cores, for the two storage types: how a block of streamed rows sits in LDS, how a lane keeps its own
// row, and the two kinds of products.
#pragma once
#include "device_util.hpp"

namespace nnt {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_huge_valf();

// ---------------------------------------------------------------- element-type traits
// What differs between the two storage types: how a block of 64 streamed rows sits in LDS, how a
// lane keeps its own row, and the two kinds of products.
//
//   rows_times_own   acc[r][c] += sum_i block[32 sub + r][i] * own[c][i]      (32 x 32, contraction over
//                    the first axis; A operand read row-wise from LDS, B operand = the lane's own row)
//   cols_times_acc   out[rb][i][c] += sum_r block[32 sub + r][32 rb + i] * p[r][c]   (contraction over the
//                    block's rows; p comes from accumulator registers: register r of lane half hh holds
//                    row acc_row(r, hh), and the A operand is read from LDS in that same order)

__device__ __forceinline__ int acc_row(int r, int hh) { return 8 * (r / 4) + 4 * hh + (r % 4); }
// the part of acc_row that is known at compile time: a bound `row < lim` on acc_row(r, hh) is the
// per-lane bound `acc_row0(r) < lim - 4 hh`, one comparison with a constant per register
__device__ __forceinline__ constexpr int acc_row0(int r) { return 8 * (r / 4) + (r % 4); }

__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; i++) z[i] = 0.f;
    return z;
}

template <int H_> struct F32Traits {
    static constexpr int H = H_;
    using T = float;
    using Vec = float4;                               // 16 bytes of a row
    static constexpr int kPer = 4;                    // elements per Vec
    static constexpr int kVec = H / 16;               // Vec per thread per block (64 rows x H / 4 over 256 threads)
    // v_mfma_f32_32x32x2_f32: a lane supplies one element per instruction, half hh the k index hh.
    // Row pitch H + 4: rows stay 16-byte aligned, so a lane fetches four k-steps of its row with one
    // 128-bit read, and 16 lanes (rows r .. r+15, 4 r + c modulo 64) cover all 64 banks.
    static constexpr int LD = H + 4;
    // pitch for a block that is only read column-wise: puts the two lane halves 32 banks apart
    static constexpr int LD_COLS = H + 8;
    static constexpr int kDkvBlocks = 2;
    struct Own { float v[H / 2]; };                   // elements s + (H/2) hh of the lane's row
    struct Packed { f32x16 v; };

    static __device__ __forceinline__ Vec zero_vec() { return make_float4(0.f, 0.f, 0.f, 0.f); }
    template <int LDX>
    static __device__ __forceinline__ void put(T* lds, int row, int c, const Vec& x) {
        T* d = lds + row * LDX + c * kPer;
        if constexpr (LDX % 4 == 0) {
            *reinterpret_cast<Vec*>(d) = x;
        } else {
            d[0] = x.x; d[1] = x.y; d[2] = x.z; d[3] = x.w;
        }
    }
    static __device__ __forceinline__ void load_own(const T* slab, int pitch, int row, int hh, bool valid, Own& o) {
        const float4* p = reinterpret_cast<const float4*>(slab + (int64_t)row * pitch + (H / 2) * hh);
#pragma unroll
        for (int s4 = 0; s4 < H / 8; s4++) {
            const float4 x = valid ? p[s4] : make_float4(0.f, 0.f, 0.f, 0.f);
            o.v[4 * s4 + 0] = x.x; o.v[4 * s4 + 1] = x.y; o.v[4 * s4 + 2] = x.z; o.v[4 * s4 + 3] = x.w;
        }
    }
    // sum over the first axis of a[i] * b[i] restricted to this lane's half of the row
    static __device__ __forceinline__ float dot_own(const Own& a, const Own& b) {
        float d = 0.f;
#pragma unroll
        for (int k = 0; k < H / 2; k++) d += a.v[k] * b.v[k];
        return d;
    }
    template <int LDX>
    static __device__ __forceinline__ f32x16 rows_times_own(const T* lds, int sub, int ln, int hh, const Own& o) {
        static_assert(LDX % 4 == 0, "128-bit fragment reads need 16-byte aligned rows");
        const float4* p = reinterpret_cast<const float4*>(lds + (32 * sub + ln) * LDX + (H / 2) * hh);
        f32x16 acc = zero16();
#pragma unroll
        for (int k4 = 0; k4 < H / 8; k4++) {
            const float4 a = p[k4];
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, o.v[4 * k4], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, o.v[4 * k4 + 1], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, o.v[4 * k4 + 2], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, o.v[4 * k4 + 3], acc, 0, 0, 0);
        }
        return acc;
    }
    static __device__ __forceinline__ void pack(const f32x16& x, Packed& pk) { pk.v = x; }
    static __device__ __forceinline__ void set(Packed& pk, int r, float x) { pk.v[r] = x; }
    template <int LDX>
    static __device__ __forceinline__ void cols_times_acc(f32x16 (&out)[H / 32], const T* lds, int sub, int lane, const Packed& pk) {
        const int ln = lane & 31, hh = lane >> 5;
#pragma unroll
        for (int r = 0; r < 16; r++)
#pragma unroll
            for (int rb = 0; rb < H / 32; rb++)
                out[rb] = __builtin_amdgcn_mfma_f32_32x32x2f32(lds[(32 * sub + acc_row(r, hh)) * LDX + 32 * rb + ln], pk.v[r], out[rb], 0, 0, 0);
    }
    static __device__ __forceinline__ void store4(T* p, float a, float b, float c, float d) {
        *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
    }
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

template <int H_> struct Bf16Traits {
    static constexpr int H = H_;
    using T = bf16_t;
    using Vec = uint4;
    static constexpr int kPer = 8;
    static constexpr int kVec = H / 32;               // 64 rows x H / 8 vectors over 256 threads
    // v_mfma_f32_32x32x16_bf16: a lane supplies 8 consecutive k per instruction, half hh the k indices 8 hh ..
    // Row-wise fragments are 16-byte reads of rows 144 (272) bytes apart: 16 lanes cover all 64 banks.
    static constexpr int LD = H + 8;
    // Column-wise fragments are transposing reads (ds_read_b64_tr_b16) of 4 rows x 64 bytes per half
    // wave: rows 64 bytes apart modulo 256 keep the four rows on different banks.
    static constexpr int LD_COLS = H + 32;
    static constexpr int kDkvBlocks = H == 64 ? 2 : 1;
    struct Own { bf16x8 v[H / 16]; };                 // elements 16 s + 8 hh .. + 7 of the lane's row
    struct Packed { bf16x8 v[2]; };                   // registers 8 m .. 8 m + 7 of an accumulator, rounded

    static __device__ __forceinline__ Vec zero_vec() { return make_uint4(0u, 0u, 0u, 0u); }
    template <int LDX>
    static __device__ __forceinline__ void put(T* lds, int row, int c, const Vec& x) {
        *reinterpret_cast<Vec*>(lds + row * LDX + c * kPer) = x;
    }
    static __device__ __forceinline__ void load_own(const T* slab, int pitch, int row, int hh, bool valid, Own& o) {
        const uint4* p = reinterpret_cast<const uint4*>(slab + (int64_t)row * pitch + 8 * hh);
#pragma unroll
        for (int s = 0; s < H / 16; s++) {
            const uint4 x = valid ? p[2 * s] : make_uint4(0u, 0u, 0u, 0u);
            o.v[s] = __builtin_bit_cast(bf16x8, x);
        }
    }
    static __device__ __forceinline__ float dot_own(const Own& a, const Own& b) {
        float d = 0.f;
#pragma unroll
        for (int s = 0; s < H / 16; s++)
#pragma unroll
            for (int e = 0; e < 8; e++) d += (float)a.v[s][e] * (float)b.v[s][e];
        return d;
    }
    template <int LDX>
    static __device__ __forceinline__ f32x16 rows_times_own(const T* lds, int sub, int ln, int hh, const Own& o, const f32x16& more = zero16()) {
        const T* p = lds + (32 * sub + ln) * LDX + 8 * hh;
        f32x16 acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(p), o.v[0], more, 0, 0, 0);
#pragma unroll
        for (int s = 1; s < H / 16; s++)
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(p + 16 * s), o.v[s], acc, 0, 0, 0);
        return acc;
    }
    static __device__ __forceinline__ void pack(const f32x16& x, Packed& pk) {
#pragma unroll
        for (int m = 0; m < 2; m++)
#pragma unroll
            for (int e = 0; e < 8; e++) pk.v[m][e] = (__bf16)x[8 * m + e];
    }
    static __device__ __forceinline__ void set(Packed& pk, int r, float x) { pk.v[r / 8][r % 8] = (__bf16)x; }
    // what pack() has rounded away
    static __device__ __forceinline__ void pack_rest(const f32x16& x, const Packed& pk, Packed& rest) {
#pragma unroll
        for (int m = 0; m < 2; m++)
#pragma unroll
            for (int e = 0; e < 8; e++) rest.v[m][e] = (__bf16)(x[8 * m + e] - (float)pk.v[m][e]);
    }
    // (`rest`: a second part of p, times the same columns)
    template <int LDX>
    static __device__ __forceinline__ void cols_times_acc(f32x16 (&out)[H / 32], const T* lds, int sub, int lane, const Packed& pk, const Packed* rest = nullptr) {
        // Accumulator registers 8 m + e of half hh are the rows 16 m + 8 (e / 4) + 4 hh + e % 4: two runs of
        // four consecutive rows, one transposing read each.  In such a read the 16 lanes of a group fetch
        // 8 bytes each -- lane j the columns 4 (j % 4) .. + 3 of row j / 4 of a 4 x 16 patch -- and lane j
        // receives the four rows of column j.
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const int j = lane & 15, grp = lane >> 4, hh = grp >> 1;
        const T* base = lds + (32 * sub + 4 * hh + (j >> 2)) * LDX + 16 * (grp & 1) + 4 * (j & 3);
#pragma unroll
        for (int m = 0; m < 2; m++)
#pragma unroll
            for (int rb = 0; rb < H / 32; rb++) {
                const T* p = base + (16 * m) * LDX + 32 * rb;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * LDX));
                const s16x8 x = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                out[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), pk.v[m], out[rb], 0, 0, 0);
                if (rest) out[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), rest->v[m], out[rb], 0, 0, 0);
            }
    }
    static __device__ __forceinline__ void store4(T* p, float a, float b, float c, float d) {
        uint2 x;
        x.x = (uint32_t)f2bf(a) | ((uint32_t)f2bf(b) << 16);
        x.y = (uint32_t)f2bf(c) | ((uint32_t)f2bf(d) << 16);
        *reinterpret_cast<uint2*>(p) = x;
    }
};

}  // namespace
}  // namespace nnt
