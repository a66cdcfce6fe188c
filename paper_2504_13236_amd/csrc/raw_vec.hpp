// Vectors of logits as they lie in memory, for the kernels that keep whole columns in registers.
#pragma once
#include "device_util.hpp"

namespace nnt {
namespace {

// Eight bf16 or four fp32 logits as they are in memory, at any address of an element; a tile's last vector may be short
// (`cnt` elements, the rest is not touched).
template <typename T> struct RawVec;
template <> struct RawVec<float> {
    static constexpr int V = 4;
    typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
    vec x;
    __device__ __forceinline__ void load(const float* p, int cnt) {
        if (cnt >= V) {
            x = *reinterpret_cast<const vec*>(p);
        } else {
#pragma unroll
            for (int j = 0; j < V; j++) x[j] = j < cnt ? p[j] : 0.f;
        }
    }
    // the same with -inf in the place of what is not there
    __device__ __forceinline__ void load_or_none(const float* p, int cnt) {
        if (cnt >= V) {
            x = *reinterpret_cast<const vec*>(p);
        } else {
#pragma unroll
            for (int j = 0; j < V; j++) x[j] = j < cnt ? p[j] : -__builtin_huge_valf();
        }
    }
    __device__ __forceinline__ void none() {
#pragma unroll
        for (int j = 0; j < V; j++) x[j] = -__builtin_huge_valf();
    }
    static constexpr bool kKeeps = true;          // holds fp32 values: the shifted exponentials can take the logits' place
    __device__ __forceinline__ float at(int j) const { return x[j]; }
    __device__ __forceinline__ void set(int j, float f) { x[j] = f; }
    // away: past the caches
    static __device__ __forceinline__ void store(float* p, const float (&f)[V], int cnt, bool away = false) {
        if (cnt >= V) {
            const vec y{f[0], f[1], f[2], f[3]};
            if (away) {
                asm volatile("");                        // (else the two stores become one, of the other kind)
                __builtin_nontemporal_store(y, reinterpret_cast<vec*>(p));
                asm volatile("");
            } else {
                *reinterpret_cast<vec*>(p) = y;
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; j++)
                if (j < cnt) p[j] = f[j];
        }
    }
};
template <> struct RawVec<bf16_t> {
    static constexpr int V = 8;
    typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
    vec x;
    __device__ __forceinline__ void load(const bf16_t* p, int cnt) {
        if (cnt >= V) {
            x = *reinterpret_cast<const vec*>(p);
        } else {
            x = vec{0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < V; j++)
                if (j < cnt) x[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
        }
    }
    __device__ __forceinline__ void load_or_none(const bf16_t* p, int cnt) {
        if (cnt >= V) {
            x = *reinterpret_cast<const vec*>(p);
        } else {
            none();
#pragma unroll
            for (int j = 0; j < V; j++)
                if (j < cnt) x[j >> 1] = (j & 1) ? (x[j >> 1] & 0xffffu) | ((uint32_t)p[j] << 16) : (x[j >> 1] & 0xffff0000u) | (uint32_t)p[j];
        }
    }
    __device__ __forceinline__ void none() { x = vec{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }
    static constexpr bool kKeeps = false;
    __device__ __forceinline__ void set(int, float) {}
    __device__ __forceinline__ float at(int j) const { return __uint_as_float((j & 1) ? (x[j >> 1] & 0xffff0000u) : (x[j >> 1] << 16)); }
    static __device__ __forceinline__ void store(bf16_t* p, const float (&f)[V], int cnt, bool away = false) {
        if (cnt >= V) {
            vec y;
#pragma unroll
            for (int j = 0; j < 4; j++) y[j] = (uint32_t)f2bf(f[2 * j]) | ((uint32_t)f2bf(f[2 * j + 1]) << 16);
            if (away) {
                asm volatile("");                        // (else the two stores become one, of the other kind)
                __builtin_nontemporal_store(y, reinterpret_cast<vec*>(p));
                asm volatile("");
            } else {
                *reinterpret_cast<vec*>(p) = y;
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; j++)
                if (j < cnt) p[j] = f2bf(f[j]);
        }
    }
};

}  // namespace
}  // namespace nnt
