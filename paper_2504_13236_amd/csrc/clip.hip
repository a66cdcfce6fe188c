// The norm of many gradients taken together, and the gradients clipped by it:
//   norm = sqrt(sum g^2),   O = min(1, max_norm / (norm + eps)) G.
//
// Bound by memory: the factor is known only when everything has been read, so the gradients are read twice and written once.
// The tiles of all tensors are cut into pieces of kPiece elements; pieces are numbered through, and the workgroups of a launch
// take them in turn.  A workgroup's sum goes to a place of its own, and one workgroup adds those up in their order: sums never
// depend on which workgroup came first.  Squares are taken and added in 64 bits: gradients of 1e-23 have squares below fp32's range, and
// 64-bit multiply-adds run at half the fp32 rate, far from what bounds this.
// 124.5 M fp32 gradients in 148 tensors: 286 us (1.49 GB at 5.2 TB/s: the second read begins with what the first ended with).  The twelve of a block of 64: 11 us, two launches.
// (Calls one after the other; the launches of one that is waited for add up to 326 and 10 us.)
#include "clip_pieces.hpp"
#include "device_util.hpp"
#include "internal.hpp"

#include <algorithm>
#include <cmath>

namespace nnt {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxGroups = 2048;       // workgroups of a launch: eight to a compute unit
constexpr int kFew = 256;              // partial sums that every workgroup of the second pass adds up by itself (the smallest block 13.3 -> 11 us)
static_assert(sizeof(List) + 64 <= 4096, "arguments of a launch");

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

template <typename T>
__device__ __forceinline__ double squares_of(const T* p, int count) {
    constexpr int V = VecOf<T>::V;
    double s = 0.0;
    int head = 0;
    if (((uintptr_t)p & 15) == 0) {
        head = count / V * V;
        for (int i = (int)threadIdx.x * V; i < head; i += kThreads * V) {
            float f[V];
            ldv<V>(p + i, f);
#pragma unroll
            for (int j = 0; j < V; j++) s = fma((double)f[j], (double)f[j], s);
        }
    }
    for (int i = head + (int)threadIdx.x; i < count; i += kThreads) {
        float f[1];
        ldv<1>(p + i, f);
        s = fma((double)f[0], (double)f[0], s);
    }
    return s;
}

__global__ void __launch_bounds__(kThreads) squares_kernel(List a, double* partial) {
    __shared__ double part[kThreads / 64];
    double s = 0.0;
    for (int w = blockIdx.x; w < a.pieces; w += gridDim.x) {
        const Piece p = piece_of(a, w);
        void* tile = p.t->in[p.tile];
        if (p.count == 0 || !tile) continue;
        s += p.t->bf16 ? squares_of<bf16_t>(global_as<const bf16_t>(tile) + p.first, p.count) : squares_of<float>(global_as<const float>(tile) + p.first, p.count);
    }
    s = wave_sum64(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) partial[blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

// Norm and factor of the partial sums, by all threads of a workgroup in a fixed order.
template <int NT>
__device__ __forceinline__ double factor_of(const double* partial, int n, double max_norm, double eps, double* norm) {
    __shared__ double part[NT / 64];
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += NT) s += partial[i];
    s = wave_sum64(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < NT / 64; w++) s += part[w];
    *norm = sqrt(s);
    const double f = max_norm / (*norm + eps);
    return *norm < __builtin_huge_val() && f < 1.0 ? f : 1.0;          // (infinite or no number: as it is)
}

// one workgroup
__global__ void __launch_bounds__(1024) norm_kernel(const double* partial, int n, double max_norm, double eps, double* factor, float* norm) {
    double r;
    const double f = factor_of<1024>(partial, n, max_norm, eps, &r);
    if (threadIdx.x == 0) {
        *factor = f;
        *norm = (float)r;
    }
}

// a 64-bit product rounded to T, once (a bf16 number is one of fp32 too)
template <typename T>
__device__ __forceinline__ float rounded(double v) {
    if constexpr (sizeof(T) == 2) return (float)(__bf16)v;
    else return (float)v;
}
template <typename T>
__device__ __forceinline__ void scale(const T* p, T* o, int count, double f) {
    constexpr int V = VecOf<T>::V;
    int head = 0;
    if ((((uintptr_t)p | (uintptr_t)o) & 15) == 0) {
        head = count / V * V;
        for (int i = (int)threadIdx.x * V; i < head; i += kThreads * V) {
            float x[V];
            ldv<V>(p + i, x);
#pragma unroll
            for (int j = 0; j < V; j++) x[j] = rounded<T>(f * (double)x[j]);
            stv<V>(o + i, x);
        }
    }
    for (int i = head + (int)threadIdx.x; i < count; i += kThreads) {
        float x[1];
        ldv<1>(p + i, x);
        x[0] = rounded<T>(f * (double)x[0]);
        stv<1>(o + i, x);
    }
}

// What a workgroup is told of the factor: the number itself, or (few: n_partial > 0) the sums it comes from, which saves a launch.
struct Factor {
    const double* at;
    const double* partial;
    int n_partial;
    double max_norm, eps;
    float* norm;
};
// (in place a factor of one leaves nothing to do)
__global__ void __launch_bounds__(kThreads) scale_kernel(List a, Factor by) {
    double f;
    if (by.n_partial) {
        double r;
        f = factor_of<kThreads>(by.partial, by.n_partial, by.max_norm, by.eps, &r);
        if (blockIdx.x == 0 && threadIdx.x == 0) *by.norm = (float)r;
    } else {
        f = *by.at;
    }
    for (int w = a.pieces - 1 - (int)blockIdx.x; w >= 0; w -= gridDim.x) {
        const Piece p = piece_of(a, w);
        void *in = p.t->in[p.tile], *out = p.t->out[p.tile];
        if (p.count == 0 || !in || (f == 1.0 && in == out)) continue;
        if (p.t->bf16) scale<bf16_t>(global_as<const bf16_t>(in) + p.first, global_as<bf16_t>(out) + p.first, p.count, f);
        else scale<float>(global_as<const float>(in) + p.first, global_as<float>(out) + p.first, p.count, f);
    }
}

int32_t launched() { return hipGetLastError() == hipSuccess ? (int32_t)NNT_OK : (int32_t)NNT_EHIP; }

#define TRY(x)                           \
    do {                                 \
        int32_t rc__ = (x);              \
        if (rc__ != NNT_OK) return rc__; \
    } while (0)

int64_t pieces_per_tile(const nnt_tensor* t) {
    int64_t n = 1;
    for (int d = 0; d < t->ndim; d++) n *= t->base[d];
    return (n + kPiece - 1) / kPiece;
}

// Lists of at most kListed tensors and 2^30 pieces.
std::vector<List> lists_of(int32_t n, nnt_tensor* const* G, nnt_tensor* const* O) {
    std::vector<List> out;
    for (int32_t k = 0; k < n; k++) {
        const int64_t per = pieces_per_tile(G[k]), pieces = per * G[k]->ntiles;
        if (out.empty() || out.back().n == kListed || out.back().pieces + pieces > (1 << 30)) {
            out.emplace_back();
            out.back().n = out.back().pieces = 0;
        }
        List& l = out.back();
        Listed& t = l.t[l.n++];
        const TiledView v = G[k]->view();
        t.in = v.tiles;
        t.out = O ? O[k]->d_tiles : nullptr;
        for (int d = 0; d < kMaxDim; d++) {
            t.shape[d] = v.shape[d];
            t.base[d] = v.base[d];
            t.grid[d] = v.grid[d];
        }
        t.first = l.pieces;
        t.per_tile = (int32_t)per;
        t.bf16 = G[k]->dtype == NNT_BF16;
        l.pieces += (int32_t)pieces;
    }
    return out;
}

unsigned groups_of(const List& l) { return (unsigned)std::min(l.pieces, kMaxGroups); }

}  // namespace

int32_t clip_check(nnt_ctx* ctx, const nnt_clip_cfg* cfg, int32_t n, nnt_tensor* const* G, nnt_tensor* const* O, const float* norm) {
    const std::string who = "nnt_clip_grad_norm";
    if (!cfg || n < 1 || !G || !norm) return fail(ctx, NNT_EINVAL, who + ": null argument or empty list");
    if (!(cfg->max_norm > 0.0) || !(cfg->eps >= 0.0 && cfg->eps < 1e30)) return fail(ctx, NNT_EINVAL, who + ": max_norm must be above 0, eps 0 or more");
    std::vector<const nnt_tensor*> in(G, G + n), out;
    for (int32_t k = 0; k < n; k++) {
        if (!G[k] || G[k]->ctx != ctx) return fail(ctx, NNT_EINVAL, who + ": gradient " + std::to_string(k) + " is missing or of another context");
        if (pieces_per_tile(G[k]) * G[k]->ntiles > (1 << 30)) return fail(ctx, NNT_EINVAL, who + ": gradient " + std::to_string(k) + " is too large");
        for (int d = 0; d < G[k]->ndim; d++)
            if (G[k]->shape[d] > INT32_MAX) return fail(ctx, NNT_EINVAL, who + ": gradient " + std::to_string(k) + " is too large");
        if (!O) continue;
        if (!O[k] || O[k]->ctx != ctx || O[k]->dtype != G[k]->dtype || !same_tiling(O[k], G[k]) || !null_alike(O[k], G[k]))
            return fail(ctx, NNT_EINVAL, who + ": result " + std::to_string(k) + " must have its gradient's type, shape, tiling and tiles");
        if (O[k] != G[k]) out.push_back(O[k]);
    }
    in.insert(in.end(), out.begin(), out.end());
    std::sort(in.begin(), in.end());
    if (std::adjacent_find(in.begin(), in.end()) != in.end()) return fail(ctx, NNT_EINVAL, who + ": a tensor is given twice");
    const int64_t launches = (int64_t)lists_of(n, G, O).size();
    return ensure_stream_scratch(ctx, 2 * (launches * kMaxGroups + 1));
}

}  // namespace nnt

using namespace nnt;

int32_t nnt_clip_grad_norm(nnt_ctx* ctx, const nnt_clip_cfg* cfg, int32_t n, nnt_tensor* const* G, nnt_tensor* const* O, float* norm) {
    return entry(ctx, [&]() -> int32_t {
        TRY(clip_check(ctx, cfg, n, G, O, norm));
        const double max_norm = cfg->max_norm, eps = cfg->eps;
        bool writes = O != nullptr;
        if (writes && max_norm == __builtin_huge_val()) {
            writes = false;
            for (int32_t k = 0; k < n; k++) writes = writes || O[k] != G[k];
        }
        const std::vector<List> lists = lists_of(n, G, O);
        std::vector<Access> acc;
        double bytes = 0.0;
        for (int32_t k = 0; k < n; k++) {
            if (O && O[k] == G[k]) acc.push_back(G[k]->all(kReadWrite));
            else acc.push_back(G[k]->all(kRead));
            if (O && O[k] != G[k]) acc.push_back(O[k]->all(kWrite));
            double e = (double)G[k]->elem_size();
            for (int d = 0; d < G[k]->ndim; d++) e *= (double)G[k]->shape[d];
            bytes += e;
        }
        OpTag tag(ctx, "clip_grad_norm", (writes ? 3.0 : 1.0) * bytes, true);
        return submit(ctx, acc, [&](hipStream_t st) -> int32_t {
            double* factor = reinterpret_cast<double*>(stream_scratch_of(ctx));
            double* partial = factor + 1;
            int at = 0;
            for (const List& l : lists) {
                hipLaunchKernelGGL(squares_kernel, dim3(groups_of(l)), dim3(kThreads), 0, st, l, partial + at);
                TRY(launched());
                at += (int)groups_of(l);
            }
            const bool few = writes && lists.size() == 1 && at <= kFew;
            if (!few) {
                hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(1024), 0, st, partial, at, max_norm, eps, factor, norm);
                TRY(launched());
            }
            // the last read first: some of it is still in the caches
            const Factor by{factor, partial, few ? at : 0, max_norm, eps, norm};
            for (size_t i = lists.size(); writes && i-- > 0;) {
                hipLaunchKernelGGL(scale_kernel, dim3(groups_of(lists[i])), dim3(kThreads), 0, st, lists[i], by);
                TRY(launched());
            }
            return NNT_OK;
        }, (int)lists.size() * (writes ? 2 : 1) + (writes && lists.size() == 1 && (int)groups_of(lists[0]) <= kFew ? 0 : 1));
    });
}
