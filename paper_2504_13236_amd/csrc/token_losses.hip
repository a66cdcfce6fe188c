// Log-probabilities of given tokens, and the two losses of post-training that are functions of them, on logits
// x[v, s, b] that are split into vocabulary tiles (as the cross-entropy loss of section 3 takes them):
//
//   logp[s, b]  = x[c] - max_j x[j] - log sum_j exp(x[j] - max),   c = label(s, b)
//   policy      L = sum w (-min(r A, clip(r) A) + kl (e^k - k - 1)),   r = exp(logp - old),  k = ref - logp
//   preference  L = sum over pairs of -(1 - e) log sig(z) - e log sig(-z),   z = R(chosen) - R(rejected),
//               R(b) = beta sum_s (logp - ref)
//
// Either way a position's logits enter through its logp alone, so with g = dL/dlogp
//   dL/dx[j] = g (onehot[j] - softmax[j]),
// and a position without a label (a prompt, padding) has the gradient 0; its logits are not even read.
// Everything here is bound by memory: one read of the logits for logp, a read and a write for the policy loss, and
// two reads and a write for the preference loss, whose coefficients need the whole pair first.  bf16 logits, 50304 to a column, 5/8 of the positions with a label:
//   logp        8192 columns    95 to 109 us for  515 MB (4.7 to 5.4 TB/s)
//   policy      8192           241 to 264 us for 1275 MB (4.8 to 5.3 TB/s; one sequence of eight has no label at all)
//   preference  4096           142 to 175 us for  927 MB (5.3 TB/s and more: part of the second read is found in the caches)
// where a copy reaches 5.1.  A single fp32 column of 50304 takes 10 us, 6 among others: the launch, four loads in a row and two exchanges between wavefronts.
#include "colwise.hpp"
#include "device_util.hpp"
#include "internal.hpp"
#include "raw_vec.hpp"

namespace nnt {
namespace {

constexpr int kTableTiles = 64;               // vocabulary tiles whose addresses a workgroup keeps in LDS
constexpr int64_t kMaxPositions = 1 << 22;    // a workgroup of 1024 threads each: 2^32 threads are more than a launch takes
constexpr int64_t kMaxVectors = 1 << 20;      // of a column: up to there `place` finds a vector's tile exactly

// Gradients of more than this leave past the caches: they would drive out logits that are still to be read a second time, and nobody finds so much of them there
// later (preference loss of 1998 fp32 columns of 32003, 256 MB: 114 -> 98 us; policy loss of 8192 of 50304 in bf16 255 -> 241).  Smaller ones are
// read from the caches by the head's products (a model's step with 103 MB of logits 886 us, 893 with this).  There, where the products read the gradient next, larger ones gain
// little or nothing: bf16 141 MB 1119 us, 1126 without this, 206 MB 1257 and 1268, 241 MB 1440 and 1446; fp32 141 to 483 MB the same either way.
constexpr int64_t kCached = (int64_t)128 << 20;

// exp(t), t <= 0, for logits of type T.  Both factors of the exponent's product with 1/ln 2 are kept, since the rounded constant alone makes
// every log-probability 6e-8 too small, and hundreds of them add up in a reward.  What is left is the rounding of y = t / ln 2, 6e-8 |t| at most: enough in front
// of bf16.  In front of fp32 it is put right: exp(t) = 2^y (1 + d), d = t - y ln 2.  There the factor in y is 2.4e-7 too large, so that d lies between 0 and
// 3e-7 |t| (its square is nothing) and the limits that keep the infinity of t = -inf out of it cost no instruction of their own: one more than the other form,
// and gradients off by 4e-8 instead of 2e-7 of their value.
template <typename T>
__device__ __forceinline__ float exp_of(float t) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_exp2f(fmaf(t, 1.4426950216293335f, t * 1.9259629911e-8f));
    const float y = t * 1.44269538f, r = __builtin_amdgcn_exp2f(y);
    return fmaf(r, __builtin_amdgcn_fmed3f(fmaf(y, -0.693147182f, t), 0.f, 1.f), r);
}

// What the kernels know of the logits.  The vectors of all vocabulary tiles are numbered through, `vt` to a tile and `nvec` in all.
struct Logits {
    const int32_t* labels;
    TiledView X;
    int32_t vt, nvec;
    float inv_vt;
    bool away;                                    // gradients leave past the caches
};

// A workgroup's column: where it lies, its label, and the vector that holds the label's logit.
template <typename T>
struct ColumnAt {
    static constexpr int V = RawVec<T>::V;
    Column c;
    bool has;
    int lab_f, lab_j;
    __device__ __forceinline__ ColumnAt(const Logits& a, int64_t col) {
        c = column_of(a.X, col);
        const int lab = a.labels[col];
        has = lab >= 0 && lab < a.X.shape[0];
        const int t = has ? lab / a.X.base[0] : 0, e = lab - t * a.X.base[0];
        lab_f = has ? t * a.vt + e / V : -1;
        lab_j = has ? e % V : 0;
    }
};

// vector f: its tile (the half keeps the product away from an integer), first element, elements that exist
template <typename T>
__device__ __forceinline__ void place(const Logits& a, int f, int& l, int& e, int& cnt) {
    l = (int)(((float)f + 0.5f) * a.inv_vt);
    e = (f - l * a.vt) * RawVec<T>::V;
    cnt = ext0_of(a.X, l) - e;
}

// Addresses of a column's tiles: from LDS, or, of a column with more tiles than the table holds, looked up.
template <typename T>
struct TileBases {
    uint64_t* table;
    void* const* tiles;
    bool in_lds;
    __device__ __forceinline__ T* at(const Logits& a, const Column& c, int l) const {
        if (in_lds) return in_global(reinterpret_cast<T*>(table[l]));
        return global_as<T>(tiles[c.tile0 + l]) + (int64_t)c.colidx * ext0_of(a.X, l);
    }
};
template <typename T>
__device__ __forceinline__ TileBases<T> bases_of(uint64_t* table, void* const* tiles, const Logits& a, const Column& c) {
    const bool in_lds = a.X.grid[0] <= kTableTiles;
    if (in_lds && threadIdx.x < (unsigned)a.X.grid[0])
        table[threadIdx.x] = reinterpret_cast<uint64_t>(global_as<T>(tiles[c.tile0 + threadIdx.x]) + (int64_t)c.colidx * ext0_of(a.X, threadIdx.x));
    return TileBases<T>{table, tiles, in_lds};
}

template <int NW>
__device__ __forceinline__ float block_max(float v, float* red) {
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; w++) v = fmaxf(v, red[w]);
    return v;
}
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
template <int NW>
__device__ __forceinline__ double block_sum64(double v, double* red) {
    v = wave_sum64(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < NW; w++) v += red[w];        // the same order in every thread
    return v;
}

// What the threads of a workgroup exchange.
template <int NW>
struct Exchange {
    float mx[NW];
    float x_label;
    double sum[NW];
};

// Maximum, sum of shifted exponentials and the label's logit of a column that is read once, U vectors per thread at a time:
// a running maximum per thread, the sum rescaled where it moves.  Hundreds of logp add up in a reward, so log(sum) is kept free of an error that all of them
// share: bf16 logits have few different values, each rounded the same way whenever it is added to a large sum, so a thread's sum is put together from
// those of U vectors, and the threads' sums meet in 64 bits.  (One chain of additions: 3.3e-8 off on average, with bf16 logits of 50304.  Now 4e-9
// at most, and 5e-9 to 4e-8 around that.)
template <typename T, int NT, int U>
__device__ __forceinline__ void stream_stats(const Logits& a, const ColumnAt<T>& at, const TileBases<T>& base, Exchange<NT / 64>& red,
                                             float& mx, double& sum, float& x_label) {
    constexpr int V = RawVec<T>::V, NW = NT / 64;
    const int tid = threadIdx.x;
    float m = -__builtin_huge_valf(), s = 0.f;
    // (what is not there counts as -inf: its exponential is 0, and no element needs a test)
    RawVec<T> raw[2][U];
    auto fetch = [&](int set, int f0) {
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int f = f0 + u * NT;
            if (f < a.nvec) {
                int l, e, cnt;
                place<T>(a, f, l, e, cnt);
                raw[set][u].load_or_none(base.at(a, at.c, l) + e, cnt);
            } else {
                raw[set][u].none();
            }
        }
    };
    auto take = [&](int set, int f0) {
        float top = m;
#pragma unroll
        for (int u = 0; u < U; u++) {
#pragma unroll
            for (int j = 0; j < V; j++) top = fmaxf(top, raw[set][u].at(j));
            if (f0 + u * NT == at.lab_f) {
#pragma unroll
                for (int j = 0; j < V; j++)
                    if (j == at.lab_j) red.x_label = raw[set][u].at(j);
            }
        }
        if (top > m) {                       // (the first time m is -inf and s 0)
            s *= exp_of<T>(m - top);
            m = top;
        }
        float part[U];
        const float shift = m == -__builtin_huge_valf() ? 0.f : m;       // nothing but -inf so far: their exponentials are 0, not NaN
#pragma unroll
        for (int u = 0; u < U; u++) {
            part[u] = exp_of<T>(raw[set][u].at(0) - shift);
#pragma unroll
            for (int j = 1; j < V; j++) part[u] += exp_of<T>(raw[set][u].at(j) - shift);
        }
        static_assert(U == 4, "added up in pairs");
        s += (part[0] + part[1]) + (part[2] + part[3]);
    };
    // the next vectors are on their way while these are worked on
    fetch(0, tid);
    for (int f0 = tid; f0 < a.nvec; f0 += 2 * U * NT) {
        fetch(1, f0 + U * NT);
        take(0, f0);
        fetch(0, f0 + 2 * U * NT);
        take(1, f0 + U * NT);
    }
    mx = block_max<NW>(m, red.mx);
    sum = block_sum64<NW>(m == mx ? s : s * exp_of<T>(m - mx), red.sum);
    x_label = red.x_label;
}

// logp in 64 bits: the differences of many of them are added up, and their large parts cancel
__device__ __forceinline__ double logp_of(float x_label, float mx, double sum) {
    return (double)x_label - (double)mx - log(sum);
}

// ---------------------------------------------------------------- log-probabilities
template <typename T, int NT>
__global__ void __launch_bounds__(NT) logprob_kernel(Logits a, float* const* logp) {
    __shared__ uint64_t table[kTableTiles];
    __shared__ Exchange<NT / 64> red;
    const ColumnAt<T> at(a, blockIdx.x);
    float* out = global_as<float>(logp[at.c.stat_tile]) + at.c.colidx;
    if (!at.has) {
        if (threadIdx.x == 0) *out = 0.f;
        return;
    }
    const TileBases<T> base = bases_of<T>(table, a.X.tiles, a, at.c);
    __syncthreads();
    float mx, x_label;
    double sum;
    stream_stats<T, NT, 4>(a, at, base, red, mx, sum, x_label);
    if (threadIdx.x == 0) *out = (float)logp_of(x_label, mx, sum);
}

// ---------------------------------------------------------------- policy loss
struct PolicyArgs {
    const float* const* old_logp;       // tiles of [N_s, N_b] like the logits' other axes; NULL: the present logp
    const float* const* ref_logp;       // NULL: no KL term
    const float* const* adv;
    int32_t adv_per_sequence;           // tiles of [N_b]
    double lo, hi, kl;                  // the clip range's ends, weight of the KL term
    const float* weight;                // per sequence; NULL: 1
    float* const* logp;
    float* losses;
    void* const* dX;                    // NULL: no gradient
};

// loss and dL/dlogp of one position, in 64 bits (one thread of a column): what is rounded to 32 is what is written
__device__ __forceinline__ void policy_of(const Logits& a, const PolicyArgs& p, const Column& c, double logp, float& loss, float& g) {
    const double w = p.weight ? (double)p.weight[c.c2] : 1.0;
    double adv;
    if (p.adv_per_sequence) {
        const int t2 = c.c2 / a.X.base[2];
        adv = (double)global_as<const float>(p.adv[t2])[c.c2 - t2 * a.X.base[2]];
    } else {
        adv = (double)global_as<const float>(p.adv[c.stat_tile])[c.colidx];
    }
    // (against itself: 1, also for a banned token, whose logp is -inf, but NaN for a column that holds one)
    const double d = p.old_logp ? logp - (double)global_as<const float>(p.old_logp[c.stat_tile])[c.colidx] : logp == logp ? 0.0 : logp;
    const double r = exp(d);
    const double free = r * adv, held = fmin(fmax(r, p.lo), p.hi) * adv;
    // (written so that a NaN comes through)
    double l = free > held ? -held : -free, s = free > held ? 0.0 : -free;
    if (p.ref_logp) {
        const double k = (double)global_as<const float>(p.ref_logp[c.stat_tile])[c.colidx] - logp;
        const double ek = expm1(k);
        // e^k - k - 1: the difference of nearly equal numbers around 0 is summed up as k^2/2 + k^3/6 + ...
        l += p.kl * (fabs(k) < 1e-3 ? k * k * (0.5 + k * (1.0 / 6 + k * (1.0 / 24))) : ek - k);
        s -= p.kl * ek;
    }
    loss = (float)(l * w);
    g = (float)(s * w);
}

// One workgroup takes one column.  SLOTS > 0: the column is read once into registers, SLOTS vectors per thread, and the gradient leaves from
// there.  SLOTS = 0: a column too long for that is read twice.
template <typename T, int SLOTS, int NT>
__global__ void __launch_bounds__(NT, (sizeof(T) == 2 && NT == 1024 && SLOTS > 0) ? 8 : 1) policy_kernel(Logits a, PolicyArgs p) {
    constexpr int V = RawVec<T>::V, NW = NT / 64;
    // Vectors that are not there count as -inf, which needs no test; with 64 registers for two workgroups of 1024 per unit the test per vector is what keeps
    // the compiler from unpacking them all at once (6 vectors of bf16: 39 registers spilled, 462 instead of 291 us for 8192 columns of 50304).
    constexpr bool kTests = sizeof(T) == 2 && NT == 1024;
    __shared__ uint64_t table[2][kTableTiles];
    __shared__ Exchange<NW> red;
    __shared__ float g_s;
    const int tid = threadIdx.x;
    const int64_t col = blockIdx.x;
    const ColumnAt<T> at(a, col);
    const TileBases<T> base = bases_of<T>(table[0], a.X.tiles, a, at.c);
    const TileBases<T> out = bases_of<T>(table[1], p.dX ? p.dX : a.X.tiles, a, at.c);
    __syncthreads();
    if (!at.has) {
        if (tid == 0) {
            *(global_as<float>(p.logp[at.c.stat_tile]) + at.c.colidx) = 0.f;
            p.losses[col] = 0.f;
        }
        if (p.dX) {
            const float z[V] = {};
            for (int f = tid; f < a.nvec; f += NT) {
                int l, e, cnt;
                place<T>(a, f, l, e, cnt);
                RawVec<T>::store(out.at(a, at.c, l) + e, z, cnt, a.away);
            }
        }
        return;
    }
    float mx, x_label;
    double sum;
    RawVec<T> raw[SLOTS ? SLOTS : 1];
    if constexpr (SLOTS > 0) {
#pragma unroll
        for (int it = 0; it < SLOTS; it++) {
            const int f = it * NT + tid;
            if (f < a.nvec) {
                int l, e, cnt;
                place<T>(a, f, l, e, cnt);
                raw[it].load_or_none(base.at(a, at.c, l) + e, cnt);
            } else if (!kTests) {
                raw[it].none();
            }
        }
        mx = -__builtin_huge_valf();
#pragma unroll
        for (int it = 0; it < SLOTS; it++) {
            const int f = it * NT + tid;
            if (kTests && f >= a.nvec) continue;
#pragma unroll
            for (int j = 0; j < V; j++) mx = fmaxf(mx, raw[it].at(j));
            if (f == at.lab_f) {
#pragma unroll
                for (int j = 0; j < V; j++)
                    if (j == at.lab_j) red.x_label = raw[it].at(j);
            }
        }
        mx = block_max<NW>(mx, red.mx);
        float s = 0.f;
#pragma unroll
        for (int it = 0; it < SLOTS; it++) {
            if (kTests && it * NT + tid >= a.nvec) continue;
            float part = 0.f;
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float x = exp_of<T>(raw[it].at(j) - mx);
                if (RawVec<T>::kKeeps) raw[it].set(j, x);
                part += x;
            }
            s += part;
        }
        sum = block_sum64<NW>(s, red.sum);
        x_label = red.x_label;
    } else {
        stream_stats<T, NT, 4>(a, at, base, red, mx, sum, x_label);
    }
    if (tid == 0) {
        const double logp = logp_of(x_label, mx, sum);
        float loss, g;
        policy_of(a, p, at.c, logp, loss, g);
        *(global_as<float>(p.logp[at.c.stat_tile]) + at.c.colidx) = (float)logp;
        p.losses[col] = loss;
        g_s = g;
    }
    if (!p.dX) return;
    __syncthreads();
    const float g = g_s, scale = -g / (float)sum;
    auto gradient = [&](int f, int it) {
        int l, e, cnt;
        place<T>(a, f, l, e, cnt);
        RawVec<T> x;
        if constexpr (SLOTS == 0) x.load(base.at(a, at.c, l) + e, cnt);
        float y[V];
#pragma unroll
        for (int j = 0; j < V; j++) {
            if constexpr (SLOTS > 0) y[j] = (RawVec<T>::kKeeps ? raw[it].at(j) : exp_of<T>(raw[it].at(j) - mx)) * scale;
            else y[j] = exp_of<T>(x.at(j) - mx) * scale;
        }
        if (f == at.lab_f) {
#pragma unroll
            for (int j = 0; j < V; j++)
                if (j == at.lab_j) y[j] += g;
        }
        RawVec<T>::store(out.at(a, at.c, l) + e, y, cnt, a.away);
    };
    if constexpr (SLOTS > 0) {
#pragma unroll
        for (int it = 0; it < SLOTS; it++) {
            const int f = it * NT + tid;
            if (f < a.nvec) gradient(f, it);
        }
    } else {
        for (int f = tid; f < a.nvec; f += NT) gradient(f, 0);
    }
}

// weight[b] of a sequence's labelled positions: 1 / (labelled positions), or 1 / (its labelled positions x sequences that have any).
// One workgroup counts them all, several labels of a thread on their way at a time.  Where sequences count, a wavefront takes one at a time, and
// where there are enough of them, or they are short, every thread its own (65536 of 33 positions: 2.5 -> 0.36 ms; 8 of 1024 3 us either way).
__global__ void __launch_bounds__(1024) weights_kernel(const int32_t* labels, int N_v, int N_s, int N_b, int per_sequence, float* weight) {
    __shared__ unsigned long long total[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto labelled = [&](int32_t l) { return l >= 0 && l < N_v ? 1 : 0; };
    unsigned long long mine = 0;                        // labelled positions, or sequences that have any
    if (!per_sequence) {
        const int64_t all = (int64_t)N_s * N_b;
#pragma unroll 8
        for (int64_t i = tid; i < all; i += 1024) mine += labelled(labels[i]);
    } else if (N_s > 32 && N_b < 1024) {
        for (int b = wave; b < N_b; b += 16) {
            const int32_t* l = labels + (int64_t)b * N_s;
            int n = 0;
#pragma unroll 8
            for (int s = lane; s < N_s; s += 64) n += labelled(l[s]);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
            if (lane == 0) {
                weight[b] = n ? 1.f / (float)n : 0.f;
                mine += n > 0;
            }
        }
    } else {
        for (int b = tid; b < N_b; b += 1024) {
            const int32_t* l = labels + (int64_t)b * N_s;
            int n = 0;
#pragma unroll 8
            for (int s = 0; s < N_s; s++) n += labelled(l[s]);
            weight[b] = n ? 1.f / (float)n : 0.f;
            mine += n > 0;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, 64);
    if (lane == 0) total[wave] = mine;
    __syncthreads();                                    // (orders the weights above towards the same workgroup, too)
    unsigned long long all = 0;
#pragma unroll
    for (int w = 0; w < 16; w++) all += total[w];
    const float one = all ? (float)(1.0 / (double)all) : 0.f;
    for (int b = tid; b < N_b; b += 1024) weight[b] = per_sequence ? weight[b] * one : one;
}

// sum of n floats by one workgroup in 64 bits: fixed assignment of elements to lanes, fixed tree
__global__ void __launch_bounds__(1024) total_kernel(const float* x, int64_t n, float* out) {
    __shared__ double part[16];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) s += (double)x[i];
    s = wave_sum64(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
#pragma unroll
        for (int w = 0; w < 16; w++) t += part[w];
        out[0] = (float)t;
    }
}

// ---------------------------------------------------------------- preference loss
// Scratch of a call: per column maximum and sum (2 floats) and logp - ref (1 double), per sequence its reward (1 double).
struct PreferenceScratch {
    float* stats;
    double* diff;
    double* reward;
};

template <typename T, int NT>
__global__ void __launch_bounds__(NT) preference_stats_kernel(Logits a, const float* const* ref, float* const* logp, PreferenceScratch w) {
    __shared__ uint64_t table[kTableTiles];
    __shared__ Exchange<NT / 64> red;
    const int64_t col = blockIdx.x;
    const ColumnAt<T> at(a, col);
    if (!at.has) {
        if (threadIdx.x == 0) {
            *(global_as<float>(logp[at.c.stat_tile]) + at.c.colidx) = 0.f;
            w.diff[col] = 0.0;
        }
        return;
    }
    const TileBases<T> base = bases_of<T>(table, a.X.tiles, a, at.c);
    __syncthreads();
    float mx, x_label;
    double sum;
    stream_stats<T, NT, 4>(a, at, base, red, mx, sum, x_label);
    if (threadIdx.x == 0) {
        const double lp = logp_of(x_label, mx, sum);
        w.diff[col] = lp - (ref ? (double)global_as<const float>(ref[at.c.stat_tile])[at.c.colidx] : 0.0);
        *(global_as<float>(logp[at.c.stat_tile]) + at.c.colidx) = (float)lp;
        w.stats[2 * col] = mx;
        w.stats[2 * col + 1] = (float)sum;
    }
}

// reward of a sequence: one workgroup, fixed order
__global__ void __launch_bounds__(256) reward_kernel(PreferenceScratch w, int N_s, double beta, float* rewards) {
    __shared__ double part[4];
    const double* d = w.diff + (int64_t)blockIdx.x * N_s;
    double s = 0.0;
    for (int i = threadIdx.x; i < N_s; i += 256) s += d[i];
    s = wave_sum64(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = beta * (part[0] + part[1] + part[2] + part[3]);
        w.reward[blockIdx.x] = s;
        rewards[blockIdx.x] = (float)s;
    }
}

// log(1 + e^-z) and 1 / (1 + e^-z) of any z
__device__ __forceinline__ double softplus_neg(double z) { return z > 0.0 ? log1p(exp(-z)) : log1p(exp(z)) - z; }
__device__ __forceinline__ double sigmoid_of(double z) { return z >= 0.0 ? 1.0 / (1.0 + exp(-z)) : exp(z) / (1.0 + exp(z)); }

struct PreferenceArgs {
    double beta, smoothing, weight;      // weight of a pair
    int32_t pairs;
};

// the losses of all pairs and their sum: one workgroup
__global__ void __launch_bounds__(256) preference_total_kernel(PreferenceScratch w, PreferenceArgs p, float* losses, float* loss) {
    __shared__ double part[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < p.pairs; i += 256) {
        const double z = w.reward[i] - w.reward[i + p.pairs];
        double l = (1.0 - p.smoothing) * softplus_neg(z);
        if (p.smoothing > 0.0) l += p.smoothing * softplus_neg(-z);      // (0 times the infinite loss of an infinite margin is none)
        l *= p.weight;
        losses[i] = (float)l;
        s += l;
    }
    s = wave_sum64(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) loss[0] = (float)(part[0] + part[1] + part[2] + part[3]);
}

// The gradient of a column, from the kept statistics.  The columns are taken in the reverse of the order in which their statistics were:
// what was read last is still in the caches.
template <typename T, int NT>
__global__ void __launch_bounds__(NT) preference_gradient_kernel(Logits a, PreferenceScratch w, PreferenceArgs p, void* const* dX) {
    constexpr int V = RawVec<T>::V;
    __shared__ uint64_t table[2][kTableTiles];
    const int tid = threadIdx.x;
    const int64_t col = (int64_t)gridDim.x - 1 - blockIdx.x;
    const ColumnAt<T> at(a, col);
    const TileBases<T> base = bases_of<T>(table[0], a.X.tiles, a, at.c);
    const TileBases<T> out = bases_of<T>(table[1], dX, a, at.c);
    __syncthreads();
    float g = 0.f, mx = 0.f, scale = 0.f;
    if (at.has) {
        const int b = at.c.c2;
        const bool chosen = b < p.pairs;
        const int i = chosen ? b : b - p.pairs;
        const double z = w.reward[i] - w.reward[i + p.pairs];
        const double slope = p.weight * p.beta * (sigmoid_of(z) - (1.0 - p.smoothing));
        g = (float)(chosen ? slope : -slope);
        mx = w.stats[2 * col];
        scale = -g / w.stats[2 * col + 1];
    }
    for (int f = tid; f < a.nvec; f += NT) {
        int l, e, cnt;
        place<T>(a, f, l, e, cnt);
        float y[V] = {};
        if (at.has) {
            RawVec<T> x;
            x.load(base.at(a, at.c, l) + e, cnt);
#pragma unroll
            for (int j = 0; j < V; j++) y[j] = exp_of<T>(x.at(j) - mx) * scale;
            if (f == at.lab_f) {
#pragma unroll
                for (int j = 0; j < V; j++)
                    if (j == at.lab_j) y[j] += g;
            }
        }
        RawVec<T>::store(out.at(a, at.c, l) + e, y, cnt, a.away);
    }
}

// ---------------------------------------------------------------- host side
// Workgroup size of a column.  One wavefront where there are many short columns: what a column costs besides its logits counts then, and 32 of them share
// a compute unit (log-probabilities of 16384 columns of 2000 in bf16 64 -> 22 us, of 8192 of 6513 35 -> 22).  256 threads where a column's vectors fit their
// registers, or where there are so many that several of them share a unit anyway (8192 columns of 50304 in bf16 192 -> 123 us); 1024 for few long ones
// (64 columns of 50304 10 us, 14 with 256).  `streams`: the kernel does not hold the column in registers.
int threads_of(int dtype, int64_t nvec, int64_t ncols, bool streams) {
    if (ncols >= 512 && nvec <= (streams || dtype == NNT_F32 ? 1024 : 512)) return 64;
    if (nvec <= (dtype == NNT_F32 ? 4096 : 2048) || (streams && ncols >= 1024)) return 256;
    return 1024;
}

using PolicyFn = void (*)(Logits, PolicyArgs);
// the instance that holds a column of `nvec` vectors with the fewest registers, and its workgroup size
PolicyFn policy_instance(int dtype, int64_t nvec, int64_t ncols, int* nt) {
    *nt = threads_of(dtype, nvec, ncols, false);
    const int64_t per = (nvec + *nt - 1) / *nt;
    if (dtype == NNT_F32) {
        if (*nt == 64) return per <= 4 ? policy_kernel<float, 4, 64> : policy_kernel<float, 16, 64>;
        if (*nt == 256) return per <= 4 ? policy_kernel<float, 4, 256> : policy_kernel<float, 16, 256>;
        return per <= 8 ? policy_kernel<float, 8, 1024> : per <= 13 ? policy_kernel<float, 13, 1024> : per <= 16 ? policy_kernel<float, 16, 1024> : policy_kernel<float, 0, 1024>;
    }
    if (*nt == 64) return per <= 2 ? policy_kernel<bf16_t, 2, 64> : policy_kernel<bf16_t, 8, 64>;
    if (*nt == 256) return per <= 2 ? policy_kernel<bf16_t, 2, 256> : policy_kernel<bf16_t, 8, 256>;
    return per <= 4 ? policy_kernel<bf16_t, 4, 1024> : per <= 7 ? policy_kernel<bf16_t, 7, 1024> : per <= 8 ? policy_kernel<bf16_t, 8, 1024> : policy_kernel<bf16_t, 0, 1024>;
}

#define NNT_PER_COLUMN(KERNEL, NT, ...)                                                                                      \
    do {                                                                                                                     \
        const dim3 grid((unsigned)ncols);                                                                                    \
        if (dt == NNT_F32) {                                                                                                 \
            if ((NT) == 64) hipLaunchKernelGGL((KERNEL<float, 64>), grid, dim3(64), 0, st, __VA_ARGS__);                     \
            else if ((NT) == 256) hipLaunchKernelGGL((KERNEL<float, 256>), grid, dim3(256), 0, st, __VA_ARGS__);             \
            else hipLaunchKernelGGL((KERNEL<float, 1024>), grid, dim3(1024), 0, st, __VA_ARGS__);                            \
        } else {                                                                                                             \
            if ((NT) == 64) hipLaunchKernelGGL((KERNEL<bf16_t, 64>), grid, dim3(64), 0, st, __VA_ARGS__);                    \
            else if ((NT) == 256) hipLaunchKernelGGL((KERNEL<bf16_t, 256>), grid, dim3(256), 0, st, __VA_ARGS__);            \
            else hipLaunchKernelGGL((KERNEL<bf16_t, 1024>), grid, dim3(1024), 0, st, __VA_ARGS__);                           \
        }                                                                                                                    \
        TRY(launched());                                                                                                     \
    } while (0)

bool all_there(const nnt_tensor* t) {
    for (void* p : t->tiles)
        if (!p) return false;
    return true;
}

// The logits' checks that all entry points share, and what the kernels are told about them.
int32_t take_logits(nnt_ctx* ctx, const std::string& who, nnt_tensor* X, const int32_t* labels, Logits* out) {
    if (X->ctx != ctx) return fail(ctx, NNT_EINVAL, who + ": tensor of another context");
    if (X->ndim != 3) return fail(ctx, NNT_EINVAL, who + ": the logits must be [N_v, N_s, N_b]");
    if (!all_there(X)) return fail(ctx, NNT_EINVAL, who + ": structural-zero tiles not allowed");
    const int64_t V = X->dtype == NNT_F32 ? 4 : 8, vt = (X->base[0] + V - 1) / V;
    const int64_t nvec = vt * (X->grid[0] - 1) + (X->tile_extent(0, X->grid[0] - 1) + V - 1) / V;
    if (nvec > kMaxVectors) return fail(ctx, NNT_EINVAL, who + ": vocabulary too long");
    if (X->shape[1] >= kMaxPositions || X->shape[2] >= kMaxPositions || X->shape[1] * X->shape[2] >= kMaxPositions) return fail(ctx, NNT_EINVAL, who + ": too many positions");
    *out = Logits{labels, X->view(), (int32_t)vt, (int32_t)nvec, 1.f / (float)vt, X->elem_size() * X->shape[0] * X->shape[1] * X->shape[2] > kCached};
    return NNT_OK;
}

// one fp32 value per position: [N_s, N_b], tiled like the logits' other axes
int32_t check_positions(nnt_ctx* ctx, const std::string& who, const char* what, const nnt_tensor* X, const nnt_tensor* t) {
    bool ok = t->ctx == ctx && t->dtype == NNT_F32 && t->ndim == 2 && all_there(t);
    for (int a = 0; ok && a < 2; a++) ok = t->shape[a] == X->shape[a + 1] && t->base[a] == X->base[a + 1];
    return ok ? (int32_t)NNT_OK : fail(ctx, NNT_EINVAL, who + ": " + what + " must be fp32 [N_s, N_b], tiled like the logits' other axes, all tiles present");
}

int32_t check_gradient(nnt_ctx* ctx, const std::string& who, const nnt_tensor* X, const nnt_tensor* dX) {
    if (dX && (dX->ctx != ctx || dX->dtype != X->dtype || !same_tiling(dX, X) || !all_there(dX)))
        return fail(ctx, NNT_EINVAL, who + ": the gradient must have the logits' type, shape and tiling, all tiles present");
    return NNT_OK;
}

int32_t launched() { return hipGetLastError() == hipSuccess ? (int32_t)NNT_OK : (int32_t)NNT_EHIP; }

float* const* out_tiles(nnt_tensor* t) { return reinterpret_cast<float* const*>(t->d_tiles); }
const float* const* in_tiles(nnt_tensor* t) { return t ? reinterpret_cast<const float* const*>(t->d_tiles) : nullptr; }

#define TRY(x)                           \
    do {                                 \
        int32_t rc__ = (x);              \
        if (rc__ != NNT_OK) return rc__; \
    } while (0)

}  // namespace

// What the entry points ask of their arguments, and the scratch that they need: the language model asks before its forward pass.
int32_t token_logprob_check(nnt_ctx* ctx, nnt_tensor* X, const int32_t* labels, nnt_tensor* logp) {
    const std::string who = "nnt_token_logprob";
    if (!X || !labels || !logp) return fail(ctx, NNT_EINVAL, who + ": null argument");
    Logits a;
    TRY(take_logits(ctx, who, X, labels, &a));
    return check_positions(ctx, who, "logp", X, logp);
}

int32_t policy_loss_check(nnt_ctx* ctx, const nnt_policy_cfg* cfg, nnt_tensor* X, const int32_t* labels, nnt_tensor* old_logp, nnt_tensor* ref_logp,
                          nnt_tensor* advantages, nnt_tensor* dX, nnt_tensor* logp, float* losses, float* loss) {
    const std::string who = "nnt_policy_loss";
    if (!cfg || !X || !labels || !advantages || !logp || !losses || !loss) return fail(ctx, NNT_EINVAL, who + ": null argument");
    if (!(cfg->clip_low >= 0.0 && cfg->clip_low <= 1.0) || !(cfg->clip_high >= 0.0 && cfg->clip_high < 1e30) || !(cfg->kl_coef >= 0.0 && cfg->kl_coef < 1e30) ||
        cfg->reduction < NNT_REDUCE_SUM || cfg->reduction > NNT_REDUCE_SEQUENCES)
        return fail(ctx, NNT_EINVAL, who + ": bad configuration");
    if (cfg->kl_coef > 0.0 && !ref_logp) return fail(ctx, NNT_EINVAL, who + ": a KL term needs the reference's log-probabilities");
    Logits a;
    TRY(take_logits(ctx, who, X, labels, &a));
    TRY(check_positions(ctx, who, "logp", X, logp));
    if (old_logp) TRY(check_positions(ctx, who, "old_logp", X, old_logp));
    if (ref_logp) TRY(check_positions(ctx, who, "ref_logp", X, ref_logp));
    if (advantages->ndim == 1) {
        if (advantages->ctx != ctx || advantages->dtype != NNT_F32 || advantages->shape[0] != X->shape[2] || advantages->base[0] != X->base[2] || !all_there(advantages))
            return fail(ctx, NNT_EINVAL, who + ": advantages per sequence must be fp32 [N_b], tiled like the logits' last axis, all tiles present");
    } else {
        TRY(check_positions(ctx, who, "advantages", X, advantages));
    }
    TRY(check_gradient(ctx, who, X, dX));
    if (logp == old_logp || logp == ref_logp || logp == advantages) return fail(ctx, NNT_EINVAL, who + ": logp must not be one of the inputs");
    return cfg->reduction == NNT_REDUCE_SUM ? (int32_t)NNT_OK : ensure_stream_scratch(ctx, X->shape[2]);
}

int32_t preference_loss_check(nnt_ctx* ctx, const nnt_preference_cfg* cfg, nnt_tensor* X, const int32_t* labels, nnt_tensor* ref_logp, nnt_tensor* dX,
                              nnt_tensor* logp, float* rewards, float* losses, float* loss) {
    const std::string who = "nnt_preference_loss";
    if (!cfg || !X || !labels || !logp || !rewards || !losses || !loss) return fail(ctx, NNT_EINVAL, who + ": null argument");
    if (!(cfg->beta > 0.0 && cfg->beta < 1e30) || !(cfg->label_smoothing >= 0.0 && cfg->label_smoothing <= 0.5) ||
        (cfg->reduction != NNT_REDUCE_SUM && cfg->reduction != NNT_REDUCE_SEQUENCES))
        return fail(ctx, NNT_EINVAL, who + ": bad configuration");
    Logits a;
    TRY(take_logits(ctx, who, X, labels, &a));
    if (X->shape[2] % 2) return fail(ctx, NNT_EINVAL, who + ": pairs need an even batch");
    TRY(check_positions(ctx, who, "logp", X, logp));
    if (ref_logp) TRY(check_positions(ctx, who, "ref_logp", X, ref_logp));
    TRY(check_gradient(ctx, who, X, dX));
    if (logp == ref_logp) return fail(ctx, NNT_EINVAL, who + ": logp must not be one of the inputs");
    return ensure_stream_scratch(ctx, 4 * X->shape[1] * X->shape[2] + 2 * X->shape[2]);
}

}  // namespace nnt

using namespace nnt;

int32_t nnt_token_logprob(nnt_ctx* ctx, nnt_tensor* X, const int32_t* labels, nnt_tensor* logp) {
    return entry(ctx, [&]() -> int32_t {
        TRY(token_logprob_check(ctx, X, labels, logp));
        Logits a;
        TRY(take_logits(ctx, "nnt_token_logprob", X, labels, &a));
        const int64_t ncols = X->shape[1] * X->shape[2];
        const int dt = X->dtype;
        float* const* out = out_tiles(logp);
        OpTag tag(ctx, "token_logprob", (double)X->shape[0] * ncols * X->elem_size(), true);
        return submit(ctx, {X->all(kRead), logp->all(kWrite)}, [=](hipStream_t st) {
            NNT_PER_COLUMN(logprob_kernel, threads_of(dt, a.nvec, ncols, true), a, out);
            return (int32_t)NNT_OK;
        });
    });
}

int32_t nnt_policy_loss(nnt_ctx* ctx, const nnt_policy_cfg* cfg, nnt_tensor* X, const int32_t* labels, nnt_tensor* old_logp, nnt_tensor* ref_logp,
                        nnt_tensor* advantages, nnt_tensor* dX, nnt_tensor* logp, float* losses, float* loss) {
    return entry(ctx, [&]() -> int32_t {
        TRY(policy_loss_check(ctx, cfg, X, labels, old_logp, ref_logp, advantages, dX, logp, losses, loss));
        Logits a;
        TRY(take_logits(ctx, "nnt_policy_loss", X, labels, &a));
        const int64_t ncols = X->shape[1] * X->shape[2];
        const int reduction = cfg->reduction;
        int nt;
        const PolicyFn fn = policy_instance(X->dtype, a.nvec, ncols, &nt);
        PolicyArgs p{};
        p.old_logp = in_tiles(old_logp);
        p.ref_logp = cfg->kl_coef > 0.0 ? in_tiles(ref_logp) : nullptr;
        p.adv = in_tiles(advantages);
        p.adv_per_sequence = advantages->ndim == 1;
        p.lo = 1.0 - cfg->clip_low;
        p.hi = 1.0 + cfg->clip_high;
        p.kl = cfg->kl_coef;
        p.logp = out_tiles(logp);
        p.losses = losses;
        p.dX = dX ? dX->d_tiles : nullptr;
        const int N_v = (int)X->shape[0], N_s = (int)X->shape[1], N_b = (int)X->shape[2];
        std::vector<Access> acc{logp->all(kWrite), advantages->all(kRead)};
        if (old_logp) acc.push_back(old_logp->all(kRead));
        if (ref_logp) acc.push_back(ref_logp->all(kRead));
        if (dX == X) acc.push_back(X->all(kReadWrite));
        else acc.push_back(X->all(kRead));
        if (dX && dX != X) acc.push_back(dX->all(kWrite));
        OpTag tag(ctx, "policy_loss", (dX ? 2.0 : 1.0) * (double)X->shape[0] * ncols * X->elem_size(), true);
        return submit(ctx, acc, [=](hipStream_t st) {
            PolicyArgs q = p;
            if (reduction != NNT_REDUCE_SUM) {
                float* weight = stream_scratch_of(ctx);
                hipLaunchKernelGGL(weights_kernel, dim3(1), dim3(1024), 0, st, labels, N_v, N_s, N_b, (int)(reduction == NNT_REDUCE_SEQUENCES), weight);
                TRY(launched());
                q.weight = weight;
            }
            hipLaunchKernelGGL(fn, dim3((unsigned)ncols), dim3((unsigned)nt), 0, st, a, q);
            TRY(launched());
            hipLaunchKernelGGL(total_kernel, dim3(1), dim3(1024), 0, st, losses, ncols, loss);
            return launched();
        }, reduction != NNT_REDUCE_SUM ? 3 : 2);
    });
}

int32_t nnt_preference_loss(nnt_ctx* ctx, const nnt_preference_cfg* cfg, nnt_tensor* X, const int32_t* labels, nnt_tensor* ref_logp, nnt_tensor* dX,
                            nnt_tensor* logp, float* rewards, float* losses, float* loss) {
    return entry(ctx, [&]() -> int32_t {
        TRY(preference_loss_check(ctx, cfg, X, labels, ref_logp, dX, logp, rewards, losses, loss));
        Logits a;
        TRY(take_logits(ctx, "nnt_preference_loss", X, labels, &a));
        const int64_t ncols = X->shape[1] * X->shape[2];
        const int N_s = (int)X->shape[1], N_b = (int)X->shape[2], dt = X->dtype;
        const PreferenceArgs p{cfg->beta, cfg->label_smoothing, cfg->reduction == NNT_REDUCE_SUM ? 1.0 : 2.0 / N_b, N_b / 2};
        const float* const* ref = in_tiles(ref_logp);
        float* const* out = out_tiles(logp);
        void* const* grad = dX ? dX->d_tiles : nullptr;
        std::vector<Access> acc{logp->all(kWrite)};
        if (ref_logp) acc.push_back(ref_logp->all(kRead));
        if (dX == X) acc.push_back(X->all(kReadWrite));
        else acc.push_back(X->all(kRead));
        if (dX && dX != X) acc.push_back(dX->all(kWrite));
        OpTag tag(ctx, "preference_loss", (dX ? 3.0 : 1.0) * (double)X->shape[0] * ncols * X->elem_size(), true);
        return submit(ctx, acc, [=](hipStream_t st) {
            PreferenceScratch w;
            w.diff = reinterpret_cast<double*>(stream_scratch_of(ctx));
            w.reward = w.diff + ncols;
            w.stats = reinterpret_cast<float*>(w.reward + N_b);
            const int nt = threads_of(dt, a.nvec, ncols, true);
            NNT_PER_COLUMN(preference_stats_kernel, nt, a, ref, out, w);
            hipLaunchKernelGGL(reward_kernel, dim3((unsigned)N_b), dim3(256), 0, st, w, N_s, p.beta, rewards);
            TRY(launched());
            // (a column's gradient has no end to wait for: here many threads keep more of it on its way)
            if (grad) NNT_PER_COLUMN(preference_gradient_kernel, threads_of(dt, a.nvec, ncols, false), a, w, p, grad);
            hipLaunchKernelGGL(preference_total_kernel, dim3(1), dim3(256), 0, st, w, p, losses, loss);
            return launched();
        }, grad ? 4 : 3);
    });
}
