// Tokens drawn from logits that are split into vocabulary tiles, with the usual filters: with m the column's largest logit,
//   e_j = exp((x_j - m) / T),  tokens ordered by (x falling, number rising),
//   top-k: the first k;  top-p: of these the shortest prefix whose sum reaches p of theirs;  min-p: e_j >= min_p;
//   token: the first kept number whose running sum (in the order of the numbers) exceeds u times the kept sum.
//
// What is drawn is a whole number that hangs on the borders of running sums, so the weights are taken in 64 bits and summed as
// whole multiples of 2^-shift: sums do not depend on their order, and where a prefix ends is the same question for every
// workgroup size and tiling.
//
// One workgroup per column; each wavefront owns a run of consecutive vectors of it, in registers where they fit.  No column is sorted:
// the place where a prefix ends is found by a histogram over 2048 equal parts of the column's range (which a monotone function of the logit picks,
// so a part is a run of the order), and only the part that holds the border is looked at more closely: sorted in LDS, or, while it
// holds more than a list of 2048, divided again by the bits of its keys.
#include "colwise.hpp"
#include "device_util.hpp"
#include "internal.hpp"
#include "raw_vec.hpp"

#include <algorithm>
#include <cmath>

namespace nnt {
namespace {

constexpr int kBins = 2048;
constexpr int kList = 2048;
constexpr int64_t kMaxVectors = 1 << 20;      // of a column: up to there `place` finds a vector's tile exactly
constexpr float kNegInf = -__builtin_huge_valf();

struct Sample {
    TiledView X;
    const int32_t* columns;
    const float* uniforms;
    int32_t* tokens;
    float* logp;
    int32_t vt, nvec, ncols;          // vectors of a whole tile, of the column; columns of X
    float inv_vt;
    int32_t top_k, greedy, shift;
    double inv_t, top_p, min_p;
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor((unsigned long long)v, o, 64);
    return v;
}
__device__ __forceinline__ uint64_t wave_scan_u64(uint64_t v) {      // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t y = __shfl_up((unsigned long long)v, o, 64);
        if (lane >= o) v += y;
    }
    return v;
}
__device__ __forceinline__ float wave_min(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fminf(v, __shfl_xor(v, o, 64));
    return v;
}

// Order of the logits as whole numbers, and back.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }

// exp(y), y <= 0: 2^n times the series of e^r, |r| <= ln 2 / 2, up to r^12 / 12!; what is left out is below 2e-16 of the value.
__device__ __forceinline__ double exp64(double y) {
    const double n = rint(y * 1.4426950408889634);
    const double r = fma(n, -1.9082149292705877e-10, fma(n, -0.6931471803691238, y));
    double p = 1.0 / 479001600.0;
    p = fma(p, r, 1.0 / 39916800.0);
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return ldexp(p, (int)n);
}

// A column as one workgroup sees it: wavefront w owns the vectors [first, end), row i of them is one vector per lane.  NV rows are held in
// registers; NV = 0: read again whenever they are needed.
template <typename T, int NT, int NV>
struct Held {
    static constexpr int V = RawVec<T>::V;
    static constexpr int NW = NT / 64;
    const Sample& a;
    Column c;
    int first, end;
    float top;              // the column's largest logit (0 where that is +infinity)
    bool top_inf;
    RawVec<T> x[NV > 0 ? NV : 1];

    __device__ __forceinline__ Held(const Sample& s, int64_t col) : a(s) {
        c = column_of(s.X, col);
        const int per = ((s.nvec + NW - 1) / NW + 63) / 64 * 64;
        first = (int)(threadIdx.x >> 6) * per;
        end = min(s.nvec, first + per);
        top = 0.f;
        top_inf = false;
    }
    // vector f: its tile (the half keeps the product away from an integer), first element, elements that exist
    __device__ __forceinline__ void place(int f, int& l, int& e, int& cnt) const {
        l = (int)(((float)f + 0.5f) * a.inv_vt);
        e = (f - l * a.vt) * V;
        cnt = ext0_of(a.X, l) - e;
    }
    __device__ __forceinline__ RawVec<T> read(int f) const {
        RawVec<T> v;
        v.none();
        if (f < end) {
            int l, e, cnt;
            place(f, l, e, cnt);
            v.load_or_none(global_as<const T>(a.X.tiles[c.tile0 + l]) + (int64_t)c.colidx * ext0_of(a.X, l) + e, cnt);
        }
        return v;
    }
    __device__ __forceinline__ void load() {
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; i++) x[i] = read(first + 64 * i + (int)(threadIdx.x & 63));
        }
    }
    // fn(vector number, vector) for all rows, in order, by whole wavefronts (the lanes beyond the end hold -inf)
    template <typename F>
    __device__ __forceinline__ void rows(F&& fn) const {
        const int lane = threadIdx.x & 63;
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; i++)
                if (first + 64 * i < end) fn(first + 64 * i + lane, x[i]);
        } else {
            for (int f = first; f < end; f += 64) fn(f + lane, read(f + lane));
        }
    }
    // the logit as it counts: no NaN, no -0, and where there are infinite ones these alone
    __device__ __forceinline__ float value(const RawVec<T>& v, int j) const {
        float y = v.at(j) + 0.f;
        if (top_inf) return y == __builtin_huge_valf() ? 0.f : kNegInf;
        return y != y ? kNegInf : y;
    }
    __device__ __forceinline__ int number(int f, int j) const {
        int l, e, cnt;
        place(f, l, e, cnt);
        return l * a.X.base[0] + e + j;
    }
    __device__ __forceinline__ double weight64(float y) const { return exp64(((double)y - (double)top) * a.inv_t); }
    // the weight in multiples of 2^-shift
    __device__ __forceinline__ uint64_t weight(float y) const {
        const double t = ((double)y - (double)top) * a.inv_t;
        if (!(t > -40.0)) return 0;
        return (uint64_t)__double_as_longlong(ldexp(exp64(t), a.shift) + 4503599627370496.0) & 0xfffffffffffffull;
    }
};

// Where a prefix of the order ends: kept are the keys above, and of equal ones those with numbers up to `number`.
struct Cut {
    uint32_t key;
    int32_t number;
    __device__ __forceinline__ bool keeps(uint32_t k, int32_t n) const { return k > key || (k == key && n <= number); }
};

template <int NW>
struct Shared {
    union {
        struct {
            unsigned long long mass[kBins];
            uint32_t count[kBins];
        } h;
        unsigned long long list[kList];
    };
    unsigned long long wave[NW];
    double sum[NW];
    float mx[NW], mn[NW];
    unsigned long long before, total;
    uint32_t key, lo, hi;
    int32_t pos, n;
    float x;
};

// Over the NT * PER numbers of a workgroup, PER consecutive ones per thread: where their running sum first passes `ends`, and the sum before
// that place (sh.pos, -1 if nowhere; sh.before).  The sum of all is left in sh.total.
template <int NT, int PER, typename F>
__device__ __forceinline__ void find_end(Shared<NT / 64>& sh, const uint64_t (&v)[PER], uint64_t base, F&& ends) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint64_t s = 0;
#pragma unroll
    for (int i = 0; i < PER; i++) s += v[i];
    const uint64_t scan = wave_scan_u64(s);
    __syncthreads();
    if (lane == 63) sh.wave[w] = scan;
    if (threadIdx.x == 0) sh.pos = -1;
    __syncthreads();
    uint64_t at = base + scan - s, all = base;
#pragma unroll
    for (int k = 0; k < NT / 64; k++) {
        if (k < w) at += sh.wave[k];
        all += sh.wave[k];
    }
    if (threadIdx.x == 0) sh.total = all;
    if (!ends(at, all)) {
        bool found = false;
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const uint64_t next = at + v[i];
            if (!found && ends(next, all)) {
                found = true;
                sh.pos = (int)threadIdx.x * PER + i;
                sh.before = at;
            }
            at = next;
        }
    }
    __syncthreads();
}

// The first number, in the order of the numbers, up to which the weights sum up to more than goal(their total): sh.n (-1: all weights are 0), sh.x its logit.
template <typename T, int NT, int NV, typename W, typename G>
__device__ __forceinline__ void locate(const Held<T, NT, NV>& h, Shared<NT / 64>& sh, W&& weight, G&& goal) {
    constexpr int V = Held<T, NT, NV>::V;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint64_t s = 0;
    h.rows([&](int f, const RawVec<T>& v) {
#pragma unroll
        for (int j = 0; j < V; j++) s += weight(f, j, h.value(v, j));
    });
    s = wave_sum_u64(s);
    __syncthreads();
    if (lane == 0) sh.wave[w] = s;
    if (threadIdx.x == 0) sh.n = -1;
    __syncthreads();
    uint64_t all = 0;
#pragma unroll
    for (int k = 0; k < NT / 64; k++) all += sh.wave[k];
    const uint64_t to = goal(all);
    uint64_t at = 0;
    int winner = -1;
#pragma unroll
    for (int k = 0; k < NT / 64; k++)
        if (winner < 0) {
            if (at + sh.wave[k] > to) winner = k;
            else at += sh.wave[k];
        }
    if (w == winner) {
        bool done = false;
        h.rows([&](int f, const RawVec<T>& v) {
            if (done) return;
            uint64_t p = 0;
#pragma unroll
            for (int j = 0; j < V; j++) p += weight(f, j, h.value(v, j));
            const uint64_t scan = wave_scan_u64(p);
            const uint64_t row = __shfl((unsigned long long)scan, 63, 64);
            if (at + row > to) {
                done = true;
                uint64_t mine = at + scan - p;
                if (mine <= to && mine + p > to) {
                    bool found = false;
#pragma unroll
                    for (int j = 0; j < V; j++) {
                        const float y = h.value(v, j);
                        mine += weight(f, j, y);
                        if (!found && mine > to) {
                            found = true;
                            sh.n = h.number(f, j);
                            sh.x = y;
                        }
                    }
                }
            }
            at += row;
        });
    }
    __syncthreads();
}

// Moves `cut` to where the prefix ends that `ends(running sum, sum of all kept)` says; `kMass`: sums of weights, else of tokens.
template <bool kMass, typename T, int NT, int NV, typename F>
__device__ __forceinline__ void select(const Held<T, NT, NV>& h, Shared<NT / 64>& sh, float range, Cut& cut, F&& ends) {
    constexpr int V = Held<T, NT, NV>::V, PER = kBins / NT;
    const int tid = threadIdx.x;
    const float scale = range > 0.f ? (float)kBins / range : 0.f;      // (0 too for a range beyond fp32: one part)
    uint32_t lo = 0, hi = 0;                                            // the keys that are looked at, and how they are divided
    int bits = -1;                                                      // -1: by the logit
    const Cut old = cut;
    auto part_of = [&](float y, uint32_t key) -> int {
        if (bits < 0) return min(kBins - 1, (int)((h.top - y) * scale));
        return (int)((hi - key) >> bits);
    };
    uint64_t before = 0, all = 0;
    int n = 0, part = 0;
    for (int level = 0;; level++) {
        __syncthreads();
        for (int i = tid; i < kBins; i += NT) {
            sh.h.count[i] = 0;
            sh.h.mass[i] = 0;
        }
        __syncthreads();
        h.rows([&](int f, const RawVec<T>& v) {
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float y = h.value(v, j);
                const uint32_t key = key_of(y);
                if (y == kNegInf || !old.keeps(key, h.number(f, j)) || (bits >= 0 && (key < lo || key > hi))) continue;
                const int b = part_of(y, key);
                atomicAdd(&sh.h.count[b], 1u);
                if (kMass) atomicAdd(&sh.h.mass[b], (unsigned long long)h.weight(y));
            }
        });
        __syncthreads();
        uint64_t v[PER];
#pragma unroll
        for (int i = 0; i < PER; i++) v[i] = kMass ? sh.h.mass[tid * PER + i] : sh.h.count[tid * PER + i];
        if (level == 0) {
            find_end<NT, PER>(sh, v, 0, ends);
            all = sh.total;
        } else {
            find_end<NT, PER>(sh, v, before, [&](uint64_t s, uint64_t) { return ends(s, all); });
        }
        part = sh.pos;
        if (part < 0) return;                                           // the prefix is everything
        before = sh.before;
        n = (int)sh.h.count[part];
        if (n <= kList) break;
        // divide again: the keys of this part are a run of all keys
        __syncthreads();
        if (tid == 0) {
            sh.lo = 0xffffffffu;
            sh.hi = 0;
        }
        __syncthreads();
        uint32_t kl = 0xffffffffu, kh = 0;
        h.rows([&](int f, const RawVec<T>& v) {
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float y = h.value(v, j);
                const uint32_t key = key_of(y);
                if (y == kNegInf || !old.keeps(key, h.number(f, j)) || (bits >= 0 && (key < lo || key > hi)) || part_of(y, key) != part) continue;
                kl = min(kl, key);
                kh = max(kh, key);
            }
        });
        if (kl <= kh) {
            atomicMin(&sh.lo, kl);
            atomicMax(&sh.hi, kh);
        }
        __syncthreads();
        lo = sh.lo;
        hi = sh.hi;
        if (lo == hi) {
            // equal logits: the first `c` of them
            uint64_t c = 1;
            const uint64_t w = kMass ? h.weight(of_key(lo)) : 1;
            uint64_t few = 1, many = (uint64_t)n;                       // (the last of them ends the prefix)
            while (few < many) {
                c = (few + many) / 2;
                if (ends(before + c * w, all)) many = c;
                else few = c + 1;
            }
            c = few;
            locate(h, sh, [&](int f, int j, float y) -> uint64_t { return key_of(y) == lo && old.keeps(lo, h.number(f, j)) ? 1 : 0; },
                   [&](uint64_t) { return c - 1; });
            cut = Cut{lo, sh.n};
            return;
        }
        bits = max(0, 32 - __clz((int)(hi - lo)) - 11);                  // (2^11 parts)
    }
    // the part fits the list: sort it
    __syncthreads();
    int padded = 64;
    while (padded < n) padded *= 2;
    for (int i = tid; i < padded; i += NT) sh.list[i] = ~0ull;
    if (tid == 0) sh.n = 0;
    __syncthreads();
    h.rows([&](int f, const RawVec<T>& v) {
#pragma unroll
        for (int j = 0; j < V; j++) {
            const float y = h.value(v, j);
            const uint32_t key = key_of(y);
            const int number = h.number(f, j);
            if (y == kNegInf || !old.keeps(key, number) || (bits >= 0 && (key < lo || key > hi)) || part_of(y, key) != part) continue;
            sh.list[atomicAdd(&sh.n, 1)] = ((uint64_t)~key << 32) | (uint32_t)number;
        }
    });
    __syncthreads();
    for (int size = 2; size <= padded; size *= 2)
        for (int step = size / 2; step > 0; step /= 2) {
            for (int i = tid; i < padded / 2; i += NT) {
                const int p = 2 * i - (i & (step - 1)), q = p + step;
                const unsigned long long x = sh.list[p], y = sh.list[q];
                if ((x > y) == ((p & size) == 0)) {
                    sh.list[p] = y;
                    sh.list[q] = x;
                }
            }
            __syncthreads();
        }
    uint64_t v[kList / NT];
#pragma unroll
    for (int i = 0; i < kList / NT; i++) {
        const int k = tid * (kList / NT) + i;
        v[i] = k >= n ? 0 : kMass ? h.weight(of_key(~(uint32_t)(sh.list[k] >> 32))) : 1;
    }
    find_end<NT, kList / NT>(sh, v, before, [&](uint64_t s, uint64_t) { return ends(s, all); });
    const unsigned long long last = sh.list[max(0, sh.pos)];
    cut = Cut{~(uint32_t)(last >> 32), (int32_t)(uint32_t)last};
    __syncthreads();
}

template <typename T, int NT, int NV>
__global__ void __launch_bounds__(NT) sample_kernel(Sample a) {
    constexpr int V = RawVec<T>::V, NW = NT / 64;
    __shared__ Shared<NW> sh;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t col = a.columns ? a.columns[blockIdx.x] : (int)blockIdx.x;
    if (col < 0 || col >= a.ncols) {
        if (tid == 0) {
            a.tokens[blockIdx.x] = -1;
            if (a.logp) a.logp[blockIdx.x] = 0.f;
        }
        return;
    }
    Held<T, NT, NV> h(a, col);
    h.load();
    float mx = kNegInf, mn = __builtin_huge_valf();
    h.rows([&](int, const RawVec<T>& v) {
#pragma unroll
        for (int j = 0; j < V; j++) {
            const float y = h.value(v, j);
            mx = fmaxf(mx, y);
            if (y > kNegInf) mn = fminf(mn, y);
        }
    });
    mx = wave_max(mx);
    mn = wave_min(mn);
    if (lane == 0) {
        sh.mx[w] = mx;
        sh.mn[w] = mn;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NW; k++) {
        mx = fmaxf(mx, sh.mx[k]);
        mn = fminf(mn, sh.mn[k]);
    }
    if (mx == kNegInf) {
        if (tid == 0) {
            a.tokens[blockIdx.x] = -1;
            if (a.logp) a.logp[blockIdx.x] = 0.f;
        }
        return;
    }
    h.top_inf = mx == __builtin_huge_valf();
    h.top = h.top_inf ? 0.f : mx;
    if (h.top_inf) mn = 0.f;
    double sum = 0.0;
    if (a.logp) {
        h.rows([&](int, const RawVec<T>& v) {
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < V; j++) s += expf(h.value(v, j) - h.top);
            sum += (double)s;
        });
        sum = wave_sum64(sum);
        if (lane == 0) sh.sum[w] = sum;
    }
    if (a.greedy) {
        locate(h, sh, [&](int, int, float y) -> uint64_t { return y == h.top ? 1 : 0; }, [](uint64_t) -> uint64_t { return 0; });
    } else {
        Cut cut{0, INT32_MAX};
        const float range = h.top - mn;
        if (a.top_k > 0 && a.top_k < a.X.shape[0]) select<false>(h, sh, range, cut, [&](uint64_t s, uint64_t) { return s >= (uint64_t)a.top_k; });
        if (a.top_p < 1.0) select<true>(h, sh, range, cut, [&](uint64_t s, uint64_t all) { return (double)s >= a.top_p * (double)all; });
        const float u = fminf(fmaxf(a.uniforms[blockIdx.x], 0.f), 0.99999994f);
        locate(h, sh,
               [&](int f, int j, float y) -> uint64_t {
                   if (y == kNegInf || !cut.keeps(key_of(y), h.number(f, j))) return 0;
                   if (a.min_p > 0.0 && !(h.weight64(y) >= a.min_p)) return 0;
                   return h.weight(y);
               },
               [&](uint64_t all) -> uint64_t { return (uint64_t)((double)u * (double)all); });
    }
    if (tid == 0) {
        a.tokens[blockIdx.x] = sh.n;
        if (a.logp) {
            sum = 0.0;
            for (int k = 0; k < NW; k++) sum += sh.sum[k];
            a.logp[blockIdx.x] = (float)((double)sh.x - (double)h.top - log(sum));
        }
    }
}

int32_t launched() { return hipGetLastError() == hipSuccess ? (int32_t)NNT_OK : (int32_t)NNT_EHIP; }

#define TRY(x)                           \
    do {                                 \
        int32_t rc__ = (x);              \
        if (rc__ != NNT_OK) return rc__; \
    } while (0)

using SampleFn = void (*)(Sample);
SampleFn sample_instance(int dtype, int64_t nvec, int* nt) {
    *nt = nvec <= 1024 ? 256 : 1024;
    if (dtype == NNT_F32) return *nt == 256 ? sample_kernel<float, 256, 0> : sample_kernel<float, 1024, 0>;
    return *nt == 256 ? sample_kernel<bf16_t, 256, 0> : sample_kernel<bf16_t, 1024, 0>;
}

int64_t vectors_of(const nnt_tensor* X, int64_t* vt) {
    const int64_t V = X->dtype == NNT_F32 ? 4 : 8;
    *vt = (X->base[0] + V - 1) / V;
    return *vt * (X->grid[0] - 1) + (X->tile_extent(0, X->grid[0] - 1) + V - 1) / V;
}

}  // namespace

int32_t sample_check(nnt_ctx* ctx, const nnt_sample_cfg* cfg, nnt_tensor* X, const int32_t* columns, int32_t n, const float* uniforms, const int32_t* tokens) {
    const std::string who = "nnt_sample_tokens";
    if (!cfg || !X || !uniforms || !tokens) return fail(ctx, NNT_EINVAL, who + ": null argument");
    if (!(cfg->temperature >= 0.0 && cfg->temperature < 1e30) || !(cfg->top_p > 0.0 && cfg->top_p <= 1.0) || !(cfg->min_p >= 0.0 && cfg->min_p <= 1.0) || cfg->top_k < 0)
        return fail(ctx, NNT_EINVAL, who + ": bad configuration");
    if (X->ctx != ctx) return fail(ctx, NNT_EINVAL, who + ": tensor of another context");
    if (X->ndim != 3) return fail(ctx, NNT_EINVAL, who + ": the logits must be [N_v, N_s, N_b]");
    for (void* p : X->tiles)
        if (!p) return fail(ctx, NNT_EINVAL, who + ": structural-zero tiles not allowed");
    int64_t vt;
    if (vectors_of(X, &vt) > kMaxVectors) return fail(ctx, NNT_EINVAL, who + ": vocabulary too long");
    if (X->shape[1] > INT32_MAX || X->shape[2] > INT32_MAX || X->shape[1] * X->shape[2] > INT32_MAX) return fail(ctx, NNT_EINVAL, who + ": too many positions");
    if (n < 1 || n >= (1 << 22) || (!columns && n > X->shape[1] * X->shape[2])) return fail(ctx, NNT_EINVAL, who + ": 1 to 2^22 - 1 columns, without a list no more than there are");
    return NNT_OK;
}

int32_t sample_ordered(nnt_ctx* ctx, const nnt_sample_cfg* cfg, nnt_tensor* X, const int32_t* columns, int32_t n, const float* uniforms, int32_t* tokens,
                       float* logp, nnt_tensor* after) {
    TRY(sample_check(ctx, cfg, X, columns, n, uniforms, tokens));
    Sample a{};
    int64_t vt;
    const int64_t nvec = vectors_of(X, &vt);
    a.X = X->view();
    a.columns = columns;
    a.uniforms = uniforms;
    a.tokens = tokens;
    a.logp = logp;
    a.vt = (int32_t)vt;
    a.nvec = (int32_t)nvec;
    a.ncols = (int32_t)(X->shape[1] * X->shape[2]);
    a.inv_vt = 1.f / (float)vt;
    a.top_k = cfg->top_k;
    a.greedy = cfg->temperature == 0.0;
    a.inv_t = a.greedy ? 1.0 : std::min(1.0 / cfg->temperature, 1e300);
    a.top_p = cfg->top_p;
    a.min_p = cfg->min_p;
    // the sum of a column's weights, 1 at most each, stays below 2^62
    int log_n = 0;
    while (((int64_t)1 << log_n) < X->shape[0]) log_n++;
    a.shift = std::min(51, 62 - log_n);
    int nt;
    const SampleFn fn = sample_instance(X->dtype, nvec, &nt);
    std::vector<Access> acc;
    if (after) after->whole_access(kReadWrite, &acc);
    acc.push_back(X->all(kRead));
    OpTag tag(ctx, "sample_tokens", (double)X->shape[0] * n * X->elem_size(), true);
    TRY(submit(ctx, acc, [=](hipStream_t st) {
        hipLaunchKernelGGL(fn, dim3((unsigned)n), dim3((unsigned)nt), 0, st, a);
        return launched();
    }));
    if (after) after->whole_submitted();
    return NNT_OK;
}

}  // namespace nnt

using namespace nnt;

int32_t nnt_sample_tokens(nnt_ctx* ctx, const nnt_sample_cfg* cfg, nnt_tensor* X, const int32_t* columns, int32_t n, const float* uniforms,
                          int32_t* tokens, float* logp) {
    return entry(ctx, [&]() -> int32_t { return sample_ordered(ctx, cfg, X, columns, n, uniforms, tokens, logp, nullptr); });
}
