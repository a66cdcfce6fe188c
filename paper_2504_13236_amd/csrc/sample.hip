// Tokens drawn from logits that are split into vocabulary tiles, with the usual filters: with m the column's largest logit,
//   e_j = exp((x_j - m) / T),  tokens ordered by (x falling, number rising),
//   top-k: the first k;  top-p: of these the shortest prefix whose sum reaches p of theirs;  min-p: e_j >= min_p;
//   token: the first kept number whose running sum (in the order of the numbers) exceeds u times the kept sum.
//
// What is drawn is a whole number that hangs on the borders of running sums, so the weights are taken in 64 bits and summed as
// whole multiples of 2^-shift: sums do not depend on their order, and where a prefix ends is the same question for every
// workgroup size and tiling.
//
// One workgroup per column.  T = 0 takes the largest in one read.  Else: no column is sorted; all filters come to one border (a logit, and the last number among equal ones), and the draw is one
// pass over the column in the order of the numbers.  Where the border lies:
//   bf16 columns of more than 1024 vectors of eight: the column is counted in LDS by 5120 codes, the bits of what is neither tiny nor huge.  There are few different values, so weights,
//     sums and borders are those of some thousand (value, count) pairs.  Columns with too much that has no code go the ways below.
//   fp32 and shorter bf16 columns, top-k of up to half the workgroup's threads (128 for columns of up to 1024 vectors, 512 for longer fp32 ones): the k-th largest of the threads' largest logits is
//     at most the k-th largest of all, and little more than k logits are at least as large: they are sorted in LDS.
//   else: a histogram over 2048 equal parts of the column's range (which a monotone function of the logit picks, so a part is a run
//     of the order); the part that holds the border is sorted in LDS, or, while it holds more than a list of 2048, divided again by the bits of its keys.
//
// Bound by instructions and LDS, not by memory: 1024 bf16 columns of 50304, top-p, 67 us (103 MB: 21 us at a copy's rate; before the last step 75, vector units 65 % busy, LDS 30 to 35 %), 64 fp32
// columns of 100003, min-p, 26 us, one of 50304, top-k, 14 us.  These and the other figures here are of calls one after the other on two streams, which overlap where one does not fill the chip;
// a call that is waited for, as in a generation that draws token after token, takes 82, 53 and 29 us.  More columns than units are what it is made for: a column over several of them would need a second launch.
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
constexpr int kTableTiles = 64;               // vocabulary tiles whose addresses a workgroup keeps in LDS
constexpr int64_t kMaxVectors = 1 << 20;      // of a column: up to there `place` finds a vector's tile exactly
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kPosInf = __builtin_huge_valf();
constexpr double kLog2e = 1.4426950408889634;

struct Sample {
    TiledView X;
    const int32_t* columns;
    const float* uniforms;
    int32_t* tokens;
    float* logp;
    int32_t vt, nvec, ncols;          // vectors of a whole tile, of the column; columns of X
    float inv_vt;
    int32_t top_k, shift;
    double c;                         // 1 / (T ln 2)
    double top_p;
    double min_fall;                  // T log(min_p): how far below the largest logit a kept one may lie
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
// Inclusive sums over a wavefront's lanes: rows of 16 lanes by shifts, then the rows' last lanes into the rows behind them (data-parallel moves: a few cycles a step,
// where a lane exchange through LDS takes a hundred).
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, kRows, 0xf, false); }
template <int kCtrl, int kRows>
__device__ __forceinline__ uint64_t moved(uint64_t v) { return (uint64_t)moved<kCtrl, kRows>((uint32_t)(v >> 32)) << 32 | moved<kCtrl, kRows>((uint32_t)v); }
template <typename U>
__device__ __forceinline__ U wave_scan(U v) {
    v += moved<0x111, 0xf>(v);
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);
    v += moved<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ uint32_t last_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, 63); }
__device__ __forceinline__ uint64_t last_lane(uint64_t v) { return (uint64_t)last_lane((uint32_t)(v >> 32)) << 32 | last_lane((uint32_t)v); }
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

// 2^(y + shift) as a whole number, -60 <= y <= 0, 0 <= shift <= 51: 2^n (n next to y) is an exponent, 2^(y - n) the polynomial of degree 10 that agrees with it
// at the eleven Chebyshev points of [-1/2, 1/2] (off by at most 4e-16; fitted in extended precision).
__device__ __forceinline__ double exp2_scaled(double y, int shift) {
    const double magic = 6755399441055744.0;              // 3 * 2^51: the sum's low word is the whole number next to y
    const double t = y + magic;
    const double r = y - (t - magic);
    double p = 7.072582572548229e-09;
    p = fma(p, r, 1.0208690372639245e-07);
    p = fma(p, r, 1.3215442609276775e-06);
    p = fma(p, r, 1.525265725977902e-05);
    p = fma(p, r, 0.0001540353044168443);
    p = fma(p, r, 0.0013333558230165855);
    p = fma(p, r, 0.009618129107606949);
    p = fma(p, r, 0.05550410866444771);
    p = fma(p, r, 0.24022650695910097);
    p = fma(p, r, 0.69314718055995);
    p = fma(p, r, 1.0);
    return __hiloint2double(__double2hiint(p) + ((__double2loint(t) + shift) << 20), __double2loint(p));
}
// exp((x - m) / T) in multiples of 2^-shift; below 2^-60 it is 0 anyhow
__device__ __forceinline__ uint64_t weight_of(const Sample& a, float x, double m) {
    const double y = fmax(((double)x - m) * a.c, -60.0);
    return (uint64_t)__double_as_longlong(exp2_scaled(y, a.shift) + 4503599627370496.0) & 0xfffffffffffffull;
}

// exp(t), t <= 0, for log-probabilities: both factors of t / ln 2 are kept, else all of them would be too small by the rounding of the first.
__device__ __forceinline__ float exp_of(float t) { return __builtin_amdgcn_exp2f(fmaf(t, 1.4426950216293335f, t * 1.9259629911e-8f)); }

// Where the kept logits end: kept are the ones above, and of equal ones the first `ties`, which have numbers up to `number`.
struct Cut {
    float x;
    uint32_t ties;
    int32_t number;
};

template <int NT>
struct Shared {
    unsigned long long wave[NT / 64];
    uint32_t ties[NT / 64];
    uint64_t table[kTableTiles];
    double sum[NT / 64];
    float mx[NT / 64], mn[NT / 64];
    unsigned long long before, total;
    uint32_t lo, hi;
    int32_t pos, n;
    float x;
};

// A column as one workgroup sees it.
template <typename T, int NT>
struct Column_ {
    static constexpr int V = RawVec<T>::V;
    static constexpr int NW = NT / 64;
    const Sample& a;
    Shared<NT>& sh;
    Column c;
    bool in_lds;
    float top;              // the column's largest logit (0 where that is +infinity)
    bool top_inf;
    double top64;

    __device__ __forceinline__ Column_(const Sample& s, Shared<NT>& shared, int64_t col) : a(s), sh(shared) {
        c = column_of(s.X, col);
        in_lds = s.X.grid[0] <= kTableTiles;
        if (in_lds && threadIdx.x < (unsigned)s.X.grid[0])
            sh.table[threadIdx.x] = reinterpret_cast<uint64_t>(global_as<const T>(s.X.tiles[c.tile0 + threadIdx.x]) + (int64_t)c.colidx * ext0_of(s.X, threadIdx.x));
        top = 0.f;
        top_inf = false;
        top64 = 0.0;
    }
    __device__ __forceinline__ void set_top(float m) {
        top_inf = m == kPosInf;
        top = top_inf ? 0.f : m;
        top64 = (double)top;
    }
    // vector f: its tile (the half keeps the product away from an integer), first element, elements that exist
    __device__ __forceinline__ void place(int f, int& l, int& e, int& cnt) const {
        l = (int)(((float)f + 0.5f) * a.inv_vt);
        e = (f - l * a.vt) * V;
        cnt = ext0_of(a.X, l) - e;
    }
    __device__ __forceinline__ RawVec<T> read(int f, int end) const {
        RawVec<T> v;
        v.none();
        if (f < end) {
            int l, e, cnt;
            place(f, l, e, cnt);
            v.load_or_none(tile_of(l) + e, cnt);
        }
        return v;
    }
    __device__ __forceinline__ const T* tile_of(int l) const {
        return in_lds ? in_global(reinterpret_cast<const T*>(sh.table[l])) : global_as<const T>(a.X.tiles[c.tile0 + l]) + (int64_t)c.colidx * ext0_of(a.X, l);
    }
    // fn(vector number, vector) for the vectors [lo, hi), tile by tile, row after row of 64, D rows on their way (the lanes beyond the end hold -inf)
    template <int D, typename F>
    __device__ __forceinline__ void rows(int lo, int hi, F&& fn) const {
        const int lane = threadIdx.x & 63;
        for (int f = lo; f < hi;) {
            const int l = __builtin_amdgcn_readfirstlane((int)(((float)f + 0.5f) * a.inv_vt));
            const int first = l * a.vt, end = min(hi, first + a.vt), ext = ext0_of(a.X, l);
            const int whole = min(end, first + ext / V);               // (a tile's last vector may be short)
            const T* p = tile_of(l);
            for (; f < whole; f += 64 * D) {
                const T* at = p + (f - first + lane) * V;
                RawVec<T> v[D];
#pragma unroll
                for (int d = 0; d < D; d++) {
                    v[d].none();
                    if (f + 64 * d + lane < whole) v[d].load(at + 64 * d * V, V);
                }
#pragma unroll
                for (int d = 0; d < D; d++)
                    if (f + 64 * d < whole) fn(f + 64 * d + lane, v[d]);
            }
            if (whole < end) {
                RawVec<T> v;
                v.none();
                if (lane == 0) v.load_or_none(p + (whole - first) * V, ext - (whole - first) * V);
                fn(whole + lane, v);
            }
            f = end;
        }
    }
    // this wavefront's share of [lo, hi): whole 128-byte lines, consecutive ones
    __device__ __forceinline__ void share(int lo, int hi, int& first, int& end) const {
        const int per = ((hi - lo + NW - 1) / NW + 7) / 8 * 8;
        first = lo + (int)(threadIdx.x >> 6) * per;
        end = min(hi, first + per);
    }
    template <int D, typename F>
    __device__ __forceinline__ void all_rows(F&& fn) const {
        int first, end;
        share(0, a.nvec, first, end);
        rows<D>(first, end, fn);
    }
    // the logit as it counts: where there are infinite ones these alone
    __device__ __forceinline__ float value(const RawVec<T>& v, int j) const {
        const float y = v.at(j);
        return top_inf ? (y == kPosInf ? 0.f : kNegInf) : y;
    }
    // ... and as a key: no NaN, no -0
    __device__ __forceinline__ float clean(const RawVec<T>& v, int j) const {
        const float y = value(v, j) + 0.f;
        return y != y ? kNegInf : y;
    }
    __device__ __forceinline__ int number(int f, int j) const {
        int l, e, cnt;
        place(f, l, e, cnt);
        return l * a.X.base[0] + e + j;
    }
    __device__ __forceinline__ uint64_t weight(float y) const { return weight_of(a, y, top64); }
};

// Over the NT * PER numbers of a workgroup, v(0) .. v(PER - 1) of each thread, consecutive ones: where their running sum first passes `ends`, and the sum before
// that place (sh.pos, -1 if nowhere; sh.before).  The sum of all is left in sh.total.
template <int NT, int PER, typename W, typename F>
__device__ __forceinline__ void find_end(Shared<NT>& sh, uint64_t base, W&& v, F&& ends) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint64_t s = 0;
#pragma unroll
    for (int i = 0; i < PER; i++) s += v(i);
    const uint64_t scan = wave_scan(s);
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
    if (!ends(at, all) && ends(at + s, all)) {
        bool found = false;
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const uint64_t next = at + v(i);
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

// The first number, in the order of the numbers, up to which the weights sum up to more than goal(their total): sh.n, sh.x its logit.
// weigh(vector number, vector, weights) gives the weights of a vector's logits above the border and says (by bits) which are equal to it: of these the first
// `limit` of the column have the weight `tie`.  Each wavefront sums an equal share of the vectors, the share that holds the place is divided
// again, until there is one vector per thread.  add(vector, sum, equals) does what the sums of a share need of it.
template <int D, typename T, int NT, typename A, typename W, typename G>
__device__ __forceinline__ void locate_by(const Column_<T, NT>& h, uint64_t tie, uint32_t limit, A&& add, W&& weigh, G&& goal) {
    constexpr int V = Column_<T, NT>::V, NW = NT / 64;
    Shared<NT>& sh = h.sh;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int lo = 0, hi = h.a.nvec;
    uint64_t at = 0, to = 0;
    uint32_t ties_at = 0;
    bool first = true;
    auto kept = [&](uint32_t before, uint32_t n) { return (uint64_t)(before >= limit ? 0u : min(limit - before, n)); };
    while (hi - lo > NT) {
        int begin, end;
        h.share(lo, hi, begin, end);
        uint64_t s = 0;
        uint32_t ties = 0;
        h.template rows<D>(begin, end, [&](int, const RawVec<T>& v) { add(v, s, ties); });
        s = wave_scan(s);
        ties = wave_scan(ties);
        __syncthreads();
        if (lane == 63) {
            sh.wave[w] = s;
            sh.ties[w] = ties;
        }
        __syncthreads();
        if (first) {
            uint64_t all = 0;
            uint32_t t = 0;
#pragma unroll
            for (int k = 0; k < NW; k++) {
                all += sh.wave[k] + kept(t, sh.ties[k]) * tie;
                t += sh.ties[k];
            }
            to = goal(all);
            first = false;
        }
        const int per = ((hi - lo + NW - 1) / NW + 7) / 8 * 8;
        int winner = NW - 1;
#pragma unroll
        for (int k = 0; k < NW - 1; k++)
            if (winner == NW - 1) {
                const uint64_t next = at + sh.wave[k] + kept(ties_at, sh.ties[k]) * tie;
                if (next > to) {
                    winner = k;
                } else {
                    at = next;
                    ties_at += sh.ties[k];
                }
            }
        lo += winner * per;
        hi = min(hi, lo + per);
    }
    uint64_t p[V], s = 0;
    const int f = lo + (int)threadIdx.x;
    const RawVec<T> v = h.read(f, hi);
    const uint32_t equal = weigh(v, p);
#pragma unroll
    for (int j = 0; j < V; j++) s += p[j];
    const uint64_t scan = wave_scan(s);
    const uint32_t ties = wave_scan((uint32_t)__popc(equal));
    __syncthreads();
    if (lane == 63) {
        sh.wave[w] = scan;
        sh.ties[w] = ties;
    }
    if (threadIdx.x == 0) sh.n = -1;
    __syncthreads();
    // the sum in front of this thread's vector, its equals counted first
    uint64_t mine = at + scan - s, all = at;
    uint32_t t_mine = ties_at + ties - __popc(equal), t_all = ties_at;
#pragma unroll
    for (int k = 0; k < NW; k++) {
        if (k < w) {
            mine += sh.wave[k];
            t_mine += sh.ties[k];
        }
        all += sh.wave[k];
        t_all += sh.ties[k];
    }
    mine += kept(ties_at, t_mine - ties_at) * tie;
    if (first) to = goal(all + kept(0, t_all) * tie);
    const uint64_t end_mine = mine + s + kept(t_mine, __popc(equal)) * tie;
    if (mine <= to && end_mine > to) {
        int found = -1;
        uint32_t t = t_mine;
#pragma unroll
        for (int j = 0; j < V; j++) {
            const bool is_tie = (equal >> j) & 1u;
            mine += is_tie ? kept(t, 1) * tie : p[j];
            t += is_tie ? 1 : 0;
            if (found < 0 && mine > to) {
                found = j;
                sh.x = h.value(v, j);
            }
        }
        sh.n = h.number(f, found);
    }
    __syncthreads();
}

// ... by what `weigh` says
template <typename T, int NT, typename W, typename G>
__device__ __forceinline__ void locate(const Column_<T, NT>& h, uint64_t tie, uint32_t limit, W&& weigh, G&& goal) {
    constexpr int V = Column_<T, NT>::V;
    locate_by<2>(h, tie, limit,
           [&](const RawVec<T>& v, uint64_t& s, uint32_t& ties) {
               uint64_t p[V];
               ties += __popc(weigh(v, p));
#pragma unroll
               for (int j = 0; j < V; j++) s += p[j];
           },
           weigh, goal);
}

// The c-th (from 0) number whose logit is `x`.
template <typename T, int NT>
__device__ __forceinline__ int32_t number_of_equal(const Column_<T, NT>& h, float x, uint64_t c) {
    constexpr int V = Column_<T, NT>::V;
    locate_by<4>(h, 1, 0xffffffffu,
           [&](const RawVec<T>& v, uint64_t&, uint32_t& ties) {
#pragma unroll
               for (int j = 0; j < V; j++) ties += h.value(v, j) == x ? 1 : 0;
           },
           [&](const RawVec<T>& v, uint64_t (&p)[V]) {
               uint32_t equal = 0;
#pragma unroll
               for (int j = 0; j < V; j++) {
                   p[j] = 0;
                   equal |= h.value(v, j) == x ? 1u << j : 0u;
               }
               return equal;
           },
           [&](uint64_t) { return c; });
    return h.sh.n;
}

// how many of n equal weights w it takes to end a prefix that the sum `before` does not end and all of them do
template <typename F>
__device__ __forceinline__ uint64_t how_many(uint64_t before, uint64_t w, uint64_t n, uint64_t all, F&& ends) {
    uint64_t few = 1, many = n;
    while (few < many) {
        const uint64_t c = (few + many) / 2;
        if (ends(before + c * w, all)) many = c;
        else few = c + 1;
    }
    return few;
}

// The border with the third filter: nothing too far below the largest logit.
__device__ __forceinline__ Cut with_least(const Sample& a, float top, Cut cut) {
    if (a.min_fall < -1e300) return cut;
    // the largest logit that is too far below
    const double least = (double)top + a.min_fall;
    float y = (float)least;
    if ((double)y >= least) y = nextafterf(y, kNegInf);
    return y >= cut.x ? Cut{y, 0u, -1} : cut;
}
__device__ __forceinline__ uint64_t share_of(float u, uint64_t all) { return (uint64_t)((double)u * (double)all); }

// The draw, once the border is known: the column's second read, weights only where a wavefront holds something above the border.
template <typename T, int NT>
__device__ __forceinline__ void draw(const Column_<T, NT>& h, Cut cut, float u) {
    constexpr int V = Column_<T, NT>::V;
    locate(h, cut.ties ? h.weight(cut.x) : 0, cut.ties,
           [&](const RawVec<T>& v, uint64_t (&p)[V]) {
               bool any = false;
               uint32_t equal = 0;
#pragma unroll
               for (int j = 0; j < V; j++) {
                   any = any || h.value(v, j) > cut.x;
                   equal |= h.value(v, j) == cut.x ? 1u << j : 0u;
                   p[j] = 0;
               }
               if (__any(any)) {
#pragma unroll
                   for (int j = 0; j < V; j++) {
                       const uint64_t w = h.weight(h.value(v, j));
                       p[j] = h.value(v, j) > cut.x ? w : 0;
                   }
               }
               return equal;
           },
           [&](uint64_t all) { return share_of(u, all); });
}

__device__ __forceinline__ float random_of(const Sample& a) { return fminf(fmaxf(a.uniforms[blockIdx.x], 0.f), 0.99999994f); }

__device__ __forceinline__ void no_token(const Sample& a) {
    if (threadIdx.x == 0) {
        a.tokens[blockIdx.x] = -1;
        if (a.logp) a.logp[blockIdx.x] = 0.f;
    }
}
template <int NT>
__device__ __forceinline__ void answer(const Sample& a, const Shared<NT>& sh, float top, double sum) {
    if (threadIdx.x == 0) {
        a.tokens[blockIdx.x] = sh.n;
        if (a.logp) a.logp[blockIdx.x] = (float)((double)sh.x - (double)top - log(sum));
    }
}

// ---------------------------------------------------------------- any column
constexpr int kMostListed = 512;              // top_k up to which the threads' largest logits are asked
struct Parts {
    union {
        struct {
            unsigned long long mass[kBins];
            uint32_t count[kBins];
        } h;
        struct {
            unsigned long long list[kList];
            unsigned long long weight[kMostListed];
        };
    };
};

// sorts list[0 .. n) (n <= kList) by rising values
template <int NT>
__device__ __forceinline__ void sort_list(unsigned long long* list, int n) {
    int padded = 64;
    while (padded < n) padded *= 2;
    for (int i = n + (int)threadIdx.x; i < padded; i += NT) list[i] = ~0ull;
    __syncthreads();
    for (int size = 2; size <= padded; size *= 2)
        for (int step = size / 2; step > 0; step /= 2) {
            for (int i = threadIdx.x; i < padded / 2; i += NT) {
                const int p = 2 * i - (i & (step - 1)), q = p + step;
                const unsigned long long x = list[p], y = list[q];
                if ((x > y) == ((p & size) == 0)) {
                    list[p] = y;
                    list[q] = x;
                }
            }
            __syncthreads();
        }
}
// the order as a whole number: falling logits, rising numbers
__device__ __forceinline__ unsigned long long entry_of(uint32_t key, int number) { return ((unsigned long long)~key << 32) | (uint32_t)number; }
__device__ __forceinline__ float logit_of(unsigned long long entry) { return of_key(~(uint32_t)(entry >> 32)); }

// the border at a place of a sorted list that holds all its equals
template <int NT>
__device__ __forceinline__ Cut cut_at(const unsigned long long* list, int pos) {
    const unsigned long long last = list[pos];
    uint32_t ties = 0;
    for (int i = 0; i < kList; i += NT) {
        const int k = i + (int)threadIdx.x;
        ties += (uint32_t)__syncthreads_count(k <= pos && (uint32_t)(list[k] >> 32) == (uint32_t)(last >> 32));
    }
    return Cut{logit_of(last), ties, (int32_t)(uint32_t)last};
}

// Moves `cut` to where the prefix ends that `ends(running sum, sum of all kept)` says; `kMass`: sums of weights, else of tokens.
template <bool kMass, typename T, int NT, typename F>
__device__ __forceinline__ void select(const Column_<T, NT>& h, Parts& sp, float range, Cut& cut, F&& ends) {
    constexpr int V = Column_<T, NT>::V, PER = kBins / NT;
    Shared<NT>& sh = h.sh;
    const int tid = threadIdx.x;
    const float scale = range > 0.f ? (float)kBins / range : 0.f;      // (0 too for a range beyond fp32: one part)
    uint32_t lo = 0, hi = 0;                                            // the keys that are looked at, and how they are divided
    int bits = -1;                                                      // -1: by the logit
    const Cut old = cut;
    auto part_of = [&](float y, uint32_t key) -> int {
        if (bits < 0) return min(kBins - 1, (int)((h.top - y) * scale));
        return (int)((hi - key) >> bits);
    };
    // fn(logit, key, number) for what is looked at
    auto members = [&](auto&& fn) {
        h.template all_rows<1>([&](int f, const RawVec<T>& v) {
            const int n0 = h.number(f, 0);
#pragma unroll 1
            for (int j = 0; j < V; j++) {            // (rolled: the calls' bodies are long, and this is the rare way)
                const float y = h.clean(v, j);
                const uint32_t key = key_of(y);
                const bool kept = y > old.x || (y == old.x && n0 + j <= old.number);
                if (y > kNegInf && kept && (bits < 0 || (key >= lo && key <= hi))) fn(y, key, n0 + j);
            }
        });
    };
    uint64_t before = 0, all = 0;
    int n = 0, part = 0;
    for (int level = 0;; level++) {
        __syncthreads();
        for (int i = tid; i < kBins; i += NT) {
            sp.h.count[i] = 0;
            sp.h.mass[i] = 0;
        }
        __syncthreads();
        members([&](float y, uint32_t key, int) {
            const int b = part_of(y, key);
            atomicAdd(&sp.h.count[b], 1u);
            if (kMass) atomicAdd(&sp.h.mass[b], (unsigned long long)h.weight(y));
        });
        __syncthreads();
        auto v = [&](int i) -> uint64_t { return kMass ? sp.h.mass[tid * PER + i] : sp.h.count[tid * PER + i]; };
        if (level == 0) {
            find_end<NT, PER>(sh, 0, v, ends);
            all = sh.total;
        } else {
            find_end<NT, PER>(sh, before, v, [&](uint64_t s, uint64_t) { return ends(s, all); });
        }
        part = sh.pos;
        if (part < 0) return;                                           // the prefix is everything
        before = sh.before;
        n = (int)sp.h.count[part];
        if (n <= kList) break;
        // divide again: the keys of this part are a run of all keys
        __syncthreads();
        if (tid == 0) {
            sh.lo = 0xffffffffu;
            sh.hi = 0;
        }
        __syncthreads();
        uint32_t kl = 0xffffffffu, kh = 0;
        members([&](float y, uint32_t key, int) {
            if (part_of(y, key) != part) return;
            kl = min(kl, key);
            kh = max(kh, key);
        });
        if (kl <= kh) {
            atomicMin(&sh.lo, kl);
            atomicMax(&sh.hi, kh);
        }
        __syncthreads();
        lo = sh.lo;
        hi = sh.hi;
        if (lo == hi) {
            // equal logits: the first `c` of them (none of them has been cut off before, or those that were have the last numbers)
            const float x = of_key(lo);
            const uint64_t c = how_many(before, kMass ? h.weight(x) : 1, (uint64_t)n, all, ends);
            cut = Cut{x, (uint32_t)c, number_of_equal(h, x, c - 1)};
            return;
        }
        bits = max(0, 32 - __clz((int)(hi - lo)) - 11);                  // (2^11 parts)
    }
    // the part fits the list: sort it
    __syncthreads();
    if (tid == 0) sh.n = 0;
    __syncthreads();
    members([&](float y, uint32_t key, int number) {
        if (part_of(y, key) == part) sp.list[atomicAdd(&sh.n, 1)] = entry_of(key, number);
    });
    __syncthreads();
    sort_list<NT>(sp.list, n);
    auto v = [&](int i) -> uint64_t {
        const int k = tid * (kList / NT) + i;
        return k >= n ? 0 : kMass ? h.weight(logit_of(sp.list[k])) : 1;
    };
    find_end<NT, kList / NT>(sh, before, v, [&](uint64_t s, uint64_t) { return ends(s, all); });
    cut = cut_at<NT>(sp.list, max(0, sh.pos));
}

// top-k by the threads' largest logits (`mine`), k up to half their number; the k largest are left sorted in the list.  false: more than a list of candidates.
template <typename T, int NT>
__device__ __forceinline__ bool list_top_k(const Column_<T, NT>& h, Parts& sp, float mine, int k) {
    constexpr int V = Column_<T, NT>::V;
    Shared<NT>& sh = h.sh;
    // the k-th largest of NT numbers, to 16 of its key's bits (a lower one does as well)
    const uint32_t key = key_of(mine + 0.f);
    uint32_t least = 0;
    for (int bit = 31; bit >= 16; bit--) {
        const uint32_t t = least | (1u << bit);
        if (__syncthreads_count(key >= t) >= k) least = t;
    }
    const float bound = fmaxf(of_key(max(least, key_of(kNegInf))), -3.402823466e38f);
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    h.template all_rows<4>([&](int f, const RawVec<T>& v) {
        bool any = false;
#pragma unroll
        for (int j = 0; j < V; j++) any = any || h.value(v, j) >= bound;
        if (!any) return;
        const int n0 = h.number(f, 0);
#pragma unroll
        for (int j = 0; j < V; j++) {
            const float y = h.value(v, j) + 0.f;
            if (y >= bound) {
                const int at = atomicAdd(&sh.n, 1);
                if (at < kList) sp.list[at] = entry_of(key_of(y), n0 + j);
            }
        }
    });
    __syncthreads();
    const int n = sh.n;
    if (n > kList) return false;
    __syncthreads();
    sort_list<NT>(sp.list, n);
    sh.n = min(n, k);
    __syncthreads();
    return true;
}

// The draw from the first n of a sorted list (n <= kMostListed): each entry's place in the order of the numbers is the sum of the weights with numbers up to its own.
template <typename T, int NT>
__device__ __forceinline__ void draw_listed(const Column_<T, NT>& h, Parts& sp, int n, float u) {
    Shared<NT>& sh = h.sh;
    const float least = with_least(h.a, h.top, Cut{kNegInf, 0u, -1}).x;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) {
        const float x = logit_of(sp.list[i]);
        sp.weight[i] = x > least ? h.weight(x) : 0;
    }
    if (threadIdx.x == 0) sh.n = -1;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) {
        const uint32_t number = (uint32_t)sp.list[i];
        uint64_t all = 0, upto = 0;
        for (int k = 0; k < n; k++) {
            const uint64_t w = sp.weight[k];
            all += w;
            upto += (uint32_t)sp.list[k] <= number ? w : 0;
        }
        const uint64_t to = share_of(u, all);
        if (upto > to && upto - sp.weight[i] <= to) {
            sh.n = (int32_t)number;
            sh.x = logit_of(sp.list[i]);
        }
    }
    __syncthreads();
}

template <typename T, int NT>
__device__ __forceinline__ void any_column(const Sample& a, Column_<T, NT>& h, Parts& sp) {
    constexpr int V = RawVec<T>::V, NW = NT / 64;
    Shared<NT>& sh = h.sh;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    __syncthreads();                                  // the tiles' addresses
    // one read for the largest and smallest logit and, each thread shifted by what it has seen so far, the sum of all exponentials
    float mine = kNegInf, mn = kPosInf, shift = -3.402823466e38f;
    double sum = 0.0;
    h.template all_rows<4>([&](int, const RawVec<T>& v) {
        float y[V];
#pragma unroll
        for (int j = 0; j < V; j++) {
            y[j] = v.at(j);
            mine = fmaxf(mine, y[j]);
            mn = y[j] > kNegInf ? fminf(mn, y[j]) : mn;
        }
        if (a.logp) {
            float s = 0.f;
            const float next = fmaxf(shift, mine);
#pragma unroll
            for (int j = 0; j < V; j++) s += exp_of(fmaxf(y[j], kNegInf) - next);           // (fmaxf: no NaN)
            sum = fma(sum, (double)exp_of(shift - next), (double)s);
            shift = next;
        }
    });
    float mx = wave_max(mine);
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
        no_token(a);
        return;
    }
    h.set_top(mx);
    if (h.top_inf) {
        mn = 0.f;
        mine = mine == kPosInf ? 0.f : kNegInf;
    }
    if (a.logp) {
        if (h.top_inf) {
            sum = 0.0;
            h.template all_rows<1>([&](int, const RawVec<T>& v) {
#pragma unroll
                for (int j = 0; j < V; j++) sum += h.value(v, j) == 0.f ? 1.0 : 0.0;
            });
        } else {
            sum *= (double)exp_of(shift - h.top);
        }
        sum = wave_sum64(sum);
        if (lane == 0) sh.sum[w] = sum;
    }
    Cut cut{kNegInf, 0u, -1};
    bool drawn = false;
    const float range = h.top - mn, u = random_of(a);
    auto ends = [&](uint64_t s, uint64_t all) { return (double)s >= a.top_p * (double)all; };
    if (a.top_k > 0 && a.top_k < a.X.shape[0]) {
        if (a.top_k <= min(kMostListed, NT / 2) && list_top_k(h, sp, mine, a.top_k)) {
            int n = sh.n;
            if (a.top_p < 1.0) {
                const uint64_t mass = tid < n ? h.weight(logit_of(sp.list[tid])) : 0;
                find_end<NT, 1>(sh, 0, [&](int) { return mass; }, ends);
                if (sh.pos >= 0) n = sh.pos + 1;
            }
            draw_listed(h, sp, n, u);
            drawn = true;
        } else {
            select<false>(h, sp, range, cut, [&](uint64_t s, uint64_t) { return s >= (uint64_t)a.top_k; });
        }
    }
    if (!drawn && a.top_p < 1.0) select<true>(h, sp, range, cut, ends);
    if (!drawn) draw(h, with_least(a, h.top, cut), u);
    sum = 0.0;
    if (a.logp && tid == 0)
        for (int k = 0; k < NW; k++) sum += sh.sum[k];
    answer(a, sh, h.top, sum);
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT) sample_kernel(Sample a) {
    __shared__ Shared<NT> sh;
    __shared__ Parts parts;
    const int64_t col = a.columns ? a.columns[blockIdx.x] : (int)blockIdx.x;
    if (col < 0 || col >= a.ncols) {
        no_token(a);
        return;
    }
    Column_<T, NT> h(a, sh, col);
    any_column(a, h, parts);
}

// ---------------------------------------------------------------- the largest logit
// One read: each thread keeps its largest logit and the first vector that holds it, beside the sum of the exponentials (shifted by what it has seen so far).
// Bound by memory: 1024 bf16 columns of 50304 take 20 us (103 MB, 5.2 TB/s), where the draw's two reads took 61, one column 4.9 (12.5; one call after the other).
template <typename T, int NT>
__global__ void __launch_bounds__(NT) greedy_kernel(Sample a) {
    constexpr int V = RawVec<T>::V, NW = NT / 64;
    __shared__ Shared<NT> sh;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t col = a.columns ? a.columns[blockIdx.x] : (int)blockIdx.x;
    if (col < 0 || col >= a.ncols) {
        no_token(a);
        return;
    }
    Column_<T, NT> h(a, sh, col);
    if (tid == 0) sh.pos = INT32_MAX;
    __syncthreads();
    float mine = kNegInf, shift = -3.402823466e38f;
    int at = INT32_MAX;
    double sum = 0.0;
    h.template all_rows<4>([&](int f, const RawVec<T>& v) {
        float y[V], m = kNegInf;
#pragma unroll
        for (int j = 0; j < V; j++) {
            y[j] = v.at(j);
            m = fmaxf(m, y[j]);
        }
        at = m > mine ? f : at;
        mine = fmaxf(mine, m);
        if (a.logp) {
            float s = 0.f;
            const float next = fmaxf(shift, mine);
#pragma unroll
            for (int j = 0; j < V; j++) s += exp_of(fmaxf(y[j], kNegInf) - next);           // (fmaxf: no NaN)
            if (next > shift) sum *= (double)exp_of(shift - next);
            sum += (double)s;
            shift = next;
        }
    });
    float top = wave_max(mine);
    if (lane == 0) sh.mx[w] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NW; k++) top = fmaxf(top, sh.mx[k]);
    if (top == kNegInf) {
        no_token(a);
        return;
    }
    if (mine == top) atomicMin(&sh.pos, at);
    h.set_top(top);
    if (a.logp) {
        if (h.top_inf) {
            sum = 0.0;
            h.template all_rows<1>([&](int, const RawVec<T>& v) {
#pragma unroll
                for (int j = 0; j < V; j++) sum += h.value(v, j) == 0.f ? 1.0 : 0.0;
            });
        } else {
            sum *= (double)exp_of(shift - top);
        }
        sum = wave_sum64(sum);
        if (lane == 0) sh.sum[w] = sum;
    }
    __syncthreads();
    if (tid > 0) return;
    const RawVec<T> v = h.read(sh.pos, a.nvec);
    int first = V - 1;
#pragma unroll
    for (int j = V - 2; j >= 0; j--)
        if (v.at(j) == top) first = j;
    sh.n = h.number(sh.pos, first);
    sh.x = h.top;
    sum = 0.0;
    if (a.logp)
        for (int k = 0; k < NW; k++) sum += sh.sum[k];
    answer(a, sh, h.top, sum);
}

// ---------------------------------------------------------------- bf16 columns, counted
// A bf16 logit with 2^-12 <= |x| < 2^8 is one of 5120: its exponent and mantissa make a code, the sign doubles it.  The column is counted by code in
// LDS, so that weights, sums and borders are those of 5120 (value, count) pairs, in their order (positive codes falling, then negative ones
// rising), ten to a thread, and the draw looks weights up.  What has no code:
//   0 is counted by itself; smaller ones, few in logits of any spread, are kept in a list (more than it holds, or a border among them: any_column);
//   larger negative ones, -infinity and NaN weigh nothing next to a largest logit that has a code (unless T is large: any_column);
//   larger positive ones: any_column.
// Two workgroups of 512 share a unit, so that one counts while the other looks for borders.
constexpr uint32_t kFirst = 0x3980u, kSide = 2560u;      // bits of 2^-12, codes of one sign
constexpr int kCodes = 2 * (int)kSide;
constexpr int kSmall = 512;
constexpr uint32_t kNegCounts = 4096u;                   // a negative code's count lies here: a bit of its own, above a code that is none (kSide)
constexpr float kLeastCoded = 0.000244140625f;           // 2^-12
constexpr int kCodeThreads = 512, kPer = kCodes / kCodeThreads, kSlots = kPer + 3;
struct Codes {
    uint32_t count[kNegCounts + kSide + 1];
    unsigned long long weight[kCodes + 2];               // each sign's with a 0 behind them, for what has no code
    uint32_t small[kSmall];                              // bits
};
constexpr unsigned long long kOneTie = 1ull << 55;       // eight weights are at most 2^54
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float of_bits(uint32_t b) { return __uint_as_float(b << 16); }
// code of the bits b, if they have one
__device__ __forceinline__ uint32_t code_of(uint32_t b, bool& has) {
    const uint32_t u = (b & 0x7fffu) - kFirst;
    has = u < kSide;
    return u + (b >> 15) * kSide;
}
__device__ __forceinline__ float of_code(uint32_t k) { return k < kSide ? of_bits(k + kFirst) : of_bits(k - kSide + kFirst + 0x8000u); }

// The rare way, out of line: its registers are not the counted columns'.
template <int NT>
__device__ __attribute__((noinline)) void far_column(const Sample a, int64_t col, Shared<NT>& sh, Parts& parts) {
    Column_<bf16_t, NT> h(a, sh, col);
    any_column(a, h, parts);
}

// What is found about a column while it is counted.
struct CodedColumn {
    float top;
    uint32_t zeros, smalls, small_up, small_down;          // the last two: of this thread's entries of the list
};

// Weights, border and draw.  false: the border lies among the small ones.
__device__ __forceinline__ bool coded_column(const Sample& a, Column_<bf16_t, kCodeThreads>& h, Codes& m, const CodedColumn& k, uint32_t (&cnt)[kSlots],
                                             const float (&x)[kPer]) {
    constexpr int NT = kCodeThreads, V = 8, PER = kPer, SLOTS = kSlots;
    Shared<NT>& sh = h.sh;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const bool neg = tid >= NT / 2, middle = tid == NT / 2 - 1;
    const float top = k.top;
    const uint32_t zeros = k.zeros, smalls = k.smalls, small_up = k.small_up, small_down = k.small_down;
    h.set_top(top);
    // weights; sums of the small ones, which meet in the middle thread's slots
    uint64_t wt[SLOTS];
    double sum = 0.0;
    float part = 0.f;                                      // (ten terms; the threads' sums meet in 64 bits)
#pragma unroll
    for (int i = 0; i < PER; i++) {
        wt[i] = cnt[i] ? h.weight(x[i]) : 0;
        if (a.logp && cnt[i]) part += (float)cnt[i] * exp_of(x[i] - top);
    }
    sum = (double)part;
    wt[PER] = wt[PER + 1] = wt[PER + 2] = 0;
    if (middle && zeros) {
        cnt[PER + 1] = zeros;
        wt[PER + 1] = h.weight(0.f);
        sum += (double)zeros * exp_of(-top);
    }
    uint64_t mass_up = 0, mass_down = 0;                   // of all small ones (in the middle thread)
    if (smalls) {
        uint64_t up = 0, down = 0;
        for (uint32_t i = tid; i < smalls; i += NT) {
            const uint32_t b = m.small[i];
            const float y = of_bits(b);
            if (b < 0x8000u) up += h.weight(y);
            else down += h.weight(y);
            sum += exp_of(y - top);
        }
        up = wave_scan(up);
        down = wave_scan(down);
        const uint64_t both = wave_scan((uint64_t)small_up | (uint64_t)small_down << 32);
        __syncthreads();
        if (tid == 0) sh.before = sh.total = 0;
        if (tid == 0) sh.wave[0] = 0;
        __syncthreads();
        if (lane == 63) {
            atomicAdd(&sh.before, (unsigned long long)up);
            atomicAdd(&sh.total, (unsigned long long)down);
            atomicAdd(&sh.wave[0], (unsigned long long)both);
        }
        __syncthreads();
        if (middle) {
            cnt[PER] = (uint32_t)sh.wave[0];
            cnt[PER + 2] = (uint32_t)(sh.wave[0] >> 32);
            mass_up = sh.before;
            mass_down = sh.total;
        }
        __syncthreads();
    }
    if (a.logp) {
        sum = wave_sum64(sum);
        if (lane == 0) sh.sum[w] = sum;
    }
    Cut cut{kNegInf, 0u, -1};
    // the border at the place `pos` of the order, of which `c` stay; what is behind it counts no more.  false: among the small ones
    auto end_at = [&](int pos, uint64_t c) {
#pragma unroll
        for (int i = 0; i < SLOTS; i++) {
            if (tid * SLOTS + i == pos) {
                cnt[i] = (uint32_t)c;
                sh.x = i < PER ? x[i < PER ? i : 0] : i == PER + 1 ? 0.f : 1e30f;
            }
            if (tid * SLOTS + i > pos) cnt[i] = 0;
        }
        __syncthreads();
        cut = Cut{sh.x, (uint32_t)c, -1};
        return cut.x != 1e30f;
    };
    bool coded = true;
    if (a.top_k > 0 && a.top_k < a.X.shape[0]) {
        find_end<NT, SLOTS>(sh, 0, [&](int i) -> uint64_t { return cnt[i]; }, [&](uint64_t s, uint64_t) { return s >= (uint64_t)a.top_k; });
        if (sh.pos >= 0) coded = end_at(sh.pos, (uint64_t)a.top_k - sh.before);
        __syncthreads();
    }
    if (coded && a.top_p < 1.0) {
        auto ends = [&](uint64_t s, uint64_t all) { return (double)s >= a.top_p * (double)all; };
        // (the small ones' sums, not one weight of theirs)
        auto v = [&](int i) -> uint64_t { return i == PER ? (cnt[i] ? mass_up : 0) : i == PER + 2 ? (cnt[i] ? mass_down : 0) : (uint64_t)cnt[i] * wt[i]; };
        find_end<NT, SLOTS>(sh, 0, v, ends);
        const int pos = sh.pos;
        if (pos >= 0) {
            const uint64_t before = sh.before, all = sh.total;
#pragma unroll
            for (int i = 0; i < SLOTS; i++)
                if (tid * SLOTS + i == pos) {
                    // (how many are left of what top-k may have cut)
                    sh.lo = cnt[i];
                    sh.wave[0] = wt[i];
                }
            __syncthreads();
            const uint64_t left = sh.lo, one = sh.wave[0];
            __syncthreads();
            coded = end_at(pos, how_many(before, one, left, all, ends));
        }
        __syncthreads();
    }
    if (!coded) return false;
    cut = with_least(a, top, cut);
    // the table: what lies above the border, and at it (where ties stay) a one above the weights, which counts them as sums are taken
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const uint32_t k = neg ? kSide + (uint32_t)((tid - NT / 2) * PER + i) : kSide - 1 - (uint32_t)(tid * PER + i);
        m.weight[k + (neg ? 1 : 0)] = x[i] > cut.x ? wt[i] : cut.ties && x[i] == cut.x ? kOneTie : 0;
    }
    if (tid < 2) m.weight[tid ? kCodes + 1 : kSide] = 0;
    __syncthreads();
    const bool tied = cut.ties != 0, small_too = cut.x < kLeastCoded && (smalls || zeros);
    bool has;
    const uint32_t border = tied ? code_of(__float_as_uint(cut.x) >> 16, has) : 0xffffffffu;
    const float u = random_of(a);
    auto weigh = [&](const RawVec<bf16_t>& v, uint64_t (&p)[V]) {
        uint32_t equal = 0;
        bool odd = false;
#pragma unroll
        for (int j = 0; j < V; j++) {
            const uint32_t b = (j & 1) ? v.x[j >> 1] >> 16 : v.x[j >> 1] & 0xffffu;
            bool coded;
            const uint32_t k = code_of(b, coded);
            p[j] = m.weight[coded ? k + (b >> 15) : kSide] & (kOneTie - 1);
            equal |= coded && k == border ? 1u << j : 0u;
            odd = odd || !coded;
        }
        if (small_too && __any(odd)) {
            equal = 0;
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float y = v.at(j);
                if (fabsf(y) < kLeastCoded) p[j] = y > cut.x ? h.weight(y) : 0;
                equal |= tied && y == cut.x ? 1u << j : 0u;
            }
        }
        return equal;
    };
    auto goal = [&](uint64_t all) { return share_of(u, all); };
    const uint64_t tie = tied ? h.weight(cut.x) : 0;
    if (cut.x >= kLeastCoded) {
        // The border has a positive code: kept are the bits from it to the largest logit's, all others go by the place behind those, whose weight is 0 (no logit
        // has that code).  Two logits of a word at a time, and the look-ups of a vector are on their way together
        // (one by one, where kept, 75 us for 1024 columns of 50304, so 67; the same below, all kept, 77 and 73).
        const uint32_t lowest = __float_as_uint(cut.x) >> 16, behind = (__float_as_uint(top) >> 16) - lowest + 1;
        const u16x2 low = {(uint16_t)lowest, (uint16_t)lowest}, most = {(uint16_t)behind, (uint16_t)behind};
        const char* table = reinterpret_cast<const char*>(m.weight + (lowest - kFirst));
        locate_by<4>(h, tie, cut.ties,
               [&](const RawVec<bf16_t>& v, uint64_t& s, uint32_t& ties) {
                   uint64_t sum8 = 0;
#pragma unroll
                   for (int k = 0; k < V / 2; k++) {
                       const u16x2 t = __builtin_elementwise_min((u16x2)(__builtin_bit_cast(u16x2, (uint32_t)v.x[k]) - low), most);
                       const uint32_t at = __builtin_bit_cast(uint32_t, (u16x2)(t << (uint16_t)3));
                       sum8 += *reinterpret_cast<const unsigned long long*>(table + (at & 0xffffu));
                       sum8 += *reinterpret_cast<const unsigned long long*>(table + (at >> 16));
                   }
                   s += sum8 & (kOneTie - 1);
                   ties += (uint32_t)(sum8 / kOneTie);
               },
               weigh, goal);
    } else {
        const u16x2 first = {(uint16_t)kFirst, (uint16_t)kFirst}, side = {(uint16_t)kSide, (uint16_t)kSide};
        locate_by<4>(h, tie, cut.ties,
               [&](const RawVec<bf16_t>& v, uint64_t& s, uint32_t& ties) {
                   uint32_t at[V / 2];
                   u16x2 largest = {0, 0};
#pragma unroll
                   for (int k = 0; k < V / 2; k++) {
                       const u16x2 mag = __builtin_elementwise_min((u16x2)(__builtin_bit_cast(u16x2, (uint32_t)v.x[k] & 0x7fff7fffu) - first), side);
                       const u16x2 sign = __builtin_bit_cast(u16x2, ((uint32_t)v.x[k] >> 15) & 0x00010001u);
                       largest = __builtin_elementwise_max(largest, mag);
                       at[k] = __builtin_bit_cast(uint32_t, (u16x2)((u16x2)(mag + sign * (u16x2)(side + (uint16_t)1)) << (uint16_t)3));
                   }
                   if (small_too && __any(largest[0] >= kSide || largest[1] >= kSide)) {
                       uint64_t p[V];
                       ties += __popc(weigh(v, p));
#pragma unroll
                       for (int j = 0; j < V; j++) s += p[j];
                       return;
                   }
                   uint64_t sum8 = 0;
#pragma unroll
                   for (int k = 0; k < V / 2; k++) {
                       sum8 += *reinterpret_cast<const unsigned long long*>(reinterpret_cast<const char*>(m.weight) + (at[k] & 0xffffu));
                       sum8 += *reinterpret_cast<const unsigned long long*>(reinterpret_cast<const char*>(m.weight) + (at[k] >> 16));
                   }
                   s += sum8 & (kOneTie - 1);
                   ties += (uint32_t)(sum8 / kOneTie);
               },
               weigh, goal);
    }
    sum = 0.0;
    if (a.logp && tid == 0)
        for (int k = 0; k < NT / 64; k++) sum += sh.sum[k];
    answer(a, sh, top, sum);
    return true;
}

__global__ void __launch_bounds__(512, 4) sample_codes_kernel(Sample a) {
    constexpr int NT = kCodeThreads, V = 8, PER = kPer, SLOTS = kSlots;
    __shared__ Shared<NT> sh;
    __shared__ union {
        Codes c;
        Parts parts;
    } m;
    __shared__ uint32_t n_zero, n_small, n_large;
    __shared__ int least_large;                           // (as an order of whole numbers: the largest of the large negative ones)
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t col = a.columns ? a.columns[blockIdx.x] : (int)blockIdx.x;
    if (col < 0 || col >= a.ncols) {
        no_token(a);
        return;
    }
    Column_<bf16_t, NT> h(a, sh, col);
    for (int i = tid; i < (int)kSide / 4; i += NT) {
        reinterpret_cast<uint4*>(m.c.count)[i] = make_uint4(0u, 0u, 0u, 0u);
        reinterpret_cast<uint4*>(m.c.count + kNegCounts)[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    if (tid == 0) n_zero = n_small = n_large = 0;
    if (tid == 0) least_large = 0;
    __syncthreads();
    h.all_rows<4>([&](int, const RawVec<bf16_t>& v) {
        // two logits of a word at a time: what has no code counts in a place that nobody reads
        u16x2 most = {0, 0};
        uint32_t magnitude[V / 2];
#pragma unroll
        for (int k = 0; k < V / 2; k++) {
            const u16x2 u = __builtin_bit_cast(u16x2, v.x[k] & 0x7fff7fffu) - u16x2{(uint16_t)kFirst, (uint16_t)kFirst};
            const u16x2 code = __builtin_elementwise_min(u, u16x2{(uint16_t)kSide, (uint16_t)kSide});
            most = __builtin_elementwise_max(most, code);
            magnitude[k] = __builtin_bit_cast(uint32_t, code);
            const uint32_t at = ((v.x[k] >> 3) & 0x10001000u) | magnitude[k];
            atomicAdd(&m.c.count[at & 0xffffu], 1u);
            atomicAdd(&m.c.count[at >> 16], 1u);
        }
        if (most[0] < kSide && most[1] < kSide) return;
        uint32_t odd = 0;
#pragma unroll
        for (int j = 0; j < V; j++)
            odd |= ((j & 1) ? magnitude[j >> 1] >> 16 : magnitude[j >> 1] & 0xffffu) >= kSide ? 1u << j : 0u;
        while (odd) {
            const int j = __ffs((int)odd) - 1;
            odd &= odd - 1;
            uint32_t word = v.x[0];
            if ((j >> 1) == 1) word = v.x[1];
            if ((j >> 1) == 2) word = v.x[2];
            if ((j >> 1) == 3) word = v.x[3];
            const uint32_t b = (word >> (16 * (j & 1))) & 0xffffu, mag = b & 0x7fffu;
            if (mag == 0) {
                atomicAdd(&n_zero, 1u);
            } else if (mag < kFirst) {
                const uint32_t at = atomicAdd(&n_small, 1u);
                if (at < (uint32_t)kSmall) m.c.small[at] = b;
            } else if (mag <= 0x7f80u && b < 0x8000u) {
                n_large = 1u;
            } else if (mag < 0x7f80u) {
                atomicMin(&least_large, -(int)(0x8000u - mag));        // the smallest magnitude
            }
        }
    });
    __syncthreads();
    const uint32_t zeros = n_zero, smalls = n_small;
    // a thread's slots, falling: its codes, and behind the smallest positive ones (thread NT / 2 - 1) the small positive ones, 0 and the small negative ones
    const bool neg = tid >= NT / 2, middle = tid == NT / 2 - 1;
    uint32_t cnt[SLOTS];
    float x[PER];
    float mine = kNegInf;
#pragma unroll
    for (int i = PER - 1; i >= 0; i--) {
        const uint32_t k = neg ? kSide + (uint32_t)((tid - NT / 2) * PER + i) : kSide - 1 - (uint32_t)(tid * PER + i);
        cnt[i] = m.c.count[neg ? k + (kNegCounts - kSide) : k];
        x[i] = of_code(k);
        if (cnt[i]) mine = x[i];
    }
    cnt[PER] = cnt[PER + 1] = cnt[PER + 2] = 0;
    if (zeros && tid == 0) mine = fmaxf(mine, 0.f);
    uint32_t small_up = 0, small_down = 0;                 // of this thread's entries of the list
    bool plain = n_large == 0 && smalls <= (uint32_t)kSmall;
    if (plain && smalls) {
        for (uint32_t i = tid; i < smalls; i += NT) {
            const uint32_t b = m.c.small[i];
            mine = fmaxf(mine, of_bits(b));
            if (b < 0x8000u) small_up++;
            else small_down++;
        }
    }
    float top = wave_max(mine);
    if (lane == 0) sh.mx[w] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NT / 64; k++) top = fmaxf(top, sh.mx[k]);
    // the large negative ones: at least 256 below 0, and weighing less than 2^-60 of the largest
    if (least_large != 0) {
        const double fall = (double)of_bits(0x8000u | (uint32_t)(0x8000 + least_large)) - (double)top;
        plain = plain && fall * a.c < -60.0 && fall * kLog2e < -60.0;
    }
    if (plain && top > kNegInf && coded_column(a, h, m.c, CodedColumn{top, zeros, smalls, small_up, small_down}, cnt, x)) return;
    far_column<NT>(a, col, sh, m.parts);                   // (nothing but -infinity and NaN: said there)
}

int32_t launched() { return hipGetLastError() == hipSuccess ? (int32_t)NNT_OK : (int32_t)NNT_EHIP; }

#define TRY(x)                           \
    do {                                 \
        int32_t rc__ = (x);              \
        if (rc__ != NNT_OK) return rc__; \
    } while (0)

using SampleFn = void (*)(Sample);
SampleFn sample_instance(int dtype, int64_t nvec, bool greedy, int* nt) {
    *nt = nvec <= 1024 ? 256 : dtype == NNT_F32 ? 1024 : 512;
    if (greedy) {
        if (dtype == NNT_F32) return *nt == 256 ? greedy_kernel<float, 256> : greedy_kernel<float, 1024>;
        return *nt == 256 ? greedy_kernel<bf16_t, 256> : greedy_kernel<bf16_t, 512>;
    }
    if (dtype == NNT_F32) return *nt == 256 ? sample_kernel<float, 256> : sample_kernel<float, 1024>;
    return *nt == 256 ? sample_kernel<bf16_t, 256> : sample_codes_kernel;
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
    const bool greedy = cfg->temperature == 0.0;
    a.c = std::min(kLog2e / cfg->temperature, 1e200);
    a.top_p = cfg->top_p;
    a.min_fall = cfg->min_p == 0.0 ? -__builtin_huge_val() : cfg->temperature * std::log(cfg->min_p);
    // the sum of a column's weights, 1 at most each, stays below 2^62
    int log_n = 0;
    while (((int64_t)1 << log_n) < X->shape[0]) log_n++;
    a.shift = std::min(51, 62 - log_n);
    int nt;
    const SampleFn fn = sample_instance(X->dtype, nvec, greedy, &nt);
    std::vector<Access> acc;
    if (after) acc.push_back(after->whole_access(kReadWrite));
    acc.push_back(X->all(kRead));
    OpTag tag(ctx, "sample_tokens", (double)X->shape[0] * n * X->elem_size(), true);
    return submit(ctx, acc, [=](hipStream_t st) {
        hipLaunchKernelGGL(fn, dim3((unsigned)n), dim3((unsigned)nt), 0, st, a);
        return launched();
    });
}

}  // namespace nnt

using namespace nnt;

int32_t nnt_sample_tokens(nnt_ctx* ctx, const nnt_sample_cfg* cfg, nnt_tensor* X, const int32_t* columns, int32_t n, const float* uniforms,
                          int32_t* tokens, float* logp) {
    return entry(ctx, [&]() -> int32_t { return sample_ordered(ctx, cfg, X, columns, n, uniforms, tokens, logp, nullptr); });
}
