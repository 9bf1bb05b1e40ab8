// Draws from rows of candidates by given random numbers
// (include/gs_budget.h): temperature, top-k, top-p, min-p, then the inverse of
// the distribution function.
//
// A candidate's mass is a whole number, so every sum is exact, however it is
// cut over lanes and workgroups: counts and masses go through integer atomics
// and scans in any order, and a draw is the same on every path. What the
// filters keep is given by a key and a number of equals: all candidates of a
// larger key, and the first `ties` of that key by index. The key is found by
// digits, not by a sort: the top_k-th largest by counts, and the one at which
// the mass before a candidate passes top_p's share by masses.
//
// A row that fits the registers and LDS of a workgroup is one launch: keys and
// masses stay in registers, the running mass goes to LDS, where the draws
// search it. Longer rows are cut into stretches over many workgroups. Where
// few candidates stay, every workgroup lists its stretch's best, and the lists
// are drawn from like a short row; otherwise every pass is a launch, and the
// running mass goes to the workspace. Bound by chains of steps with a barrier or
// a launch each, not by the scores' bytes: 64 rows of 50021 bfloat16 logits,
// top-k 200 and top-p, 24 us (the lists 14.5, the draws 9.9); 419430 draws from 2
// M candidates, top-p, 63 us (four passes over the scores 5 to 12 each, running
// masses 9, the draws' random reads 22).
// A short row, and one drawn from lists, has one workgroup for all of its draws:
// 10^5 and 10^6 draws from 4096 candidates 298 us and 3.5 ms, 10^6 from 16384 1.5
// ms.

#include <type_traits>

#include "budget.h"

namespace gs {
namespace {

size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }

// How a row's scores become masses; by the settings alone.
enum { kRatio = 0, kPower = 1, kExp = 2, kBest = 3 };

struct DrawArgs {
    const void *scores;
    int64_t rows, n, stride, draws;
    const int32_t *lengths;
    const double *uniform;
    int32_t *ids;
    float *prob;
    double rate;      // kPower: 1 / T, kExp: log2(e) / T
    double least;     // min_p 2^k
    uint64_t share;   // floor(top_p 2^53)
    uint32_t top_k;   // 2^32 - 1: off
    uint32_t top_p;   // whether top_p is on
    uint32_t bf16, form;
    uint32_t flip;    // logits: all ones, weights: 0
    float floor;      // scores are drawn above it: -infinity, 0
    int32_t bits;     // k
};

// A score's place in the order as an unsigned number; 0: never drawn. (Without
// a branch: floor and flip stand for the form of the scores.)
__device__ __forceinline__ uint32_t key_of(const DrawArgs &a, uint32_t b) {
    const float x = __uint_as_float(b);
    const uint32_t c = __float_as_uint(x + 0.0f);  // -0 as 0
    const uint32_t k = c ^ (((uint32_t)((int32_t)c >> 31) | 0x80000000u) & a.flip);
    return x > a.floor ? k : 0u;
}
__device__ __forceinline__ uint32_t score_key(const DrawArgs &a, int64_t at) {
    return key_of(a, a.bf16 ? (uint32_t)((const uint16_t *)a.scores)[at] << 16 : ((const uint32_t *)a.scores)[at]);
}
__device__ __forceinline__ double key_score(const DrawArgs &a, uint32_t key) {
    return (double)__uint_as_float(key ^ (((uint32_t)((int32_t)~key >> 31) | 0x80000000u) & a.flip));
}

// Keys of U quads of a row, `apart` candidates from each other, the first at j:
// 0 from `end` on (a multiple of 4, or the row's length). No load depends on
// another's branch: a quad that passes the row's end is read from its last four
// candidates and moved down, one past `end` is read from there too, for
// nothing.
template <int U>
__device__ __forceinline__ void load_quads(const DrawArgs &a, int64_t row, uint32_t j, uint32_t apart, uint32_t end,
                                           uint32_t len, uint32_t k[U][4]) {
    typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
    const int64_t base = row * a.stride;
    if (len < 4) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (uint32_t t = 0; t < 4; ++t)
                k[u][t] = j + u * apart + t < end ? score_key(a, base + j + u * apart + t) : 0u;
        return;
    }
    uint32_t at[U], down[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t q = j + u * apart, last = len - 4;
        at[u] = q < last ? q : last;
        down[u] = q < end ? q - at[u] : 4u;
    }
    if (a.bf16) {
        u2 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = *(const u2 *)((const uint16_t *)a.scores + base + at[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            k[u][0] = v[u].x << 16;
            k[u][1] = v[u].x & 0xFFFF0000u;
            k[u][2] = v[u].y << 16;
            k[u][3] = v[u].y & 0xFFFF0000u;
        }
    } else {
        u4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = *(const u4 *)((const uint32_t *)a.scores + base + at[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            k[u][0] = v[u].x;
            k[u][1] = v[u].y;
            k[u][2] = v[u].z;
            k[u][3] = v[u].w;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int t = 0; t < 4; ++t) k[u][t] = key_of(a, k[u][t]);
        const uint32_t d = down[u], k1 = k[u][1], k2 = k[u][2], k3 = k[u][3];
        k[u][0] = d == 0 ? k[u][0] : d == 1 ? k1 : d == 2 ? k2 : d == 3 ? k3 : 0u;
        k[u][1] = d == 0 ? k1 : d == 1 ? k2 : d == 2 ? k3 : 0u;
        k[u][2] = d == 0 ? k2 : d == 1 ? k3 : 0u;
        k[u][3] = d == 0 ? k3 : 0u;
    }
}
__device__ __forceinline__ void load_keys(const DrawArgs &a, int64_t row, uint32_t j, uint32_t end, uint32_t len,
                                          uint32_t k[4]) {
    uint32_t q[1][4];
    load_quads<1>(a, row, j, 0, end, len, q);
#pragma unroll
    for (int t = 0; t < 4; ++t) k[t] = q[0][t];
}

// log2 of a positive float, in float64: with x = 2^e m, m in [sqrt(1/2),
// sqrt(2)), and r = (m - 1) / (m + 1), |r| < 0.172: e + 2 / ln 2 (r + r^3 / 3 +
// ... + r^21 / 21); the next term is below 2^-56 of the sum.
__device__ __forceinline__ double log2_of(double x) {
    int e = __builtin_amdgcn_frexp_exp(x);
    double m = __builtin_amdgcn_frexp_mant(x);  // [1/2, 1)
    if (m < 0.70710678118654752) {
        m += m;
        --e;
    }
    const double r = (m - 1.0) / (m + 1.0), s = r * r;
    double p = 1.0 / 21.0;
#pragma unroll
    for (int i = 19; i >= 1; i -= 2) p = __builtin_fma(p, s, 1.0 / i);
    return __builtin_fma(r * p, 2.8853900817779268, (double)e);
}

// 2^z in float64, z <= 0: 2^n times the series of e^(f ln 2) with f = z - n,
// |f| <= 1/2, up to the 13th power; the next term is below 2^-56.
__device__ __forceinline__ double exp2_of(double z, int more) {
    constexpr double inv[14] = {1.0,         1.0,          1.0 / 2,       1.0 / 6,        1.0 / 24,
                                1.0 / 120,   1.0 / 720,    1.0 / 5040,    1.0 / 40320,    1.0 / 362880,
                                1.0 / 3628800, 1.0 / 39916800, 1.0 / 479001600, 1.0 / 6227020800.0};
    z = z > -1100.0 ? z : -1100.0;
    const double n = rint(z), y = (z - n) * 0.69314718055994531;
    double p = inv[13];
#pragma unroll
    for (int i = 12; i >= 0; --i) p = __builtin_fma(p, y, inv[i]);
    return __builtin_amdgcn_ldexp(p, (int)n + more);
}

// What turns a row's keys into masses, given its largest key. (No library call
// a candidate, and no division but the logarithm's: they cost more than the
// candidate itself.)
struct Scale {
    uint32_t top;
    double at;  // kRatio: 2^k / max, kPower: log2 max, kExp: max
    bool best;  // the best alone has mass
};
__device__ __forceinline__ Scale scale_of(const DrawArgs &a, uint32_t top) {
    Scale s{top, 0.0, a.form == kBest};
    if (top == 0 || s.best) return s;
    const double m = key_score(a, top);
    s.best = m == __builtin_inf();
    if (s.best) return s;
    s.at = a.form == kRatio ? (double)((uint64_t)1 << a.bits) / m : a.form == kPower ? log2_of(m) : m;
    return s;
}

// q of N candidates, side by side: the chains of float64 operations are long.
// Adding 2^52 to a number from 0 to 2^52 rounds it to a whole one, which the
// sum's bits then count.
template <int N>
__device__ __forceinline__ void masses_of(const DrawArgs &a, const uint32_t key[N], const Scale &s, uint64_t q[N]) {
    double v[N];
#pragma unroll
    for (int t = 0; t < N; ++t) v[t] = 0.0;
    if (!s.best) {
        double x[N];
#pragma unroll
        for (int t = 0; t < N; ++t) x[t] = key_score(a, key[t] ? key[t] : s.top);
        if (a.form == kRatio) {
#pragma unroll
            for (int t = 0; t < N; ++t) v[t] = x[t] * s.at;
        } else {
            if (a.form == kPower) {
#pragma unroll
                for (int t = 0; t < N; ++t) x[t] = log2_of(x[t]);
            }
#pragma unroll
            for (int t = 0; t < N; ++t) v[t] = exp2_of((x[t] - s.at) * a.rate, a.bits);
        }
    }
#pragma unroll
    for (int t = 0; t < N; ++t) {
        const uint64_t r = __builtin_bit_cast(uint64_t, v[t] + 0x1p52) - __builtin_bit_cast(uint64_t, 0x1p52);
        q[t] = key[t] == 0 ? 0 : key[t] == s.top ? (uint64_t)1 << a.bits : r;
    }
}
__device__ __forceinline__ uint64_t mass_of(const DrawArgs &a, uint32_t key, const Scale &s) {
    uint64_t q;
    masses_of<1>(a, &key, s, &q);
    return q;
}

// floor(m total / 2^53), m <= 2^53, total < 2^63
__device__ __forceinline__ uint64_t share_of(uint64_t m, uint64_t total) {
    const uint64_t lo = m * total, hi = __umul64hi(m, total);
    return hi << 11 | lo >> 53;
}
__device__ __forceinline__ uint64_t uniform_bits(double u) {
    // a NaN takes the first branch
    if (!(u > 0.0)) return 0;
    return u < 1.0 ? (uint64_t)(u * 0x1p53) : ((uint64_t)1 << 53) - 1;
}

// What the filters keep of a row: larger keys, and `ties` of this key.
struct Kept {
    uint32_t key, ties;
};

// Candidates of a thread that can be drawn.
template <int ITEMS>
__device__ __forceinline__ uint32_t live(const uint32_t key[ITEMS]) {
    uint32_t n = 0;
#pragma unroll
    for (int t = 0; t < ITEMS; ++t) n += key[t] ? 1u : 0u;
    return n;
}

__device__ __forceinline__ uint32_t row_length(const DrawArgs &a, int64_t row) {
    if (!a.lengths) return (uint32_t)a.n;
    const int32_t l = a.lengths[row];
    return l < 0 ? 0u : l > a.n ? (uint32_t)a.n : (uint32_t)l;
}

__device__ __forceinline__ void write_draw(const DrawArgs &a, int64_t at, int64_t id, uint64_t q, uint64_t total) {
    a.ids[at] = (int32_t)id;
    if (a.prob) a.prob[at] = id >= 0 ? (float)((double)q / (double)total) : 0.0f;
}

// ---- sums over waves and workgroups --------------------------------------

template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp_u64(uint64_t x) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xF, false);
    return (uint64_t)hi << 32 | lo;
}
// Inclusive sums over the wave, every lane active (the steps of wave_incl_sum).
__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {
    x += dpp_u64<0x111, 0xF>(x);
    x += dpp_u64<0x112, 0xF>(x);
    x += dpp_u64<0x114, 0xF>(x);
    x += dpp_u64<0x118, 0xF>(x);
    x += dpp_u64<0x142, 0xA>(x);
    x += dpp_u64<0x143, 0xC>(x);
    return x;
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) { return wave_incl_sum(x); }
// The same over the first 16 lanes.
__device__ __forceinline__ uint64_t row_scan(uint64_t x) {
    x += dpp_u64<0x111, 0xF>(x);
    x += dpp_u64<0x112, 0xF>(x);
    x += dpp_u64<0x114, 0xF>(x);
    x += dpp_u64<0x118, 0xF>(x);
    return x;
}
__device__ __forceinline__ uint32_t row_scan(uint32_t x) { return wave_incl_sum(x); }
__device__ __forceinline__ uint64_t lane_of(uint64_t x, uint32_t lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(x >> 32), lane) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((uint32_t)x, lane);
}
__device__ __forceinline__ uint32_t lane_of(uint32_t x, uint32_t lane) { return __builtin_amdgcn_readlane(x, lane); }

// Exclusive sums over a workgroup of NT threads; *total gets the sum. lds: NT /
// kWave entries, free again after a barrier.
template <int NT, typename V>
__device__ __forceinline__ V group_scan(V x, uint64_t *lds, V *total) {
    const V incl = wave_scan(x);
    if (NT == kWave) {
        *total = lane_of(incl, kWave - 1);
        return incl - x;
    }
    // the waves' sums, a lane each (16 loads and sums of every thread take 30
    // registers: 300 rows of 16000, top-k 50, 43 us instead of 37)
    constexpr uint32_t kWaves = NT / kWave;
    static_assert(kWaves <= 16, "the waves' sums are a row of lanes");
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    __syncthreads();
    if (lane == kWave - 1) lds[wave] = incl;
    __syncthreads();
    const V upto = row_scan(lane < kWaves ? (V)lds[lane] : (V)0);
    *total = lane_of(upto, kWaves - 1);
    return (wave ? lane_of(upto, wave - 1) : (V)0) + incl - x;
}
template <int NT, typename V>
__device__ __forceinline__ V group_sum(V x, uint64_t *lds) {
    V total;
    group_scan<NT>(x, lds, &total);
    return total;
}
template <int NT>
__device__ __forceinline__ uint32_t group_max(uint32_t x, uint64_t *lds) {
    x = wave_max_uniform(x);
    if (NT == kWave) return x;
    __syncthreads();
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = x;
    __syncthreads();
    return wave_max_uniform(threadIdx.x % kWave < NT / kWave ? (uint32_t)lds[threadIdx.x % kWave] : 0u);
}

// ---- rows of a workgroup --------------------------------------------------

// The key that a filter ends at is found by digits of 8 bits of key - least,
// least the row's smallest key: subtracting it leaves as many digits as the
// row's scores spread over, and spreads the first of them over its bins.
// (Trying the key's bits one by one takes a sum over the workgroup for each:
// rows of 512, 41 us for 4096 of them.)
constexpr uint32_t kSmallBins = 256;

// The bin from the top in which the running sum passes `most` (above <= most <
// above + c), and the sum above it; bin 0 and all of the sum if none does.
// hist: LDS; out: LDS, 2 entries. By the first wave; ends with a barrier.
template <int NT>
__device__ __forceinline__ uint32_t pass_bin(const unsigned long long *hist, uint64_t most, uint64_t *above_bin,
                                             uint64_t *out) {
    __syncthreads();
    if (threadIdx.x < kWave) {
        constexpr uint32_t kMine = kSmallBins / kWave;
        const uint32_t top = kSmallBins - 1 - threadIdx.x * kMine;
        uint64_t c[kMine], sum = 0;
#pragma unroll
        for (uint32_t j = 0; j < kMine; ++j) sum += c[j] = hist[top - j];
        const uint64_t incl = wave_scan(sum);
        uint64_t above = incl - sum;
        const bool here = above <= most && most < incl;
        if (here) {
            uint32_t bin = 0;
            uint64_t at = 0;
#pragma unroll
            for (uint32_t j = 0; j < kMine; ++j) {
                if (above <= most && most < above + c[j]) {
                    bin = top - j;
                    at = above;
                }
                above += c[j];
            }
            out[0] = bin;
            out[1] = at;
        }
        if (__ballot(here) == 0 && threadIdx.x == kWave - 1) {
            out[0] = 0;
            out[1] = incl;
        }
    }
    __syncthreads();
    *above_bin = out[1];
    return (uint32_t)out[0];
}

// The digits of a workgroup's keys: of key - least, moved up so that the spread
// fills 32 bits and the first digit its bins (few of them would be met by most
// candidates, which wait for each other there). Keys below `least` have none.
struct Digits {
    uint32_t least;
    int lift;
    // whether the digit at `shift` tells anything
    __device__ __forceinline__ bool more(int shift) const { return shift + 8 > lift; }
    // whether the digits above `shift` of a candidate's offset are those of z
    __device__ __forceinline__ bool reach(uint32_t k, uint32_t z, int shift) const {
        return k >= least && (shift >= 24 || ((k - least) << lift >> (shift + 8)) == z);
    }
    __device__ __forceinline__ uint32_t at(uint32_t k, int shift) const { return (k - least) << lift >> shift & 255u; }
    // the key of the digits z down to the one at `shift`
    __device__ __forceinline__ uint32_t key(uint32_t z, int shift) const { return least + (z << shift >> lift); }
};
__device__ __forceinline__ Digits digits_of(uint32_t top, uint32_t least) {
    const uint32_t spread = top > least ? top - least : 0u;
    return Digits{least, __builtin_clz(spread | 1u)};
}

// A key that at least `want` <= NT candidates of a workgroup reach, given each
// thread's largest: want / waves of a wave's lanes reach what its top 16 bits
// are found to be, bit by bit, and every wave that of the least one.
template <int NT>
__device__ __forceinline__ uint32_t reached_by(uint32_t mine, uint32_t want, uint64_t *lds) {
    const uint32_t share = (want + NT / kWave - 1) / (NT / kWave);
    uint32_t t = 0;
    for (uint32_t bit = 1u << 31; bit >= 1u << 16; bit >>= 1)
        if ((uint32_t)__popcll(__ballot(mine >= (t | bit))) >= share) t |= bit;
    return ~group_max<NT>(~t, lds);
}

// The first top_k of a workgroup's candidates; all of them if they are no more.
// top, least: the keys' largest and least; mine: the thread's largest. (Where
// top_k <= NT, the few candidates that can be among them are found first:
// scores have few exponents, and adds of all of them to the first digit's bins
// wait for each other: stretches of 16384 logits, 200 to be kept, 19 -> 14 us.)
template <int NT, int ITEMS>
__device__ __forceinline__ Kept top_kept(const uint32_t key[ITEMS], uint32_t mine, uint32_t top_k, uint32_t top,
                                         uint32_t least, unsigned long long *s_hist, uint64_t *lds, uint64_t *s_out) {
    if (group_sum<NT>(live<ITEMS>(key), lds) <= top_k) return Kept{0, 0xFFFFFFFFu};
    if (top_k <= NT) least = umax_(least, reached_by<NT>(mine, top_k, lds));
    const Digits dg = digits_of(top, least);
    uint64_t need = top_k;
    uint32_t z = 0;
    int shift = 24;
    for (; dg.more(shift); shift -= 8) {
        __syncthreads();
        for (uint32_t b = threadIdx.x; b < kSmallBins; b += NT) s_hist[b] = 0;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < ITEMS; ++t)
            if (dg.reach(key[t], z, shift)) atomicAdd((uint32_t *)&s_hist[dg.at(key[t], shift)], 1u);
        uint64_t above;
        z = z << 8 | pass_bin<NT>(s_hist, need - 1, &above, s_out);
        need -= above;
    }
    return Kept{dg.key(z, shift + 8), (uint32_t)need};
}

// The places of a workgroup's kept candidates in their order: put(t, place) for
// each of them. Returns how many.
template <int NT, int ITEMS, typename F>
__device__ __forceinline__ uint32_t place_kept(const uint32_t key[ITEMS], const Kept &kept, uint64_t *lds, F put) {
    uint32_t mine = 0, total;  // larger: low half, equal: high half
#pragma unroll
    for (int t = 0; t < ITEMS; ++t)
        mine += key[t] > kept.key ? 1u : key[t] && key[t] == kept.key ? 0x10000u : 0u;
    uint32_t run = group_scan<NT>(mine, lds, &total);
#pragma unroll
    for (int t = 0; t < ITEMS; ++t) {
        const bool up = key[t] > kept.key, tie = key[t] && key[t] == kept.key;
        const uint32_t equals = run >> 16, place = (run & 0xFFFFu) + (equals < kept.ties ? equals : kept.ties);
        if (up || (tie && equals < kept.ties)) put(t, place);
        run += up ? 1u : tie ? 0x10000u : 0u;
    }
    const uint32_t ties = total >> 16;
    return (total & 0xFFFFu) + (ties < kept.ties ? ties : kept.ties);
}

// Lists of candidates that stand for the rows: keys (0: none) and numbers.
struct Lists {
    uint32_t *key, *id;  // [rows][stride]
    uint32_t stride, stretches, want;  // want: entries of a stretch's list
};

// Draws from a row whose candidates the threads of a workgroup hold, in order,
// after top-k has kept `kept` of them; id(j): the j-th candidate's number. s_run:
// LDS, NT (ITEMS + 1) entries.
template <int NT, int ITEMS, typename F>
__device__ __forceinline__ void draw_from(const DrawArgs &a, int64_t row, const uint32_t key[ITEMS], Kept kept,
                                          uint32_t top, uint32_t least, uint64_t *s_run, unsigned long long *s_hist,
                                          uint64_t *lds, uint64_t *s_out, F id) {
    uint64_t q[ITEMS];
    const Scale scale = scale_of(a, top);
    constexpr int kSide = ITEMS < 4 ? ITEMS : 4;
#pragma unroll
    for (int t = 0; t < ITEMS; t += kSide) masses_of<kSide>(a, key + t, scale, q + t);
    if (a.top_p) {
        // masses of what top-k left: the equals at its end count as far as
        // they were taken
        const Digits dg = digits_of(top, umax_(least, kept.key));
        const uint64_t qk = kept.key ? mass_of(a, kept.key, scale) * kept.ties : 0;
        uint64_t sum = 0;
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) sum += key[t] > kept.key ? q[t] : 0;
        sum = group_sum<NT>(sum, lds) + qk;
        uint64_t most = share_of(a.share, sum);
        uint32_t z = 0;
        int shift = 24;
        for (; dg.more(shift); shift -= 8) {
            __syncthreads();
            for (uint32_t b = threadIdx.x; b < kSmallBins; b += NT) s_hist[b] = 0;
            __syncthreads();
#pragma unroll
            for (int t = 0; t < ITEMS; ++t)
                if (key[t] > kept.key && q[t] && dg.reach(key[t], z, shift))
                    atomicAdd(&s_hist[dg.at(key[t], shift)], (unsigned long long)q[t]);
            if (qk && threadIdx.x == 0 && dg.reach(kept.key, z, shift))
                atomicAdd(&s_hist[dg.at(kept.key, shift)], (unsigned long long)qk);
            uint64_t above;
            z = z << 8 | pass_bin<NT>(s_hist, most, &above, s_out);
            most -= above;
        }
        const uint32_t k = top ? dg.key(z, shift + 8) : 0u;
        const uint64_t qp = mass_of(a, k, scale);
        uint64_t ties = qp ? most / qp + 1 : 0;
        if (k == kept.key && ties > kept.ties) ties = kept.ties;
        kept = Kept{k, ties < 0xFFFFFFFFu ? (uint32_t)ties : 0xFFFFFFFFu};
    }
    if (kept.key) {  // equals of the last key in earlier threads
        uint32_t mine = 0, all;
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) mine += key[t] == kept.key ? 1u : 0u;
        uint32_t place = group_scan<NT>(mine, lds, &all);
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) {
            if (key[t] < kept.key) q[t] = 0;
            if (key[t] == kept.key && place++ >= kept.ties) q[t] = 0;
        }
    }
    uint64_t run = 0, total;
#pragma unroll
    for (int t = 0; t < ITEMS; ++t) {
        if ((double)q[t] < a.least) q[t] = 0;
        run += q[t];
    }
    run = group_scan<NT>(run, lds, &total);
    // a thread's entries are followed by an empty one, so that threads do not
    // meet in a bank
    constexpr int kApart = ITEMS > 1 ? ITEMS + 1 : 1;
#pragma unroll
    for (int t = 0; t < ITEMS; ++t) s_run[threadIdx.x * kApart + t] = run += q[t];
    __syncthreads();
    auto run_at = [&](uint32_t j) { return s_run[ITEMS > 1 ? j + j / ITEMS : j]; };
    for (int64_t d = threadIdx.x; d < a.draws; d += NT) {
        const int64_t at = row * a.draws + d;
        const uint64_t r = share_of(uniform_bits(a.uniform[at]), total);
        uint32_t lo = 0;  // candidates with at most r up to them
#pragma unroll
        for (uint32_t step = NT * ITEMS / 2; step > 0; step /= 2)
            if (run_at(lo + step - 1) <= r) lo += step;
        if (total == 0)
            write_draw(a, at, -1, 0, 1);
        else
            write_draw(a, at, id(lo), run_at(lo) - (lo ? run_at(lo - 1) : 0), total);
    }
    __syncthreads();
}

// Draws from rows of a workgroup. kList: the rows are lists, a.n entries each,
// of which a.top_k <= NT stay. kFew: a.top_k <= NT stay of a row. These are put
// side by side before anything is done about their masses: a candidate a
// thread, where forming them all takes most of the time (a row of 16384
// entries, 128 to be kept, without and with top-p: 28 and 40 us, 19 and 23 side
// by side).
enum { kAll = 0, kFew = 1, kList = 2 };
constexpr int waves_of(int NT) { return NT == kBlock ? 3 : 4; }  // of a SIMD: registers are held to that
template <int NT, int ITEMS, int FORM>
__global__ __launch_bounds__(NT, waves_of(NT)) void k_draw_rows(DrawArgs a, Lists lists) {
    constexpr int kHeld = FORM == kAll ? ITEMS : 1;  // candidates of a thread that masses are formed of
    __shared__ uint64_t s_run[NT * (kHeld + 1)];
    __shared__ unsigned long long s_hist[kSmallBins];
    __shared__ uint64_t lds[NT / kWave + 2];
    uint64_t *s_out = lds + NT / kWave;
    uint32_t *s_key = (uint32_t *)(s_run + NT), *s_id = s_key + NT;  // behind the running masses of one each
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        uint32_t key[ITEMS], mine = 0, over = 0;  // the largest, and ~key, for the least
        const uint32_t j0 = threadIdx.x * ITEMS;
        const uint32_t *list_id = FORM == kList ? lists.id + row * lists.stride : nullptr;
        if (FORM == kList) {
#pragma unroll
            for (int t = 0; t < ITEMS; t += 4) {
                const uint32_t j = j0 + t, last = lists.stride - 4;
                const uint4 v = *(const uint4 *)(lists.key + row * lists.stride + (j < last ? j : last));
                key[t] = j <= last ? v.x : 0u;
                key[t + 1] = j <= last ? v.y : 0u;
                key[t + 2] = j <= last ? v.z : 0u;
                key[t + 3] = j <= last ? v.w : 0u;
            }
        } else {
            const uint32_t len = row_length(a, row);
#pragma unroll
            for (int t = 0; t < ITEMS; t += 4) load_keys(a, row, j0 + t, len, len, key + t);
        }
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) {
            mine = umax_(mine, key[t]);
            over = umax_(over, key[t] ? ~key[t] : 0u);
        }
        const uint32_t top = group_max<NT>(mine, lds);
        const bool filters = a.top_k < (uint32_t)a.n || a.top_p;
        const uint32_t least = filters ? ~group_max<NT>(over, lds) : 0u;
        Kept kept{0, 0xFFFFFFFFu};
        if (a.form == kBest)
            kept = Kept{top, 1};
        else if (a.top_k < (uint32_t)a.n)
            kept = top_kept<NT, ITEMS>(key, mine, a.top_k, top, least, s_hist, lds, s_out);
        if (FORM == kAll) {
            draw_from<NT, kHeld>(a, row, key, kept, top, least, s_run, s_hist, lds, s_out,
                                 [&](uint32_t j) { return j; });
            continue;
        }
        const uint32_t count = place_kept<NT, ITEMS>(key, kept, lds, [&](int t, uint32_t place) {
            s_key[place] = key[t];
            s_id[place] = FORM == kList ? list_id[j0 + t] : j0 + t;
        });
        __syncthreads();
        const uint32_t held[kHeld] = {threadIdx.x < count ? s_key[threadIdx.x] : 0u};
        draw_from<NT, kHeld>(a, row, held, Kept{0, 0xFFFFFFFFu}, top, umax_(least, kept.key), s_run, s_hist, lds,
                             s_out, [&](uint32_t j) { return s_id[j]; });
    }
}

// ---- lists of a long row's best --------------------------------------------

// A stretch of a row: its first `want` candidates in the order of the scores,
// listed in the order of the row. The first `want` of the row are among those
// of its stretches. (256 stretches of bfloat16 logits, 200 of each: 14.5 us.)
// WAVES of a SIMD, to which registers are held: 8 put two workgroups on a
// compute unit and spill some (2048 stretches: 90 -> 77 us, 256: 16 -> 18, with
// the launch).
constexpr int kListThreads = 1024, kListItems = 16;
constexpr uint32_t kListStretch = kListThreads * kListItems;
constexpr uint64_t kListOnce = 256;  // stretches that the compute units take at once, one each
template <int WAVES>
__global__ __launch_bounds__(kListThreads, WAVES) void k_draw_list(DrawArgs a, Lists w, uint64_t block0) {
    __shared__ unsigned long long s_hist[kSmallBins];
    __shared__ uint64_t lds[kListThreads / kWave + 2];
    const uint64_t block = block0 + blockIdx.x;
    const int64_t row = (int64_t)(block / w.stretches);
    const uint32_t at = (uint32_t)(block % w.stretches), len = row_length(a, row);
    const uint32_t i0 = at * kListStretch, j0 = i0 + threadIdx.x * kListItems;
    const uint32_t i1 = len <= i0 ? i0 : len - i0 < kListStretch ? len : i0 + kListStretch;
    uint32_t key[kListItems], mine = 0, over = 0;
#pragma unroll
    for (int t = 0; t < kListItems; t += 4) load_keys(a, row, j0 + t, i1, len, key + t);
#pragma unroll
    for (int t = 0; t < kListItems; ++t) {
        mine = umax_(mine, key[t]);
        over = umax_(over, key[t] ? ~key[t] : 0u);
    }
    const uint32_t top = group_max<kListThreads>(mine, lds), least = ~group_max<kListThreads>(over, lds);
    const Kept kept = top_kept<kListThreads, kListItems>(key, mine, w.want, top, least, s_hist, lds,
                                                         lds + kListThreads / kWave);
    const size_t first = (size_t)row * w.stride + (size_t)at * w.want;
    const uint32_t count = place_kept<kListThreads, kListItems>(key, kept, lds, [&](int t, uint32_t place) {
        w.key[first + place] = key[t];
        w.id[first + place] = j0 + t;
    });
    const uint32_t end = at + 1 == w.stretches ? w.stride - at * w.want : w.want;
    for (uint32_t e = count + threadIdx.x; e < end; e += kListThreads) w.key[first + e] = 0;
}

// ---- rows over many workgroups --------------------------------------------

// The filters' passes cut a row into stretches, a large workgroup each; the
// running masses are made in parts, kParts to a stretch, of slices of kSlice
// candidates, a wave each, and quads of four, a lane each.
constexpr uint32_t kThreads = 1024;
constexpr uint32_t kParts = 4;
constexpr uint32_t kSlice = 4 * kWave;
constexpr int64_t kPartTile = 4 * kBlock;
constexpr int64_t kGranule = kParts * kSlice;  // a stretch is of whole slices of parts
constexpr uint32_t kStretches = 256;  // of all rows, about; of a row, at most
// A pass ends with an atomic add for every bin that a workgroup met, 20 to
// 25 of them in a nanosecond on the whole chip: the first digit, which every
// candidate has, gets few bins, the later ones the rest. Adds to one address
// wait for each other, so rows of many stretches have copies of its bins.
constexpr uint32_t kDigits = 3;
constexpr uint32_t kCopies = 4, kCopiesFrom = 64;
constexpr uint32_t kBins0 = 512, kBins1 = 4096, kBins2 = 2048;
constexpr uint32_t kBinsAll = kCopies * kBins0 + kBins1 + kBins2;
__device__ constexpr uint32_t bins_of(int digit) { return digit == 0 ? kBins0 : digit == 1 ? kBins1 : kBins2; }
__device__ constexpr uint32_t bins_before(int digit) {
    return digit == 0 ? 0u : digit == 1 ? kCopies * kBins0 : kCopies * kBins0 + kBins1;
}

// The digits found of an offset; left: candidates to be taken (top-k) or mass
// that may still stand before (top-p) among those that have them.
struct Digit {
    uint64_t left;
    uint32_t z, pad;
};
// What a row's passes have found; slot p: after digit p.
struct RowState {
    uint32_t top, least, lift;                       // the row's keys, see Ends
    uint32_t pad;
    Digit count[kDigits], mass[kDigits];             // top-k, top-p
    uint32_t in_key, in_ties;                        // what top-k leaves
    uint32_t kept_key, kept_ties;                    // what both leave
    uint64_t ranked;                                 // whether some equals of kept_key go
};
// The workgroups of a row are counted as they end a pass, in groups first (adds
// to one address wait for each other).
constexpr uint32_t kGroups = 16;
constexpr uint32_t kTickets = kGroups + 1;
constexpr uint32_t kPasses = 2;  // that end with the last workgroup: top-k's and top-p's last

struct LongWork {
    RowState *state;      // [rows]
    uint32_t *tickets;    // [rows][kPasses][kTickets]
    uint2 *ends;          // [rows][stretches] largest key, largest ~key
    uint32_t *counts;     // [rows][kBinsAll]
    uint64_t *masses;     // [rows][kBinsAll]
    uint32_t *ties;       // [rows][parts] equals of the last key
    uint64_t *sums;       // [rows][parts] masses
    uint64_t *slice_run;  // [rows][parts][slices] mass up to the slice's end, in the part
    uint64_t *oct_run;    // [rows][parts][slices][8] mass up to the end of eight quads, in the slice
    uint64_t *quad_run;   // [rows][quads] mass up to the quad's end, in the slice
    int64_t stretch, part, quads;
    uint32_t stretches, parts, slices, copies;
    size_t bytes;
};

LongWork long_layout(void *base, int64_t rows, int64_t n) {
    LongWork w;
    const int64_t most = rows >= (int64_t)kStretches ? 1 : (int64_t)kStretches / rows;
    w.stretch = ((n + most - 1) / most + kGranule - 1) / kGranule * kGranule;
    w.stretches = (uint32_t)((n + w.stretch - 1) / w.stretch);
    w.part = w.stretch / kParts;
    w.parts = (uint32_t)((n + w.part - 1) / w.part);
    w.slices = (uint32_t)(w.part / kSlice);
    w.quads = (n + 3) / 4;
    w.copies = w.stretches >= kCopiesFrom ? kCopies : 1;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        void *p = base ? (char *)base + off : nullptr;
        off += al256(bytes);
        return p;
    };
    const size_t r = (size_t)rows;
    w.state = (RowState *)take(sizeof(RowState) * r);
    w.tickets = (uint32_t *)take(4 * r * kPasses * kTickets);
    w.ends = (uint2 *)take(8 * r * w.stretches);
    w.counts = (uint32_t *)take(4 * r * kBinsAll);
    w.masses = (uint64_t *)take(8 * r * kBinsAll);
    w.ties = (uint32_t *)take(4 * r * w.parts);
    w.sums = (uint64_t *)take(8 * r * w.parts);
    w.slice_run = (uint64_t *)take(8 * (r * w.parts * w.slices + 8));
    w.oct_run = (uint64_t *)take(64 * r * w.parts * w.slices);
    w.quad_run = (uint64_t *)take(8 * (r * (size_t)w.quads + 8));
    w.bytes = off;
    return w;
}

// A row's largest and smallest key, and its offsets key - least moved up so
// that they fill 32 bits: the first digit tells as much as it can.
struct Ends {
    uint32_t top, least, lift;
};
__device__ __forceinline__ Ends state_ends(const RowState &s) { return Ends{s.top, s.least, s.lift}; }
__device__ __forceinline__ uint32_t offset_of(uint32_t key, const Ends &e) { return (key - e.least) << e.lift; }
__device__ __forceinline__ uint32_t offset_key(uint32_t z, const Ends &e) { return e.least + (z >> e.lift); }
__device__ __forceinline__ uint32_t digit_of(uint32_t z, int digit) {
    return digit == 0 ? z >> 23 : digit == 1 ? z >> 11 & 4095u : z & 2047u;
}
__device__ __forceinline__ uint32_t digit_shift(int digit) { return digit == 0 ? 23u : digit == 1 ? 11u : 0u; }
// whether an offset has the digits before `digit` of another
__device__ __forceinline__ bool same_before(uint32_t a, uint32_t b, int digit) {
    return digit == 0 || ((a ^ b) >> digit_shift(digit - 1)) == 0;
}

template <int NT>
__device__ __forceinline__ Ends row_ends(const LongWork &w, int64_t row, uint64_t *lds) {
    static_assert(NT >= (int)kStretches, "a stretch a thread");
    uint2 e = make_uint2(0, 0);
    if (threadIdx.x < w.stretches) e = w.ends[row * w.stretches + threadIdx.x];
    const uint32_t top = group_max<NT>(e.x, lds), over = group_max<NT>(e.y, lds);
    const uint32_t spread = top ? top - ~over : 0u;
    return Ends{top, ~over, (uint32_t)__builtin_clz(spread | 1u)};
}

// A word that other workgroups have added to in this launch.
template <typename V>
__device__ __forceinline__ V agent_load(const V *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The bin from the top in which the running sum passes `most` (above <= most <
// above + its count); left: what `most` is more than the sum above it, in_bin:
// its count. False if
// the sum of all is no more than `most`. share (not 2^64 - 1): most is that
// share of the sum. extra is added to bin extra_bin.
template <int NT, int DIGIT, typename V>
__device__ bool cross_bin(const V *hist, uint32_t copies, uint64_t most, uint64_t share, uint32_t extra_bin,
                          uint64_t extra, uint32_t *bin, uint64_t *left, uint64_t *in_bin, uint64_t *lds) {
    constexpr uint32_t kBins = bins_of(DIGIT), kMine = kBins > NT ? kBins / NT : 1;
    uint64_t *out = lds + NT / kWave;
    const uint32_t top = kBins - 1 - threadIdx.x * kMine;
    uint64_t c[kMine], sum = 0, total;
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) {
        c[j] = 0;
        if (threadIdx.x * kMine + j < kBins) {
            if (top - j == extra_bin) c[j] = extra;
            for (uint32_t r = 0; r < (DIGIT ? 1u : copies); ++r)
                c[j] += agent_load(&hist[r * kBins0 + bins_before(DIGIT) + top - j]);
        }
        sum += c[j];
    }
    uint64_t above = group_scan<NT>(sum, lds, &total);
    if (share != ~(uint64_t)0) most = share_of(share, total);
    if (threadIdx.x == 0) {
        out[0] = 0;
        out[1] = 0;
        out[2] = 0;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) {
        if (above <= most && most < above + c[j]) {
            out[0] = top - j;
            out[1] = most - above;
            out[2] = c[j];
        }
        above += c[j];
    }
    __syncthreads();
    *bin = (uint32_t)out[0];
    *left = out[1];
    *in_bin = out[2];
    return most < total;
}

// Whether this workgroup is the last of its row to end a pass: it sees what the
// others have added. Only atomics pass between the workgroups, and all of
// them work on memory that the whole chip sees: each wave waits for its own to
// be done, and the last workgroup reads with atomic loads. (A fence for the
// whole chip would write the caches back: 70 us a pass.)
__device__ bool last_of_row(const LongWork &w, int64_t row, uint32_t at, int pass, uint64_t *lds) {
    uint32_t *t = w.tickets + ((size_t)row * kPasses + pass) * kTickets;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t g = at % kGroups, groups = w.stretches < kGroups ? w.stretches : kGroups;
        const uint32_t members = (w.stretches - g + kGroups - 1) / kGroups;
        bool last = __hip_atomic_fetch_add(&t[g], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == members;
        if (last)
            last = __hip_atomic_fetch_add(&t[kGroups], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == groups;
        lds[0] = last;
    }
    __syncthreads();
    const bool last = lds[0] != 0;
    __syncthreads();
    return last;
}

// A digit is read off its counts by every workgroup of the next pass on its
// own (all at once: 2 M candidates, 7 to 8 us a pass; by the last workgroup of
// its pass 11 us), the last digit by the last workgroup of its pass, since the
// passes after it are of many small workgroups. keep: whether to keep it.

// top-k's offset with the digit that pass DIGIT has counted.
// (before: with the digits before; what another workgroup of this launch
// keeps is not to be read.)
template <int DIGIT>
__device__ Digit end_count(const DrawArgs &a, const LongWork &w, int64_t row, const Ends &e, const Digit &before,
                           bool keep, uint64_t *lds) {
    RowState &s = w.state[row];
    const uint32_t z0 = DIGIT ? before.z : 0u, n0 = DIGIT ? (uint32_t)before.left : a.top_k;
    uint64_t left, in_bin;
    uint32_t b;
    const bool found = cross_bin<kThreads, DIGIT>(w.counts + (size_t)row * kBinsAll, w.copies,
                                                  (uint64_t)n0 - 1, ~(uint64_t)0, ~0u, 0, &b, &left, &in_bin, lds);
    // (need 0: the row has fewer than top_k candidates, and keeps them all)
    const uint32_t z = z0 | b << digit_shift(DIGIT), need = n0 && found ? (uint32_t)left + 1u : 0u;
    const Digit d{need, z, 0};
    if (!keep || threadIdx.x != 0) return d;
    s.count[DIGIT] = d;
    if (DIGIT == kDigits - 1) {
        const bool all = need == 0 || e.top == 0;
        s.in_key = s.kept_key = all ? 0u : offset_key(z, e);
        s.in_ties = s.kept_ties = all ? 0xFFFFFFFFu : need;
        s.ranked = !all && need < in_bin;
    }
    return d;
}

// What top-k left.
__device__ __forceinline__ Kept count_kept(const DrawArgs &a, const LongWork &w, int64_t row) {
    if (a.top_k >= (uint32_t)a.n) return Kept{0, 0xFFFFFFFFu};
    return Kept{w.state[row].in_key, w.state[row].in_ties};
}

// The same of top-p's digits, by masses.
template <int DIGIT>
__device__ Digit end_mass(const DrawArgs &a, const LongWork &w, int64_t row, const Kept &in, const Ends &e,
                          const Scale &scale, const Digit &before, bool keep, uint64_t *lds) {
    RowState &s = w.state[row];
    const uint32_t z0 = DIGIT ? before.z : 0u;
    // top-k's equals, which the histogram leaves out
    const uint64_t extra = in.key ? mass_of(a, in.key, scale) * in.ties : 0;
    const uint32_t zi = in.key ? offset_of(in.key, e) : 0u;
    const uint32_t extra_bin = in.key && same_before(zi, z0, DIGIT) ? digit_of(zi, DIGIT) : ~0u;
    uint32_t b;
    uint64_t left, in_bin;
    cross_bin<kThreads, DIGIT>(w.masses + (size_t)row * kBinsAll, w.copies,
                               DIGIT ? before.left : 0, DIGIT ? ~(uint64_t)0 : a.share,
                               extra_bin, extra, &b, &left, &in_bin, lds);
    const uint32_t z = z0 | b << digit_shift(DIGIT);
    const Digit d{left, z, 0};
    if (!keep || threadIdx.x != 0) return d;
    s.mass[DIGIT] = d;
    if (DIGIT == kDigits - 1) {
        const uint32_t key = e.top ? offset_key(z, e) : 0u;
        const uint64_t q = mass_of(a, key, scale);
        uint64_t ties = q ? left / q + 1 : 0;
        if (key == in.key && ties > in.ties) ties = in.ties;
        s.kept_key = key;
        s.kept_ties = ties < 0xFFFFFFFFu ? (uint32_t)ties : 0xFFFFFFFFu;
        // the bin's mass is that of all equals that could stay; of those that
        // top-k cut, some are not in it
        s.ranked = q && (ties * q < in_bin || (key == in.key && in.ties != 0xFFFFFFFFu));
    }
    return d;
}

// Every candidate's key of [i0, i1) of a row, over a workgroup of NT threads,
// two quads on their way at a time; N keys a visit.
template <int NT, int N, typename F>
__device__ __forceinline__ void each_key(const DrawArgs &a, int64_t row, uint32_t i0, uint32_t i1, uint32_t len,
                                         F visit) {
    constexpr int kAhead = 2;
    for (uint32_t t0 = i0; t0 < i1; t0 += kAhead * 4 * NT) {
        uint32_t k[kAhead][4];
        load_quads<kAhead>(a, row, t0 + threadIdx.x * 4, 4 * NT, i1, len, k);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (t0 + u * 4 * NT >= i1) break;
#pragma unroll
            for (int t = 0; t < 4; t += N) visit(k[u] + t);
        }
    }
}

struct Place {
    int64_t row;
    uint32_t i0, i1, len;  // the stretch (or part) of the row, cut to its length
    uint32_t at;           // its number in the row
};
__device__ __forceinline__ Place place_of(const DrawArgs &a, uint32_t pieces, int64_t length, uint64_t block) {
    Place p;
    p.row = (int64_t)(block / pieces);
    p.at = (uint32_t)(block % pieces);
    p.len = row_length(a, p.row);
    p.i0 = p.at * (uint32_t)length;
    p.i1 = p.len <= p.i0 ? p.i0 : p.len - p.i0 < (uint32_t)length ? p.len : p.i0 + (uint32_t)length;
    return p;
}

// Largest and smallest keys; clears the row's bins for the passes that follow.
__global__ __launch_bounds__(kThreads) void k_draw_ends(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint64_t lds[kThreads / kWave];
    const Place p = place_of(a, w.stretches, w.stretch, block0 + blockIdx.x);
    const uint32_t bins = kBinsAll;
    if (p.at == 0 && threadIdx.x < kPasses * kTickets) w.tickets[(size_t)p.row * kPasses * kTickets + threadIdx.x] = 0;
    for (uint32_t b = p.at * kThreads + threadIdx.x; b < bins; b += w.stretches * kThreads) {
        if (a.top_k < (uint32_t)a.n) w.counts[(size_t)p.row * bins + b] = 0;
        if (a.top_p) w.masses[(size_t)p.row * bins + b] = 0;
    }
    uint32_t top = 0, over = 0;
    each_key<kThreads, 1>(a, p.row, p.i0, p.i1, p.len, [&](const uint32_t *k) {
        top = umax_(top, *k);
        over = umax_(over, *k ? ~*k : 0u);
    });
    top = group_max<kThreads>(top, lds);
    over = group_max<kThreads>(over, lds);
    if (threadIdx.x == 0) w.ends[p.row * w.stretches + p.at] = make_uint2(top, over);
}

// The ends of a row in its first pass, which keeps them, and in the others.
__device__ __forceinline__ Ends pass_ends(const LongWork &w, const Place &p, bool first, uint64_t *lds) {
    RowState &s = w.state[p.row];
    if (!first) return state_ends(s);
    const Ends e = row_ends<kThreads>(w, p.row, lds);
    if (p.at == 0 && threadIdx.x == 0) {
        s.top = e.top;
        s.least = e.least;
        s.lift = e.lift;
    }
    return e;
}

// Counts of a digit of the offsets that have top-k's earlier digits.
template <int DIGIT>
__global__ __launch_bounds__(kThreads) void k_draw_count(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint32_t s_hist[bins_of(DIGIT)];
    __shared__ uint64_t lds[kThreads / kWave + 3];
    const Place p = place_of(a, w.stretches, w.stretch, block0 + blockIdx.x);
    for (uint32_t b = threadIdx.x; b < bins_of(DIGIT); b += kThreads) s_hist[b] = 0;
    const Ends e = pass_ends(w, p, DIGIT == 0, lds);
    Digit before{};
    if (DIGIT > 1) before = w.state[p.row].count[DIGIT > 1 ? DIGIT - 2 : 0];
    if (DIGIT > 0) before = end_count<DIGIT ? DIGIT - 1 : 0>(a, w, p.row, e, before, p.at == 0, lds);
    const uint32_t z0 = before.z;
    __syncthreads();
    each_key<kThreads, 1>(a, p.row, p.i0, p.i1, p.len, [&](const uint32_t *k) {
        const uint32_t z = offset_of(*k, e);
        if (*k && same_before(z, z0, DIGIT)) atomicAdd(&s_hist[digit_of(z, DIGIT)], 1u);
    });
    __syncthreads();
    uint32_t *out = w.counts + (size_t)p.row * kBinsAll + bins_before(DIGIT) + (DIGIT ? 0u : p.at % w.copies * kBins0);
    for (uint32_t b = threadIdx.x; b < bins_of(DIGIT); b += kThreads)
        if (s_hist[b]) atomicAdd(&out[b], s_hist[b]);
    if (DIGIT == kDigits - 1 && last_of_row(w, p.row, p.at, 0, lds))
        end_count<DIGIT>(a, w, p.row, e, before, true, lds);
}

// Adds the masses of four candidates above `in` to a digit's bins, those that
// have the digits of z0 before it.
template <int DIGIT>
__device__ __forceinline__ void add_masses(const DrawArgs &a, const uint32_t k[4], uint32_t in, uint32_t z0,
                                           const Ends &e, const Scale &scale, unsigned long long *hist) {
    uint32_t z[4], some = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        z[t] = offset_of(k[t], e);
        some |= (k[t] > in && same_before(z[t], z0, DIGIT) ? 1u : 0u) << t;
    }
    if (some == 0) return;
    uint64_t q[4];
    masses_of<4>(a, k, scale, q);
#pragma unroll
    for (int t = 0; t < 4; ++t)
        if (some >> t & 1u && q[t]) atomicAdd(&hist[digit_of(z[t], DIGIT)], (unsigned long long)q[t]);
}

// Masses of a digit of the offsets that have top-p's earlier digits.
template <int DIGIT>
__global__ __launch_bounds__(kThreads) void k_draw_mass(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ unsigned long long s_hist[bins_of(DIGIT)];
    __shared__ uint64_t lds[kThreads / kWave + 3];
    const Place p = place_of(a, w.stretches, w.stretch, block0 + blockIdx.x);
    for (uint32_t b = threadIdx.x; b < bins_of(DIGIT); b += kThreads) s_hist[b] = 0;
    const Ends e = pass_ends(w, p, DIGIT == 0 && a.top_k >= (uint32_t)a.n, lds);
    const Scale scale = scale_of(a, e.top);
    const Kept in = count_kept(a, w, p.row);
    Digit before{};
    if (DIGIT > 1) before = w.state[p.row].mass[DIGIT > 1 ? DIGIT - 2 : 0];
    if (DIGIT > 0) before = end_mass<DIGIT ? DIGIT - 1 : 0>(a, w, p.row, in, e, scale, before, p.at == 0, lds);
    const uint32_t z0 = before.z;
    __syncthreads();
    each_key<kThreads, 4>(a, p.row, p.i0, p.i1, p.len, [&](const uint32_t *k) {
        add_masses<DIGIT>(a, k, in.key, z0, e, scale, s_hist);
    });
    __syncthreads();
    unsigned long long *out = (unsigned long long *)(
        w.masses + (size_t)p.row * kBinsAll + bins_before(DIGIT) + (DIGIT ? 0u : p.at % w.copies * kBins0));
    for (uint32_t b = threadIdx.x; b < bins_of(DIGIT); b += kThreads)
        if (s_hist[b]) atomicAdd(&out[b], s_hist[b]);
    if (DIGIT == kDigits - 1 && last_of_row(w, p.row, p.at, 1, lds))
        end_mass<DIGIT>(a, w, p.row, in, e, scale, before, true, lds);
}

// The row's largest key and what the filters keep of it.
__device__ __forceinline__ uint32_t row_kept(const DrawArgs &a, const LongWork &w, int64_t row, Kept *kept,
                                             uint64_t *lds) {
    if (a.top_p || a.top_k < (uint32_t)a.n) {
        const RowState &s = w.state[row];
        *kept = Kept{s.kept_key, s.kept_ties};
        return s.top;
    }
    const uint32_t top = row_ends<kBlock>(w, row, lds).top;
    *kept = a.form == kBest ? Kept{top, 1} : Kept{0, 0};
    return top;
}

__device__ __forceinline__ uint32_t ties_of(const Kept &kept, const uint32_t k[4]) {
    uint32_t n = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) n += k[t] == kept.key ? 1u : 0u;
    return n;
}

// Whether some of the equals of the last key go, so that their order counts.
__device__ __forceinline__ bool row_ranked(const DrawArgs &a, const LongWork &w, int64_t row) {
    return a.form == kBest || ((a.top_p || a.top_k < (uint32_t)a.n) && w.state[row].ranked);
}

// Equals of the last key, per part.
__global__ __launch_bounds__(kBlock) void k_draw_ties(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint64_t lds[kWavesPerBlock + 2];
    const Place p = place_of(a, w.parts, w.part, block0 + blockIdx.x);
    Kept kept;
    row_kept(a, w, p.row, &kept, lds);
    if (!row_ranked(a, w, p.row)) return;
    uint32_t ties = 0;
    each_key<kBlock, 4>(a, p.row, p.i0, p.i1, p.len, [&](const uint32_t *k) { ties += ties_of(kept, k); });
    ties = group_sum<kBlock>(ties, lds);
    if (threadIdx.x == 0) w.ties[p.row * w.parts + p.at] = ties;
}

// What of four candidates' masses the filters leave: `before` equals of the
// last key come earlier, which counts if they are ranked.
__device__ __forceinline__ uint64_t masses_left(const DrawArgs &a, const Scale &scale, const Kept &kept, bool ranked,
                                                const uint32_t k[4], uint32_t before, uint64_t q[4]) {
    uint32_t some = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        some |= k[t] && k[t] >= kept.key ? 1u : 0u;
        q[t] = 0;
    }
    if (some == 0) return 0;
    masses_of<4>(a, k, scale, q);
    uint64_t sum = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        bool stays = k[t] > kept.key;
        if (k[t] == kept.key) stays = !ranked || before++ < kept.ties;
        if (!stays || (double)q[t] < a.least) q[t] = 0;
        sum += q[t];
    }
    return sum;
}

// Running masses of the quads of a slice, the slices of a part, and the parts'
// sums. CUT: whether a filter by order is on.
template <bool CUT>
__global__ __launch_bounds__(kBlock) void k_draw_run(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint64_t lds[kWavesPerBlock];
    const uint64_t block = block0 + blockIdx.x;
    const Place p = place_of(a, w.parts, w.part, block);
    const uint32_t lane = threadIdx.x % kWave;
    Kept kept;
    const Scale scale = scale_of(a, row_kept(a, w, p.row, &kept, lds));
    uint32_t place = 0;  // equals before
    const bool ranked = CUT && row_ranked(a, w, p.row);
    if (ranked) {
        for (uint32_t b = threadIdx.x; b < p.at; b += kBlock) place += w.ties[p.row * w.parts + b];
        place = group_sum<kBlock>(place, lds);
    }
    uint64_t run = 0;
    const uint32_t n = (uint32_t)a.n, end = n - p.i0 < (uint32_t)w.part ? n : p.i0 + (uint32_t)w.part;
    constexpr int kAhead = 2;
    for (uint32_t t0 = p.i0; t0 < end; t0 += kAhead * (uint32_t)kPartTile) {
        uint32_t keys[kAhead][4];
        load_quads<kAhead>(a, p.row, t0 + threadIdx.x * 4, (uint32_t)kPartTile, p.i1, p.len, keys);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t tile = t0 + u * (uint32_t)kPartTile, j = tile + threadIdx.x * 4;
            if (tile >= end) break;
            const uint32_t *k = keys[u];
            uint32_t before = 0, all;
            if (ranked) {
                before = place + group_scan<kBlock>(ties_of(kept, k), lds, &all);
                place += all;
            }
            uint64_t q[4], total;
            const uint64_t mine = masses_left(a, scale, kept, ranked, k, before, q);
            const uint64_t upto = wave_scan(mine);  // in the slice
            if (j < end) w.quad_run[p.row * w.quads + j / 4] = upto;
            const uint64_t slice = run + group_scan<kBlock>(mine, lds, &total) + mine;
            const uint32_t c = (tile - p.i0) / kSlice + threadIdx.x / kWave;
            if (c < w.slices) {  // (a tile may pass the part's end)
                const size_t at = block * w.slices + c;
                if (lane % 8 == 7) w.oct_run[at * 8 + lane / 8] = upto;
                if (lane == kWave - 1) w.slice_run[at] = slice;
            }
            run += total;
        }
    }
    if (threadIdx.x == 0) w.sums[p.row * w.parts + p.at] = run;
}

// The first of `count` <= 8 running sums that is more than r; r: what is left.
// All eight are loaded at once (the array has room for them): a draw waits for
// the memory once a level, not three times.
__device__ __forceinline__ uint32_t pick8(const uint64_t *v, uint32_t count, uint64_t &r) {
    typedef uint64_t u2 __attribute__((ext_vector_type(2), aligned(8)));
    u2 x[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) x[t] = *(const u2 *)(v + 2 * t);
    uint32_t at = 0;
    uint64_t below = 0;
#pragma unroll
    for (uint32_t t = 0; t < 7; ++t) {
        const uint64_t y = t & 1 ? x[t / 2].y : x[t / 2].x;
        if (t + 1 < count && y <= r) {
            at = t + 1;
            below = y;
        }
    }
    r -= below;
    return at;
}

// The draws, a thread each: a workgroup takes kBlock of a row's. The part is
// found in LDS, the slice and the quad in their running masses, and the
// candidate from the scores of its quad.
template <bool CUT>
__global__ __launch_bounds__(kBlock) void k_draw_search(DrawArgs a, LongWork w, uint64_t groups, uint64_t block0) {
    constexpr uint32_t kMost = kStretches * kParts, kMine = kMost / kBlock;
    __shared__ uint64_t s_run[kMost];
    __shared__ uint64_t lds[kWavesPerBlock];
    const int64_t row = (int64_t)((block0 + blockIdx.x) / groups);
    const int64_t d = (int64_t)((block0 + blockIdx.x) % groups) * kBlock + threadIdx.x;
    uint64_t c[kMine], sum = 0, total;
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) {
        const uint32_t at = threadIdx.x * kMine + j;
        sum += c[j] = at < w.parts ? w.sums[row * w.parts + at] : 0;
    }
    uint64_t run = group_scan<kBlock>(sum, lds, &total);
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) s_run[threadIdx.x * kMine + j] = run += c[j];
    Kept kept;
    const Scale scale = scale_of(a, row_kept(a, w, row, &kept, lds));
    __syncthreads();
    if (d >= a.draws) return;
    const int64_t at = row * a.draws + d;
    if (total == 0) {
        write_draw(a, at, -1, 0, 1);
        return;
    }
    uint64_t r = share_of(uniform_bits(a.uniform[at]), total);
    uint32_t part = 0;
#pragma unroll
    for (uint32_t step = kMost / 2; step > 0; step /= 2)
        if (s_run[part + step - 1] <= r) part += step;
    if (part) r -= s_run[part - 1];
    const int64_t rest = a.n - (int64_t)part * w.part;
    uint32_t slice = 0, slices = (uint32_t)(rest < w.part ? (rest + kSlice - 1) / kSlice : w.slices);
    const size_t slice0 = ((size_t)row * w.parts + part) * w.slices;
    uint64_t below = 0;
    while (slices > 8) {
        const uint32_t half = slices / 2;
        const uint64_t x = w.slice_run[slice0 + slice + half - 1];
        if (x <= r) {
            slice += half;
            slices -= half;
            below = x;
        } else {
            slices = half;
        }
    }
    // (running sums of the part up to here: the first of the eight are compared
    // with r itself)
    const uint64_t in_part = r;
    slice += pick8(w.slice_run + slice0 + slice, slices, r);
    r = r == in_part ? in_part - below : r;
    const int64_t first = (int64_t)part * w.part + (int64_t)slice * kSlice;
    const uint32_t count = first + kSlice < a.n ? kSlice / 4 : (uint32_t)((a.n - first + 3) / 4);
    const uint64_t in_slice = r;
    const uint32_t oct = pick8(w.oct_run + (slice0 + slice) * 8, (count + 7) / 8, r);
    const uint64_t *quads = w.quad_run + row * w.quads + first / 4;
    const uint64_t oct_from = in_slice - r;
    r = in_slice;
    uint32_t quad = pick8(quads + oct * 8, count - oct * 8 < 8 ? count - oct * 8 : 8, r);
    uint64_t quad_from = in_slice - r;
    if (quad == 0) quad_from = oct_from;
    r = in_slice - quad_from;
    quad += oct * 8;
    const uint32_t j = (uint32_t)first + quad * 4, len = row_length(a, row);
    uint32_t k[4];
    load_keys(a, row, j, len, len, k);
    uint64_t q[4], larger = 0, equal = 0;
    masses_of<4>(a, k, scale, q);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if (k[t] < kept.key || (double)q[t] < a.least) q[t] = 0;
        if (k[t] > kept.key)
            larger += q[t];
        else
            equal = equal > q[t] ? equal : q[t];
    }
    // how many of the equals stay: what is in the quad's mass
    uint64_t staying = ~(uint64_t)0;
    if (CUT && equal) staying = (quads[quad] - quad_from - larger) / equal;
    uint32_t id = 0;
    uint64_t mass = 0, upto = 0;
    bool found = false;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if (k[t] == kept.key && (staying == 0 || staying-- == 0)) q[t] = 0;
        upto += q[t];
        if (!found && upto > r) {
            found = true;
            id = t;
            mass = q[t];
        }
    }
    write_draw(a, at, j + id, mass, total);
}

constexpr int64_t kRowSmall = 512, kRowMiddle = 4096, kRowLarge = 16384;
// Lists of a row's best are drawn from where they have no more entries than a
// workgroup has threads, and all of a row's fit into a workgroup; two launches
// where the passes take up to ten. Without and with top-p, logits: 64 rows of
// 50021, top_k 1000: 32 and 36 us (lists), 57 and 94 (passes); one row of
// 131072, top_k 1000: 35 and 40, 35 and 57; one of 2 M, top_k 128: 29 and 34, 42
// and 66. (Lists of 4096 entries: 63 and 78 us for 64 rows, as the passes. That is
// for few draws a row: 400000 from one row of 2 M, top_k 128, take 358 us, with a
// top_k for passes 62.)
constexpr int64_t kListRow = kRowLarge;
size_t list_bytes(int64_t rows) { return 2 * al256(4 * (size_t)rows * kListRow); }
constexpr uint64_t kBlocksMost = (uint64_t)1 << 21;  // workgroups of a launch (fewer than 2^32 threads)

}  // namespace

size_t draw_work_bytes(int64_t rows, int64_t n, int64_t) {
    if (n <= kRowLarge || rows == 0) return 256;
    const size_t passes = long_layout(nullptr, rows, n).bytes, lists = list_bytes(rows);
    return passes > lists ? passes : lists;
}

hipError_t launch_draw(int64_t rows, int64_t n, const void *scores, int64_t stride, const int32_t *lengths,
                       const gs_draw_params &p, int64_t draws, const double *uniform, int32_t *ids, float *prob,
                       void *work, hipStream_t s) {
    if (rows <= 0 || draws <= 0) return hipSuccess;
    DrawArgs a;
    a.scores = scores;
    a.rows = rows;
    a.n = n;
    a.stride = stride;
    a.draws = draws;
    a.lengths = lengths;
    a.uniform = uniform;
    a.ids = ids;
    a.prob = prob;
    const bool logits = p.logits != 0;
    a.flip = logits ? ~0u : 0u;
    a.floor = logits ? -__builtin_inff() : 0.0f;
    a.form = p.temperature == 0.0 ? kBest : logits ? kExp : p.temperature == 1.0 ? kRatio : kPower;
    a.rate = a.form == kBest ? 0.0 : (logits ? 1.4426950408889634 : 1.0) / p.temperature;
    int up = 0;
    while (((int64_t)1 << up) < n) ++up;
    a.bits = 62 - up < 52 ? 62 - up : 52;
    a.least = p.min_p * (double)((uint64_t)1 << a.bits);
    a.top_p = p.top_p < 1.0 && a.form != kBest;
    a.share = (uint64_t)(p.top_p * 0x1p53);
    a.top_k = p.top_k > 0 && p.top_k < n && a.form != kBest ? (uint32_t)p.top_k : 0xFFFFFFFFu;
    a.bf16 = p.type == GS_SCORE_BF16;
    const int64_t want = a.form == kBest ? 1 : a.top_k;
    auto rows_by = [&](auto threads, auto items, auto form, const DrawArgs &d, const Lists &l) {
        constexpr int NT = decltype(threads)::value;
        const int64_t most = (int64_t)1 << (NT == 64 ? 20 : 16);
        prof_begin("draw_rows", s);
        hipLaunchKernelGGL((k_draw_rows<NT, decltype(items)::value, decltype(form)::value>),
                           dim3((uint32_t)(rows < most ? rows : most)), dim3(NT), 0, s, d, l);
        prof_end("draw_rows", s);
        return hipGetLastError();
    };
    using I4 = std::integral_constant<int, 4>;
    using I8 = std::integral_constant<int, 8>;
    using I16 = std::integral_constant<int, 16>;
    using T64 = std::integral_constant<int, 64>;
    using T256 = std::integral_constant<int, 256>;
    using T1024 = std::integral_constant<int, 1024>;
    using All = std::integral_constant<int, kAll>;
    using Few = std::integral_constant<int, kFew>;
    using List = std::integral_constant<int, kList>;
    if (n <= kRowLarge) {
        a.top_k = want < n ? (uint32_t)want : 0xFFFFFFFFu;
        auto by = [&](auto threads, auto items) {
            if (a.top_k <= (uint32_t)decltype(threads)::value) return rows_by(threads, items, Few(), a, Lists{});
            return rows_by(threads, items, All(), a, Lists{});
        };
        return n <= kRowSmall ? by(T64(), I8()) : n <= kRowMiddle ? by(T256(), I16()) : by(T1024(), I16());
    }
    auto over = [](uint64_t blocks, auto launch) {
        for (uint64_t b = 0; b < blocks; b += kBlocksMost)
            launch(dim3((uint32_t)(blocks - b < kBlocksMost ? blocks - b : kBlocksMost)), b);
    };
    const int64_t stretches = (n + kListStretch - 1) / kListStretch;
    if (want <= kListThreads && stretches * want <= kListRow) {
        Lists l;
        l.stretches = (uint32_t)stretches;
        l.want = (uint32_t)want;
        l.stride = (uint32_t)(stretches * want + 3) / 4 * 4;
        l.key = (uint32_t *)work;
        l.id = (uint32_t *)((char *)work + list_bytes(rows) / 2);
        prof_begin("draw_list", s);
        over((uint64_t)rows * l.stretches, [&](dim3 nb, uint64_t b) {
            if ((uint64_t)rows * l.stretches > kListOnce)
                hipLaunchKernelGGL(k_draw_list<8>, nb, dim3(kListThreads), 0, s, a, l, b);
            else
                hipLaunchKernelGGL(k_draw_list<4>, nb, dim3(kListThreads), 0, s, a, l, b);
        });
        prof_end("draw_list", s);
        DrawArgs d = a;
        d.n = stretches * want;
        d.top_k = (uint32_t)want;
        if (d.n <= 1024 && want <= 256) return rows_by(T256(), I4(), List(), d, l);
        if (d.n <= 4096) return rows_by(T1024(), I4(), List(), d, l);
        return rows_by(T1024(), I16(), List(), d, l);
    }
    const LongWork w = long_layout(work, rows, n);
    const uint64_t blocks = (uint64_t)rows * w.stretches, parts = (uint64_t)rows * w.parts;
    const dim3 tb(kThreads), pb(kBlock);
    prof_begin("draw_filter", s);
    over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_ends, nb, tb, 0, s, a, w, b); });
    if (a.top_k != 0xFFFFFFFFu) {
        over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_count<0>, nb, tb, 0, s, a, w, b); });
        over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_count<1>, nb, tb, 0, s, a, w, b); });
        over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_count<2>, nb, tb, 0, s, a, w, b); });
    }
    if (a.top_p) {
        over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_mass<0>, nb, tb, 0, s, a, w, b); });
        over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_mass<1>, nb, tb, 0, s, a, w, b); });
        over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_mass<2>, nb, tb, 0, s, a, w, b); });
    }
    const bool cut = a.top_k != 0xFFFFFFFFu || a.top_p || a.form == kBest;
    if (cut) over(parts, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_ties, nb, pb, 0, s, a, w, b); });
    prof_end("draw_filter", s);
    prof_begin("draw_pick", s);
    const uint64_t groups = ((uint64_t)draws + kBlock - 1) / kBlock, draw_blocks = (uint64_t)rows * groups;
    if (cut) {
        over(parts, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_run<true>, nb, pb, 0, s, a, w, b); });
        over(draw_blocks, [&](dim3 nb, uint64_t b) {
            hipLaunchKernelGGL(k_draw_search<true>, nb, pb, 0, s, a, w, groups, b);
        });
    } else {
        over(parts, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_run<false>, nb, pb, 0, s, a, w, b); });
        over(draw_blocks, [&](dim3 nb, uint64_t b) {
            hipLaunchKernelGGL(k_draw_search<false>, nb, pb, 0, s, a, w, groups, b);
        });
    }
    prof_end("draw_pick", s);
    return hipGetLastError();
}

}  // namespace gs
