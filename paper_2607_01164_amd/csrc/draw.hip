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
// search it. Longer rows are cut into stretches over many workgroups, with a
// launch for each pass, and the running mass in the workspace.
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
    uint32_t logits, bf16, form;
    int32_t bits;     // k
};

// A score's place in the order as an unsigned number; 0: never drawn.
__device__ __forceinline__ uint32_t key_of(const DrawArgs &a, uint32_t b) {
    const float x = __uint_as_float(b);
    if (!a.logits) return x > 0.0f ? b : 0u;
    if (!(x > -__builtin_inff())) return 0u;
    const uint32_t c = __float_as_uint(x + 0.0f);  // -0 as 0
    return c ^ ((uint32_t)((int32_t)c >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint32_t score_key(const DrawArgs &a, int64_t at) {
    return key_of(a, a.bf16 ? (uint32_t)((const uint16_t *)a.scores)[at] << 16 : ((const uint32_t *)a.scores)[at]);
}
__device__ __forceinline__ double key_score(const DrawArgs &a, uint32_t key) {
    const uint32_t b = !a.logits ? key : (key & 0x80000000u) ? key ^ 0x80000000u : ~key;
    return (double)__uint_as_float(b);
}

// Keys of candidates j .. j + 3 of a row, 0 from len on.
__device__ __forceinline__ void load_keys(const DrawArgs &a, int64_t row, int64_t j, int64_t len, uint32_t k[4]) {
    typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
    const int64_t at = row * a.stride + j;
    if (j + 4 <= len) {
        if (a.bf16) {
            const u2 v = *(const u2 *)((const uint16_t *)a.scores + at);
            k[0] = v.x << 16;
            k[1] = v.x & 0xFFFF0000u;
            k[2] = v.y << 16;
            k[3] = v.y & 0xFFFF0000u;
        } else {
            const u4 v = *(const u4 *)((const uint32_t *)a.scores + at);
            k[0] = v.x;
            k[1] = v.y;
            k[2] = v.z;
            k[3] = v.w;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) k[t] = key_of(a, k[t]);
    } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) k[t] = j + t < len ? score_key(a, at + t) : 0u;
    }
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

// What turns a row's keys into masses, given its largest key. (Formed without
// a division or a library call a candidate: they cost more than the candidate
// itself.)
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

// q of a candidate. Adding 2^52 to a number from 0 to 2^52 rounds it to a whole
// one, which the sum's bits then count.
__device__ __forceinline__ uint64_t mass_of(const DrawArgs &a, uint32_t key, const Scale &s) {
    if (key == s.top) return key ? (uint64_t)1 << a.bits : 0;
    if (key == 0 || s.best) return 0;
    const double x = key_score(a, key);
    double v;
    if (a.form == kRatio)
        v = x * s.at;
    else if (a.form == kPower)
        v = exp2_of((log2_of(x) - s.at) * a.rate, a.bits);
    else
        v = exp2_of((x - s.at) * a.rate, a.bits);
    return __builtin_bit_cast(uint64_t, v + 0x1p52) - __builtin_bit_cast(uint64_t, 0x1p52);
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

__device__ __forceinline__ int64_t row_length(const DrawArgs &a, int64_t row) {
    if (!a.lengths) return a.n;
    const int64_t l = a.lengths[row];
    return l < 0 ? 0 : l > a.n ? a.n : l;
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
__device__ __forceinline__ uint64_t last_lane(uint64_t x) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(x >> 32), kWave - 1) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((uint32_t)x, kWave - 1);
}
__device__ __forceinline__ uint32_t last_lane(uint32_t x) { return __builtin_amdgcn_readlane(x, kWave - 1); }

// Exclusive sums over a workgroup of NT threads; *total gets the sum. lds: NT /
// kWave entries, free again after a barrier.
template <int NT, typename V>
__device__ __forceinline__ V group_scan(V x, uint64_t *lds, V *total) {
    const V incl = wave_scan(x);
    if (NT == kWave) {
        *total = last_lane(incl);
        return incl - x;
    }
    const uint32_t wave = threadIdx.x / kWave;
    __syncthreads();
    if (threadIdx.x % kWave == kWave - 1) lds[wave] = incl;
    __syncthreads();
    V before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) {
        const V v = (V)lds[w];
        if ((uint32_t)w < wave) before += v;
        all += v;
    }
    *total = all;
    return before + incl - x;
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
    x = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) x = umax_(x, (uint32_t)lds[w]);
    return x;
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

template <int NT, int ITEMS>
__global__ __launch_bounds__(NT) void k_draw_rows(DrawArgs a) {
    // a thread's entries are followed by an empty one, so that threads do not
    // meet in a bank
    __shared__ uint64_t s_run[NT * (ITEMS + 1)];
    __shared__ unsigned long long s_hist[kSmallBins];
    __shared__ uint64_t lds[NT / kWave + 2];
    uint64_t *s_out = lds + NT / kWave;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t len = row_length(a, row);
        uint32_t key[ITEMS], top = 0, over = 0;  // over: ~key, for the least
        uint64_t q[ITEMS];
        const int64_t j0 = (int64_t)threadIdx.x * ITEMS;
#pragma unroll
        for (int t = 0; t < ITEMS; t += 4) load_keys(a, row, j0 + t, len, key + t);
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) {
            top = umax_(top, key[t]);
            over = umax_(over, key[t] ? ~key[t] : 0u);
        }
        top = group_max<NT>(top, lds);
        const Scale scale = scale_of(a, top);
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) q[t] = mass_of(a, key[t], scale);
        Kept kept{0, 0xFFFFFFFFu};
        if (a.form == kBest) {
            kept = Kept{top, 1};
        } else if (a.top_k < (uint32_t)a.n || a.top_p) {
            const uint32_t least = ~group_max<NT>(over, lds);  // 2^32 - 1: no candidate
            const uint32_t spread = top ? top - least : 0u;
            const int first = spread ? (31 - __builtin_clz(spread)) / 8 * 8 : 0;
            // the digits above `shift` of a candidate's offset are those of z
            auto in_reach = [&](uint32_t k, uint32_t z, int shift) {
                return k != 0 && (shift >= 24 || ((k - least) >> (shift + 8)) == z);
            };
            // (with no more than top_k candidates all of them stay)
            if (a.top_k < (uint32_t)a.n && a.top_k < group_sum<NT>(live<ITEMS>(key), lds)) {
                uint64_t need = a.top_k;
                uint32_t z = 0;
                for (int shift = first; shift >= 0; shift -= 8) {
                    __syncthreads();
                    for (uint32_t b = threadIdx.x; b < kSmallBins; b += NT) s_hist[b] = 0;
                    __syncthreads();
#pragma unroll
                    for (int t = 0; t < ITEMS; ++t)
                        if (in_reach(key[t], z, shift))
                            atomicAdd((uint32_t *)&s_hist[(key[t] - least) >> shift & 255u], 1u);
                    uint64_t above;
                    z = z << 8 | pass_bin<NT>(s_hist, need - 1, &above, s_out);
                    need -= above;
                }
                kept = Kept{least + z, (uint32_t)need};
            }
            if (a.top_p) {
                // masses of what top-k left: the equals at its end count as
                // far as they were taken
                const uint64_t qk = kept.key ? mass_of(a, kept.key, scale) * kept.ties : 0;
                uint64_t sum = 0;
#pragma unroll
                for (int t = 0; t < ITEMS; ++t) sum += key[t] > kept.key ? q[t] : 0;
                sum = group_sum<NT>(sum, lds) + qk;
                uint64_t most = share_of(a.share, sum);
                uint32_t z = 0;
                for (int shift = first; shift >= 0; shift -= 8) {
                    __syncthreads();
                    for (uint32_t b = threadIdx.x; b < kSmallBins; b += NT) s_hist[b] = 0;
                    __syncthreads();
#pragma unroll
                    for (int t = 0; t < ITEMS; ++t)
                        if (key[t] > kept.key && q[t] && in_reach(key[t], z, shift))
                            atomicAdd(&s_hist[(key[t] - least) >> shift & 255u], (unsigned long long)q[t]);
                    if (qk && threadIdx.x == 0 && in_reach(kept.key, z, shift))
                        atomicAdd(&s_hist[(kept.key - least) >> shift & 255u], (unsigned long long)qk);
                    uint64_t above;
                    z = z << 8 | pass_bin<NT>(s_hist, most, &above, s_out);
                    most -= above;
                }
                const uint32_t k = top ? least + z : 0u;
                const uint64_t qp = mass_of(a, k, scale);
                uint64_t ties = qp ? most / qp + 1 : 0;
                if (k == kept.key && ties > kept.ties) ties = kept.ties;
                kept = Kept{k, ties < 0xFFFFFFFFu ? (uint32_t)ties : 0xFFFFFFFFu};
            }
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
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) s_run[threadIdx.x * (ITEMS + 1) + t] = run += q[t];
        __syncthreads();
        auto run_at = [&](uint32_t j) { return s_run[j + j / ITEMS]; };
        for (int64_t d = threadIdx.x; d < a.draws; d += NT) {
            const int64_t at = row * a.draws + d;
            const uint64_t r = share_of(uniform_bits(a.uniform[at]), total);
            uint32_t lo = 0;  // candidates with at most r up to them
#pragma unroll
            for (uint32_t step = NT * ITEMS / 2; step > 0; step /= 2)
                if (run_at(lo + step - 1) <= r) lo += step;
            if (total == 0) {
                write_draw(a, at, -1, 0, 1);
            } else {
                write_draw(a, at, lo, run_at(lo) - (lo ? run_at(lo - 1) : 0), total);
            }
        }
        __syncthreads();
    }
}

// ---- rows over many workgroups --------------------------------------------

// A row is cut into stretches, a workgroup each, and a stretch into slices of
// kSlice candidates, a wave each, four a lane.
constexpr uint32_t kThreads = 1024;
constexpr uint32_t kSlice = 4 * kWave;
constexpr int64_t kTile = 4 * kThreads;
constexpr uint32_t kStretches = 256;  // of all rows, about; of a row, at most
constexpr uint32_t kBins = 2048;      // of a digit: 11, 11, 10 bits
constexpr uint32_t kDigits = 3;
// A pass ends with an atomic add for every bin that a workgroup met; those to
// one address wait for each other, so rows of many stretches have copies of
// their bins.
constexpr uint32_t kCopies = 4, kCopiesFrom = 64;
// Up to one draw in so many candidates, a wave works out the masses of the
// slice that a draw falls in; from there on every candidate's running mass is
// written out, 8 bytes each, and a draw is a search. (A wave takes 300
// instructions a draw: 10000 draws from 2 M candidates take it 6 us, as long
// as the 16 MB.)
constexpr int64_t kDrawSparse = 128;

// What a row's passes have found so far; slot p: after digit p.
struct RowState {
    uint32_t count_z[kDigits], count_need[kDigits];  // top-k
    uint32_t mass_z[kDigits], kept_ties;             // top-p; at the end what both keep
    uint64_t mass_left[kDigits];                     // mass that may still stand before
    uint32_t kept_key, pad;
};

struct LongWork {
    RowState *state;      // [rows]
    uint2 *ends;          // [rows][stretches] largest key, largest ~key
    uint32_t *counts;     // [rows][copies][kDigits][kBins]
    uint64_t *masses;     // [rows][copies][kDigits][kBins]
    uint32_t *ties;       // [rows][stretches]
    uint64_t *sums;       // [rows][stretches]
    uint64_t *slice_run;  // [rows][stretches][slices]: mass up to the slice's end, in the stretch
    uint32_t *slice_tie;  // [rows][stretches][slices]: equals of the last key before the slice, in the row
    uint64_t *run;        // [rows][n]: mass in the slice (null: not kept)
    int64_t stretch;
    uint32_t stretches, slices, copies;
    size_t bytes;
};

bool draws_sparse(int64_t n, int64_t draws) { return draws <= n / kDrawSparse; }

LongWork long_layout(void *base, int64_t rows, int64_t n, int64_t draws) {
    LongWork w;
    const int64_t most = rows >= (int64_t)kStretches ? 1 : (int64_t)kStretches / rows;
    w.stretch = ((n + most - 1) / most + kTile - 1) / kTile * kTile;
    w.stretches = (uint32_t)((n + w.stretch - 1) / w.stretch);
    w.slices = (uint32_t)(w.stretch / kSlice);
    w.copies = w.stretches >= kCopiesFrom ? kCopies : 1;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        void *p = base ? (char *)base + off : nullptr;
        off += al256(bytes);
        return p;
    };
    const size_t r = (size_t)rows, c = r * w.stretches;
    w.state = (RowState *)take(sizeof(RowState) * r);
    w.ends = (uint2 *)take(8 * c);
    w.counts = (uint32_t *)take(4 * r * w.copies * kDigits * kBins);
    w.masses = (uint64_t *)take(8 * r * w.copies * kDigits * kBins);
    w.ties = (uint32_t *)take(4 * c);
    w.sums = (uint64_t *)take(8 * c);
    w.slice_run = (uint64_t *)take(8 * c * w.slices);
    w.slice_tie = (uint32_t *)take(4 * c * w.slices);
    w.run = draws_sparse(n, draws) ? nullptr : (uint64_t *)take(8 * r * (size_t)n);
    w.bytes = off;
    return w;
}

// A row's largest and smallest key, and its offsets key - least moved up so
// that they fill 32 bits: the first digit tells as much as it can.
struct Ends {
    uint32_t top, least, lift;
};
__device__ __forceinline__ uint32_t offset_of(uint32_t key, const Ends &e) { return (key - e.least) << e.lift; }
__device__ __forceinline__ uint32_t offset_key(uint32_t z, const Ends &e) { return e.least + (z >> e.lift); }
__device__ __forceinline__ uint32_t digit_of(uint32_t z, int digit) {
    return digit == 0 ? z >> 21 : digit == 1 ? z >> 10 & 2047u : z & 1023u;
}
__device__ __forceinline__ uint32_t digit_shift(int digit) { return digit == 0 ? 21u : digit == 1 ? 10u : 0u; }
// whether an offset has the digits before `digit` of another
__device__ __forceinline__ bool same_before(uint32_t a, uint32_t b, int digit) {
    return digit == 0 || ((a ^ b) >> digit_shift(digit - 1)) == 0;
}

__device__ __forceinline__ Ends row_ends(const LongWork &w, int64_t row, uint64_t *lds) {
    uint2 e = make_uint2(0, 0);
    if (threadIdx.x < w.stretches) e = w.ends[row * w.stretches + threadIdx.x];
    const uint32_t top = group_max<kThreads>(e.x, lds), over = group_max<kThreads>(e.y, lds);
    const uint32_t spread = top ? top - ~over : 0u;
    return Ends{top, ~over, (uint32_t)__builtin_clz(spread | 1u)};
}

// The bin from the top in which the running sum passes `most` (above <= most <
// above + its count); left: what `most` is more than the sum above it. False if
// the sum of all is no more than `most`. share (not 2^64 - 1): most is that
// share of the sum. extra is added to bin extra_bin.
template <typename V>
__device__ bool cross_bin(const V *hist, uint32_t copies, uint64_t most, uint64_t share, uint32_t extra_bin,
                          uint64_t extra, uint32_t *bin, uint64_t *left, uint64_t *lds) {
    constexpr uint32_t kMine = kBins / kThreads;
    uint64_t *out = lds + kThreads / kWave;
    const uint32_t top = kBins - 1 - threadIdx.x * kMine;
    uint64_t c[kMine], sum = 0, total;
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) {
        c[j] = top - j == extra_bin ? extra : 0;
        for (uint32_t r = 0; r < copies; ++r) c[j] += hist[(size_t)r * kDigits * kBins + top - j];
        sum += c[j];
    }
    uint64_t above = group_scan<kThreads>(sum, lds, &total);
    if (share != ~(uint64_t)0) most = share_of(share, total);
    if (threadIdx.x == 0) {
        out[0] = 0;
        out[1] = 0;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) {
        if (above <= most && most < above + c[j]) {
            out[0] = top - j;
            out[1] = most - above;
        }
        above += c[j];
    }
    __syncthreads();
    *bin = (uint32_t)out[0];
    *left = out[1];
    return most < total;
}

// top-k's offset with its digit `digit`, which pass `digit` counted; the row's
// first workgroup keeps it for the later passes.
__device__ Kept count_digit(const DrawArgs &a, const LongWork &w, int64_t row, int digit, bool keep, uint64_t *lds) {
    RowState &s = w.state[row];
    const uint32_t z0 = digit ? s.count_z[digit - 1] : 0u;
    const uint32_t n0 = digit ? s.count_need[digit - 1] : a.top_k;
    uint64_t left;
    uint32_t b;
    const bool found = cross_bin(w.counts + ((size_t)row * w.copies * kDigits + digit) * kBins, w.copies,
                                 (uint64_t)n0 - 1, ~(uint64_t)0, kBins, 0, &b, &left, lds);
    // (need 0: the row has fewer than top_k candidates)
    const Kept k{z0 | b << digit_shift(digit), n0 && found ? (uint32_t)left + 1u : 0u};
    if (keep && threadIdx.x == 0) {
        s.count_z[digit] = k.key;
        s.count_need[digit] = k.ties;
    }
    return k;
}

// What top-k leaves, after its passes; digit: whether its last digit is still
// to be read off.
__device__ Kept count_kept(const DrawArgs &a, const LongWork &w, int64_t row, const Ends &e, bool digit, bool keep,
                           uint64_t *lds) {
    Kept k{0, 0xFFFFFFFFu};
    if (a.top_k >= (uint32_t)a.n) return k;
    if (digit) {
        k = count_digit(a, w, row, kDigits - 1, keep, lds);
    } else {
        k.key = w.state[row].count_z[kDigits - 1];
        k.ties = w.state[row].count_need[kDigits - 1];
    }
    // a row of fewer than top_k candidates keeps them all
    if (k.ties == 0 || e.top == 0) return Kept{0, 0xFFFFFFFFu};
    return Kept{offset_key(k.key, e), k.ties};
}

// The same of top-p's offset, by masses; `in`: what top-k left.
__device__ Kept mass_digit(const DrawArgs &a, const LongWork &w, int64_t row, int digit, bool keep, Kept in,
                           const Ends &e, const Scale &scale, uint64_t *left, uint64_t *lds) {
    RowState &s = w.state[row];
    const uint32_t z0 = digit ? s.mass_z[digit - 1] : 0u;
    // top-k's equals, which the histogram leaves out
    const uint64_t extra = in.key ? mass_of(a, in.key, scale) * in.ties : 0;
    const uint32_t zi = in.key ? offset_of(in.key, e) : 0u;
    const uint32_t extra_bin = in.key && same_before(zi, z0, digit) ? digit_of(zi, digit) : kBins;
    uint32_t b;
    cross_bin(w.masses + ((size_t)row * w.copies * kDigits + digit) * kBins, w.copies,
              digit ? s.mass_left[digit ? digit - 1 : 0] : 0, digit ? ~(uint64_t)0 : a.share, extra_bin, extra, &b,
              left, lds);
    const Kept k{z0 | b << digit_shift(digit), 0};
    if (keep && threadIdx.x == 0) {
        s.mass_z[digit] = k.key;
        s.mass_left[digit] = *left;
    }
    return k;
}

struct Place {
    int64_t row, i0, i1;  // the stretch of the row, cut to its length
    uint32_t stretch;
};
__device__ __forceinline__ Place place_of(const DrawArgs &a, const LongWork &w, uint64_t block) {
    Place p;
    p.row = (int64_t)(block / w.stretches);
    p.stretch = (uint32_t)(block % w.stretches);
    const int64_t len = row_length(a, p.row);
    p.i0 = (int64_t)p.stretch * w.stretch;
    p.i1 = p.i0 + w.stretch < len ? p.i0 + w.stretch : len;
    return p;
}

// Largest and smallest keys; clears the row's bins for the passes that follow.
__global__ __launch_bounds__(kThreads) void k_draw_ends(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint64_t lds[kThreads / kWave];
    const Place p = place_of(a, w, block0 + blockIdx.x);
    const uint32_t bins = w.copies * kDigits * kBins;
    for (uint32_t b = p.stretch * kThreads + threadIdx.x; b < bins; b += w.stretches * kThreads) {
        if (a.top_k < (uint32_t)a.n) w.counts[(size_t)p.row * bins + b] = 0;
        if (a.top_p) w.masses[(size_t)p.row * bins + b] = 0;
    }
    uint32_t top = 0, over = 0;
    for (int64_t i = p.i0 + threadIdx.x * 4; i < p.i1; i += kTile) {
        uint32_t k[4];
        load_keys(a, p.row, i, p.i1, k);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            top = umax_(top, k[t]);
            over = umax_(over, k[t] ? ~k[t] : 0u);
        }
    }
    top = group_max<kThreads>(top, lds);
    over = group_max<kThreads>(over, lds);
    if (threadIdx.x == 0) w.ends[p.row * w.stretches + p.stretch] = make_uint2(top, over);
}

// Counts of a digit of the offsets that have top-k's earlier digits.
template <int DIGIT>
__global__ __launch_bounds__(kThreads) void k_draw_count(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint32_t s_hist[kBins];
    __shared__ uint64_t lds[kThreads / kWave + 2];
    const Place p = place_of(a, w, block0 + blockIdx.x);
    for (uint32_t b = threadIdx.x; b < kBins; b += kThreads) s_hist[b] = 0;
    const Ends e = row_ends(w, p.row, lds);
    uint32_t z0 = 0;
    if (DIGIT > 0) z0 = count_digit(a, w, p.row, DIGIT - 1, p.stretch == 0, lds).key;
    __syncthreads();
    for (int64_t i = p.i0 + threadIdx.x * 4; i < p.i1; i += kTile) {
        uint32_t k[4];
        load_keys(a, p.row, i, p.i1, k);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint32_t z = offset_of(k[t], e);
            if (k[t] && same_before(z, z0, DIGIT)) atomicAdd(&s_hist[digit_of(z, DIGIT)], 1u);
        }
    }
    __syncthreads();
    uint32_t *out = w.counts + (((size_t)p.row * w.copies + p.stretch % w.copies) * kDigits + DIGIT) * kBins;
    for (uint32_t b = threadIdx.x; b < kBins; b += kThreads)
        if (s_hist[b]) atomicAdd(&out[b], s_hist[b]);
}

// Masses of a digit of the offsets that have top-p's earlier digits.
template <int DIGIT>
__global__ __launch_bounds__(kThreads) void k_draw_mass(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ unsigned long long s_hist[kBins];
    __shared__ uint64_t lds[kThreads / kWave + 2];
    const Place p = place_of(a, w, block0 + blockIdx.x);
    for (uint32_t b = threadIdx.x; b < kBins; b += kThreads) s_hist[b] = 0;
    const Ends e = row_ends(w, p.row, lds);
    const Scale scale = scale_of(a, e.top);
    const Kept in = count_kept(a, w, p.row, e, DIGIT == 0, p.stretch == 0, lds);
    uint32_t z0 = 0;
    uint64_t left;
    if (DIGIT > 0) z0 = mass_digit(a, w, p.row, DIGIT - 1, p.stretch == 0, in, e, scale, &left, lds).key;
    __syncthreads();
    for (int64_t i = p.i0 + threadIdx.x * 4; i < p.i1; i += kTile) {
        uint32_t k[4];
        load_keys(a, p.row, i, p.i1, k);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint32_t z = offset_of(k[t], e);
            if (k[t] > in.key && same_before(z, z0, DIGIT)) {
                const uint64_t q = mass_of(a, k[t], scale);
                if (q) atomicAdd(&s_hist[digit_of(z, DIGIT)], (unsigned long long)q);
            }
        }
    }
    __syncthreads();
    unsigned long long *out = (unsigned long long *)(
        w.masses + (((size_t)p.row * w.copies + p.stretch % w.copies) * kDigits + DIGIT) * kBins);
    for (uint32_t b = threadIdx.x; b < kBins; b += kThreads)
        if (s_hist[b]) atomicAdd(&out[b], s_hist[b]);
}

// What both filters keep; every workgroup of a row works it out.
__device__ Kept row_kept(const DrawArgs &a, const LongWork &w, int64_t row, const Ends &e, const Scale &scale,
                         uint64_t *lds) {
    if (a.form == kBest) return Kept{e.top, 1};
    const Kept in = count_kept(a, w, row, e, !a.top_p, false, lds);
    if (!a.top_p) return in;
    uint64_t left;
    const Kept k = mass_digit(a, w, row, kDigits - 1, false, in, e, scale, &left, lds);
    const uint32_t key = e.top ? offset_key(k.key, e) : 0u;
    const uint64_t q = mass_of(a, key, scale);
    uint64_t ties = q ? left / q + 1 : 0;
    if (key == in.key && ties > in.ties) ties = in.ties;
    return Kept{key, ties < 0xFFFFFFFFu ? (uint32_t)ties : 0xFFFFFFFFu};
}

// Equals of the last key, per stretch; the row's first workgroup keeps what
// the filters keep.
__global__ __launch_bounds__(kThreads) void k_draw_ties(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint64_t lds[kThreads / kWave + 2];
    const Place p = place_of(a, w, block0 + blockIdx.x);
    const Ends e = row_ends(w, p.row, lds);
    const Kept kept = row_kept(a, w, p.row, e, scale_of(a, e.top), lds);
    uint32_t ties = 0;
    for (int64_t i = p.i0 + threadIdx.x * 4; i < p.i1; i += kTile) {
        uint32_t k[4];
        load_keys(a, p.row, i, p.i1, k);
#pragma unroll
        for (int t = 0; t < 4; ++t) ties += k[t] == kept.key ? 1u : 0u;
    }
    ties = group_sum<kThreads>(ties, lds);
    if (threadIdx.x == 0) {
        w.ties[p.row * w.stretches + p.stretch] = ties;
        if (p.stretch == 0) {
            w.state[p.row].kept_key = kept.key;
            w.state[p.row].kept_ties = kept.ties;
        }
    }
}

// q of four candidates of which `before` equals of the last key come earlier.
template <bool CUT>
__device__ __forceinline__ void masses_of(const DrawArgs &a, const Scale &scale, const Kept &kept, const uint32_t k[4],
                                          uint32_t before, uint64_t q[4]) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        bool stays = !CUT || k[t] > kept.key;
        if (CUT && k[t] == kept.key) stays = before++ < kept.ties;
        q[t] = stays ? mass_of(a, k[t], scale) : 0;
        if ((double)q[t] < a.least) q[t] = 0;
    }
}
__device__ __forceinline__ uint32_t ties_of(const Kept &kept, const uint32_t k[4]) {
    uint32_t n = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) n += k[t] == kept.key ? 1u : 0u;
    return n;
}

// Running masses of the slices of a stretch, and where wanted of their
// candidates. CUT: whether a filter by order is on.
template <bool CUT>
__global__ __launch_bounds__(kThreads) void k_draw_run(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint64_t lds[kThreads / kWave];
    const Place p = place_of(a, w, block0 + blockIdx.x);
    const uint32_t lane = threadIdx.x % kWave;
    const Ends e = row_ends(w, p.row, lds);
    const Scale scale = scale_of(a, e.top);
    Kept kept{0, 0};
    uint32_t place = 0;  // equals before
    if (CUT) {
        kept = Kept{w.state[p.row].kept_key, w.state[p.row].kept_ties};
        place = group_sum<kThreads>(threadIdx.x < p.stretch ? w.ties[p.row * w.stretches + threadIdx.x] : 0u, lds);
    }
    uint64_t run = 0;
    const int64_t end = p.i0 + w.stretch < a.n ? p.i0 + w.stretch : a.n;
    for (int64_t t0 = p.i0; t0 < end; t0 += kTile) {
        const int64_t j = t0 + threadIdx.x * 4;
        uint32_t k[4];
        load_keys(a, p.row, j, p.i1, k);
        uint32_t before = 0, all;
        if (CUT) {
            before = place + group_scan<kThreads>(ties_of(kept, k), lds, &all);
            place += all;
        }
        uint64_t q[4], total;
        masses_of<CUT>(a, scale, kept, k, before, q);
        const uint64_t mine = q[0] + q[1] + q[2] + q[3];
        const uint64_t to = run + group_scan<kThreads>(mine, lds, &total) + mine;  // up to this lane's end
        const uint64_t at = (uint64_t)blockIdx.x + block0;
        const size_t slice = at * w.slices + (size_t)((t0 - p.i0) / kSlice) + threadIdx.x / kWave;
        if (lane == kWave - 1) w.slice_run[slice] = to;
        if (CUT && lane == 0) w.slice_tie[slice] = before;
        if (w.run && j < end) {
            // from the slice's start
            const uint64_t from = to - mine;
            const uint64_t r = from - ((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(from >> 32)) << 32 |
                                 (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)from));
            uint64_t *out = w.run + p.row * a.n + j;
            const uint64_t r0 = r + q[0], r1 = r0 + q[1], r2 = r1 + q[2], r3 = r2 + q[3];
            if (j + 4 <= end) {
                typedef uint64_t u2 __attribute__((ext_vector_type(2), aligned(8)));
                *(u2 *)out = u2{r0, r1};
                *(u2 *)(out + 2) = u2{r2, r3};
            } else {
                out[0] = r0;
                if (j + 1 < end) out[1] = r1;
                if (j + 2 < end) out[2] = r2;
            }
        }
        run += total;
    }
    if (threadIdx.x == 0) w.sums[p.row * w.stretches + p.stretch] = run;
}

// Running masses of a row's stretches, in LDS (kBlock threads).
__device__ __forceinline__ uint64_t stretch_runs(const LongWork &w, int64_t row, uint64_t *s_run, uint64_t *lds) {
    static_assert(kStretches == kBlock, "a stretch a thread");
    uint64_t total;
    const uint64_t sum = threadIdx.x < w.stretches ? w.sums[row * w.stretches + threadIdx.x] : 0;
    s_run[threadIdx.x] = group_scan<kBlock>(sum, lds, &total) + sum;
    __syncthreads();
    return total;
}

// The stretch and slice that mass r of a row falls in; r becomes what it is
// into the slice.
struct Found {
    uint32_t stretch, slice;
};
__device__ __forceinline__ Found find_slice(const DrawArgs &a, const LongWork &w, int64_t row, const uint64_t *s_run,
                                            uint64_t &r) {
    Found f{0, 0};
#pragma unroll
    for (uint32_t step = kStretches / 2; step > 0; step /= 2)
        if (s_run[f.stretch + step - 1] <= r) f.stretch += step;
    if (f.stretch) r -= s_run[f.stretch - 1];
    const uint64_t *v = w.slice_run + ((size_t)row * w.stretches + f.stretch) * w.slices;
    const int64_t rest = a.n - (int64_t)f.stretch * w.stretch;
    uint32_t hi = (uint32_t)(rest < w.stretch ? (rest + kSlice - 1) / kSlice : w.slices) - 1;
    while (f.slice < hi) {
        const uint32_t mid = (f.slice + hi) / 2;
        if (v[mid] > r)
            hi = mid;
        else
            f.slice = mid + 1;
    }
    if (f.slice) r -= v[f.slice - 1];
    return f;
}

// The draws, a thread each: a workgroup takes kBlock of a row's.
__global__ __launch_bounds__(kBlock) void k_draw_search(DrawArgs a, LongWork w, uint64_t groups, uint64_t block0) {
    __shared__ uint64_t s_run[kStretches];
    __shared__ uint64_t lds[kWavesPerBlock];
    const int64_t row = (int64_t)((block0 + blockIdx.x) / groups);
    const int64_t d = (int64_t)((block0 + blockIdx.x) % groups) * kBlock + threadIdx.x;
    const uint64_t total = stretch_runs(w, row, s_run, lds);
    if (d >= a.draws) return;
    const int64_t at = row * a.draws + d;
    if (total == 0) {
        write_draw(a, at, -1, 0, 1);
        return;
    }
    uint64_t r = share_of(uniform_bits(a.uniform[at]), total);
    const Found f = find_slice(a, w, row, s_run, r);
    const int64_t first = (int64_t)f.stretch * w.stretch + (int64_t)f.slice * kSlice;
    const uint64_t *v = w.run + row * a.n + first;
    uint32_t lo = 0, last = (uint32_t)((first + kSlice < a.n ? (int64_t)kSlice : a.n - first) - 1);
    while (lo < last) {
        const uint32_t mid = (lo + last) / 2;
        if (v[mid] > r)
            last = mid;
        else
            lo = mid + 1;
    }
    write_draw(a, at, first + lo, v[lo] - (lo ? v[lo - 1] : 0), total);
}

// The draws, a wave each, from the scores of their slices.
template <bool CUT>
__global__ __launch_bounds__(kBlock) void k_draw_slice(DrawArgs a, LongWork w, uint64_t groups, uint64_t block0) {
    __shared__ uint64_t s_run[kStretches];
    __shared__ uint64_t lds[kThreads / kWave];
    const int64_t row = (int64_t)((block0 + blockIdx.x) / groups);
    const int64_t d = (int64_t)((block0 + blockIdx.x) % groups) * kWavesPerBlock + threadIdx.x / kWave;
    const uint32_t lane = threadIdx.x % kWave;
    const uint64_t total = stretch_runs(w, row, s_run, lds);
    uint32_t top = 0;
    if (threadIdx.x < w.stretches) top = w.ends[row * w.stretches + threadIdx.x].x;
    const Scale scale = scale_of(a, group_max<kBlock>(top, lds));
    if (d >= a.draws) return;
    const int64_t at = row * a.draws + d;
    if (total == 0) {
        if (lane == 0) write_draw(a, at, -1, 0, 1);
        return;
    }
    uint64_t r = share_of(uniform_bits(a.uniform[at]), total);
    const Found f = find_slice(a, w, row, s_run, r);
    const int64_t first = (int64_t)f.stretch * w.stretch + (int64_t)f.slice * kSlice;
    Kept kept{0, 0};
    uint32_t k[4], before = 0;
    load_keys(a, row, first + lane * 4, row_length(a, row), k);
    if (CUT) {
        kept = Kept{w.state[row].kept_key, w.state[row].kept_ties};
        const uint32_t mine = ties_of(kept, k);
        before = w.slice_tie[((size_t)row * w.stretches + f.stretch) * w.slices + f.slice] + wave_scan(mine) - mine;
    }
    uint64_t q[4];
    masses_of<CUT>(a, scale, kept, k, before, q);
    const uint64_t mine = q[0] + q[1] + q[2] + q[3];
    uint64_t run = wave_scan(mine) - mine;
    // the one lane and candidate whose mass holds r
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if (run <= r && r < run + q[t]) write_draw(a, at, first + lane * 4 + t, q[t], total);
        run += q[t];
    }
}

constexpr int64_t kRowSmall = 512, kRowMiddle = 4096, kRowLarge = 16384;
constexpr uint64_t kBlocksMost = (uint64_t)1 << 21;  // workgroups of a launch (fewer than 2^32 threads)

}  // namespace

size_t draw_work_bytes(int64_t rows, int64_t n, int64_t draws) {
    return n <= kRowLarge || rows == 0 ? 256 : long_layout(nullptr, rows, n, draws).bytes;
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
    a.logits = p.logits != 0;
    a.form = p.temperature == 0.0 ? kBest : a.logits ? kExp : p.temperature == 1.0 ? kRatio : kPower;
    a.rate = a.form == kBest ? 0.0 : (a.logits ? 1.4426950408889634 : 1.0) / p.temperature;
    int up = 0;
    while (((int64_t)1 << up) < n) ++up;
    a.bits = 62 - up < 52 ? 62 - up : 52;
    a.least = p.min_p * (double)((uint64_t)1 << a.bits);
    a.top_p = p.top_p < 1.0 && a.form != kBest;
    a.share = (uint64_t)(p.top_p * 0x1p53);
    a.top_k = p.top_k > 0 && p.top_k < n && a.form != kBest ? (uint32_t)p.top_k : 0xFFFFFFFFu;
    a.bf16 = p.type == GS_SCORE_BF16;
    if (n <= kRowLarge) {
        const uint32_t most = n <= kRowSmall ? 1u << 20 : 1u << 16;
        const dim3 nb(rows < (int64_t)most ? (uint32_t)rows : most);
        prof_begin("draw_rows", s);
        if (n <= kRowSmall)
            hipLaunchKernelGGL((k_draw_rows<64, 8>), nb, dim3(64), 0, s, a);
        else if (n <= kRowMiddle)
            hipLaunchKernelGGL((k_draw_rows<256, 16>), nb, dim3(256), 0, s, a);
        else
            hipLaunchKernelGGL((k_draw_rows<1024, 16>), nb, dim3(1024), 0, s, a);
        prof_end("draw_rows", s);
        return hipGetLastError();
    }
    const LongWork w = long_layout(work, rows, n, draws);
    auto over = [](uint64_t blocks, auto launch) {
        for (uint64_t b = 0; b < blocks; b += kBlocksMost)
            launch(dim3((uint32_t)(blocks - b < kBlocksMost ? blocks - b : kBlocksMost)), b);
    };
    const uint64_t blocks = (uint64_t)rows * w.stretches;
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
    if (cut) over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_ties, nb, tb, 0, s, a, w, b); });
    prof_end("draw_filter", s);
    prof_begin("draw_pick", s);
    if (cut)
        over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_run<true>, nb, tb, 0, s, a, w, b); });
    else
        over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_run<false>, nb, tb, 0, s, a, w, b); });
    const uint64_t each = w.run ? kBlock : kWavesPerBlock;
    const uint64_t groups = ((uint64_t)draws + each - 1) / each;
    if (w.run)
        over((uint64_t)rows * groups,
             [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_search, nb, pb, 0, s, a, w, groups, b); });
    else if (cut)
        over((uint64_t)rows * groups,
             [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_slice<true>, nb, pb, 0, s, a, w, groups, b); });
    else
        over((uint64_t)rows * groups,
             [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_slice<false>, nb, pb, 0, s, a, w, groups, b); });
    prof_end("draw_pick", s);
    return hipGetLastError();
}

}  // namespace gs
