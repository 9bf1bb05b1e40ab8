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

struct DrawArgs {
    const void *scores;
    int64_t rows, n, stride, draws;
    const int32_t *lengths;
    const double *uniform;
    int32_t *ids;
    float *prob;
    double temperature;
    double least;     // min_p 2^k
    uint64_t share;   // floor(top_p 2^53)
    uint32_t top_k;   // 2^32 - 1: off
    uint32_t top_p;   // whether top_p is on
    uint32_t logits, bf16;
    int32_t bits;     // k
};

// A score's place in the order as an unsigned number; 0: never drawn.
__device__ __forceinline__ uint32_t score_key(const DrawArgs &a, int64_t at) {
    const uint32_t b = a.bf16 ? (uint32_t)((const uint16_t *)a.scores)[at] << 16 : ((const uint32_t *)a.scores)[at];
    const float x = __uint_as_float(b);
    if (!a.logits) return x > 0.0f ? b : 0u;
    if (!(x > -__builtin_inff())) return 0u;
    const uint32_t c = __float_as_uint(x + 0.0f);  // -0 as 0
    return c ^ ((uint32_t)((int32_t)c >> 31) | 0x80000000u);
}
__device__ __forceinline__ double key_score(const DrawArgs &a, uint32_t key) {
    const uint32_t b = !a.logits ? key : (key & 0x80000000u) ? key ^ 0x80000000u : ~key;
    return (double)__uint_as_float(b);
}

// q of a candidate, given the row's largest key.
__device__ __forceinline__ uint64_t mass_of(const DrawArgs &a, uint32_t key, uint32_t top) {
    const uint64_t unit = (uint64_t)1 << a.bits;
    if (key == top) return key ? unit : 0;
    if (key == 0 || a.temperature == 0.0) return 0;
    const double x = key_score(a, key), m = key_score(a, top);
    if (m == __builtin_inf()) return 0;
    double e;
    if (a.logits)
        e = exp((x - m) / a.temperature);
    else if (a.temperature == 1.0)
        e = x / m;
    else
        e = exp(log(x / m) / a.temperature);
    return (uint64_t)rint(e * (double)unit);
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

__device__ __forceinline__ int64_t row_length(const DrawArgs &a, int64_t row) {
    if (!a.lengths) return a.n;
    const int64_t l = a.lengths[row];
    return l < 0 ? 0 : l > a.n ? a.n : l;
}

__device__ __forceinline__ void write_draw(const DrawArgs &a, int64_t at, int64_t id, uint64_t q, uint64_t total) {
    a.ids[at] = (int32_t)id;
    if (a.prob) a.prob[at] = id >= 0 ? (float)((double)q / (double)total) : 0.0f;
}

// ---- rows of a workgroup --------------------------------------------------

template <int NT>
__device__ __forceinline__ uint64_t group_sum(uint64_t x, uint64_t *lds) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
    if (NT == kWave) return x;
    const uint32_t wave = threadIdx.x / kWave;
    __syncthreads();
    if (threadIdx.x % kWave == 0) lds[wave] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) x += lds[w];
    return x;
}

template <int NT>
__device__ __forceinline__ uint64_t group_excl_scan(uint64_t x, uint64_t *lds, uint64_t *total) {
    const uint64_t incl = wave_incl_sum64(x);
    const uint32_t wave = threadIdx.x / kWave;
    __syncthreads();
    if (threadIdx.x % kWave == kWave - 1) lds[wave] = incl;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) {
        const uint64_t v = lds[w];
        if ((uint32_t)w < wave) before += v;
        all += v;
    }
    *total = all;
    return before + incl - x;
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

template <int NT, int ITEMS>
__global__ __launch_bounds__(NT) void k_draw_rows(DrawArgs a) {
    __shared__ uint64_t s_run[NT * ITEMS];
    __shared__ uint64_t lds[NT / kWave];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t len = row_length(a, row);
        uint32_t key[ITEMS], top = 0;
        uint64_t q[ITEMS];
        const int64_t j0 = (int64_t)threadIdx.x * ITEMS;
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) {
            key[t] = j0 + t < len ? score_key(a, row * a.stride + j0 + t) : 0u;
            top = umax_(top, key[t]);
        }
        top = group_max<NT>(top, lds);
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) q[t] = mass_of(a, key[t], top);
        Kept kept{0, 0xFFFFFFFFu};
        if (a.temperature == 0.0) {
            kept = Kept{top, 1};
        } else {
            if (a.top_k < (uint32_t)a.n) {
                // the largest key that top_k candidates reach, bit by bit
                uint32_t k = 0;
                for (int b = 31; b >= 0; --b) {
                    const uint32_t c = k | 1u << b;
                    uint32_t reach = 0;
#pragma unroll
                    for (int t = 0; t < ITEMS; ++t) reach += key[t] >= c ? 1u : 0u;
                    if (group_sum<NT>(reach, lds) >= a.top_k) k = c;
                }
                uint32_t above = 0;
#pragma unroll
                for (int t = 0; t < ITEMS; ++t) above += key[t] > k ? 1u : 0u;
                kept = Kept{k, a.top_k - (uint32_t)group_sum<NT>(above, lds)};
            }
            if (a.top_p) {
                // masses of what top-k left: the equals at its end count as
                // far as they were taken
                const uint64_t qk = mass_of(a, kept.key, top);
                uint64_t sum = 0;
#pragma unroll
                for (int t = 0; t < ITEMS; ++t) sum += key[t] > kept.key ? q[t] : 0;
                sum = group_sum<NT>(sum, lds) + (qk ? qk * kept.ties : 0);
                const uint64_t most = share_of(a.share, sum);
                // the least key with at most that much above it, bit by bit
                uint32_t k = 0xFFFFFFFFu;
                for (int b = 31; b >= 0; --b) {
                    const uint32_t c = k & ~(1u << b);
                    if (c < kept.key) continue;
                    uint64_t above = 0;
#pragma unroll
                    for (int t = 0; t < ITEMS; ++t) above += key[t] > c ? q[t] : 0;
                    if (group_sum<NT>(above, lds) <= most) k = c;
                }
                uint64_t above = 0;
#pragma unroll
                for (int t = 0; t < ITEMS; ++t) above += key[t] > k ? q[t] : 0;
                above = group_sum<NT>(above, lds);
                const uint64_t qp = mass_of(a, k, top);
                uint64_t ties = qp ? (most - above) / qp + 1 : 0;
                if (k == kept.key && ties > kept.ties) ties = kept.ties;
                kept = Kept{k, ties < 0xFFFFFFFFu ? (uint32_t)ties : 0xFFFFFFFFu};
            }
        }
        // equals of the last key in earlier threads
        uint64_t place = 0, total;
        uint32_t mine = 0;
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) mine += key[t] == kept.key ? 1u : 0u;
        place = group_excl_scan<NT>(mine, lds, &total);
        uint64_t run = 0;
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) {
            bool stays = key[t] > kept.key;
            if (key[t] == kept.key) stays = place++ < kept.ties;
            if (!stays || (double)q[t] < a.least) q[t] = 0;
            run += q[t];
        }
        run = group_excl_scan<NT>(run, lds, &total);
#pragma unroll
        for (int t = 0; t < ITEMS; ++t) s_run[j0 + t] = run += q[t];
        __syncthreads();
        for (int64_t d = threadIdx.x; d < a.draws; d += NT) {
            const int64_t at = row * a.draws + d;
            const uint64_t r = share_of(uniform_bits(a.uniform[at]), total);
            uint32_t lo = 0, hi = NT * ITEMS - 1;  // the first with more than r
            while (lo < hi) {
                const uint32_t mid = (lo + hi) / 2;
                if (s_run[mid] > r)
                    hi = mid;
                else
                    lo = mid + 1;
            }
            const uint64_t q1 = s_run[lo] - (lo ? s_run[lo - 1] : 0);
            write_draw(a, at, total ? (int64_t)lo : -1, q1, total);
        }
        __syncthreads();
    }
}

// ---- rows over many workgroups --------------------------------------------

constexpr uint32_t kStretches = 1024;  // of a row, at most
constexpr int64_t kStretchLeast = 2048;
constexpr uint32_t kBins = 2048;       // of a digit: 11, 11, 10 bits
constexpr uint32_t kDigits = 3;
constexpr int kEach = 8;               // candidates of a thread in a tile

// What a row's passes have found so far; slot p: after digit p.
struct RowState {
    uint32_t count_key[kDigits], count_need[kDigits];  // top-k
    uint32_t mass_key[kDigits];
    uint32_t pad;
    uint64_t mass_left[kDigits];                       // top-p: mass that may still stand before
};

struct LongWork {
    RowState *state;     // [rows]
    uint32_t *tops;      // [rows][stretches] largest keys
    uint32_t *counts;    // [rows][kDigits][kBins]
    uint64_t *masses;    // [rows][kDigits][kBins]
    uint32_t *ties;      // [rows][stretches]
    uint64_t *sums;      // [rows][stretches]
    uint64_t *run;       // [rows][n]
    int64_t stretch;
    uint32_t stretches;
    size_t bytes;
};

LongWork long_layout(void *base, int64_t rows, int64_t n) {
    LongWork w;
    w.stretch = (n + kStretches - 1) / kStretches;
    w.stretch = (w.stretch + kStretchLeast - 1) / kStretchLeast * kStretchLeast;
    if (w.stretch < kStretchLeast) w.stretch = kStretchLeast;
    w.stretches = (uint32_t)((n + w.stretch - 1) / w.stretch);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        void *p = base ? (char *)base + off : nullptr;
        off += al256(bytes);
        return p;
    };
    const size_t r = (size_t)rows, c = r * w.stretches;
    w.state = (RowState *)take(sizeof(RowState) * r);
    w.tops = (uint32_t *)take(4 * c);
    w.counts = (uint32_t *)take(4 * r * kDigits * kBins);
    w.masses = (uint64_t *)take(8 * r * kDigits * kBins);
    w.ties = (uint32_t *)take(4 * c);
    w.sums = (uint64_t *)take(8 * c);
    w.run = (uint64_t *)take(8 * r * (size_t)n);
    w.bytes = off;
    return w;
}

__device__ __forceinline__ uint32_t digit_of(uint32_t key, int digit) {
    return digit == 0 ? key >> 21 : digit == 1 ? key >> 10 & 2047u : key & 1023u;
}
__device__ __forceinline__ uint32_t digit_shift(int digit) { return digit == 0 ? 21u : digit == 1 ? 10u : 0u; }
// whether a key has the digits before `digit` of another
__device__ __forceinline__ bool same_before(uint32_t a, uint32_t b, int digit) {
    return digit == 0 || ((a ^ b) >> digit_shift(digit - 1)) == 0;
}

__device__ __forceinline__ uint32_t row_top(const LongWork &w, int64_t row, uint64_t *lds) {
    uint32_t top = 0;
    for (uint32_t c = threadIdx.x; c < w.stretches; c += kBlock) top = umax_(top, w.tops[row * w.stretches + c]);
    return group_max<kBlock>(top, lds);
}

// The bin in which the running sum from the top passes: the first whose sum
// with all above it is more than `most`; below: the sum above it. extra is
// added to bin extra_bin. If the sum of all is no more, bin 0 with all of it
// below.
template <typename V>
__device__ uint32_t cross_bin(const V *__restrict__ hist, uint64_t most, uint32_t extra_bin, uint64_t extra,
                              uint64_t *above_bin, uint64_t *lds) {
    constexpr uint32_t kMine = kBins / kBlock;
    const uint32_t top = kBins - 1 - threadIdx.x * kMine;
    uint64_t c[kMine], sum = 0, total;
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) {
        c[j] = hist[top - j];
        if (top - j == extra_bin) c[j] += extra;
        sum += c[j];
    }
    uint64_t above = group_excl_scan<kBlock>(sum, lds, &total);
    if (threadIdx.x == 0) {
        lds[kWavesPerBlock] = 0;
        lds[kWavesPerBlock + 1] = total;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) {
        if (above <= most && most < above + c[j]) {
            lds[kWavesPerBlock] = top - j;
            lds[kWavesPerBlock + 1] = above;
        }
        above += c[j];
    }
    __syncthreads();
    const uint32_t bin = (uint32_t)lds[kWavesPerBlock];
    *above_bin = lds[kWavesPerBlock + 1];
    __syncthreads();
    return bin;
}

// Total mass of a digit's bins.
__device__ uint64_t bins_sum(const uint64_t *__restrict__ hist, uint64_t *lds) {
    uint64_t sum = 0;
    for (uint32_t b = threadIdx.x; b < kBins; b += kBlock) sum += hist[b];
    return group_sum<kBlock>(sum, lds);
}

// The digit of top-k's key that pass `digit` counted, appended to the row's
// state; the first workgroup of the row keeps it for the later passes.
__device__ void count_digit(const DrawArgs &a, const LongWork &w, int64_t row, int digit, bool keep, uint32_t *key,
                            uint32_t *need, uint64_t *lds) {
    RowState &s = w.state[row];
    const uint32_t k0 = digit ? s.count_key[digit - 1] : 0u;
    const uint32_t n0 = digit ? s.count_need[digit - 1] : a.top_k;
    uint64_t above;
    const uint32_t b = cross_bin(w.counts + (row * kDigits + digit) * kBins, n0 - 1, kBins, 0, &above, lds);
    *key = k0 | b << digit_shift(digit);
    *need = n0 - (uint32_t)above;
    if (keep && threadIdx.x == 0) {
        s.count_key[digit] = *key;
        s.count_need[digit] = *need;
    }
}

// What top-k leaves, after its passes.
__device__ Kept count_kept(const DrawArgs &a, const LongWork &w, int64_t row) {
    if (a.top_k >= (uint32_t)a.n) return Kept{0, 0xFFFFFFFFu};
    return Kept{w.state[row].count_key[kDigits - 1], w.state[row].count_need[kDigits - 1]};
}

// The same of top-p's key, by masses; `in`: what top-k left.
__device__ void mass_digit(const DrawArgs &a, const LongWork &w, int64_t row, int digit, bool keep, Kept in,
                           uint32_t top, uint32_t *key, uint64_t *left, uint64_t *lds) {
    RowState &s = w.state[row];
    const uint64_t *hist = w.masses + (row * kDigits + digit) * kBins;
    const uint32_t k0 = digit ? s.mass_key[digit - 1] : 0u;
    // top-k's equals, which the histogram leaves out
    const uint64_t qk = mass_of(a, in.key, top);
    const uint64_t extra = qk ? qk * in.ties : 0;
    const uint32_t extra_bin = same_before(in.key, k0, digit) ? digit_of(in.key, digit) : kBins;
    uint64_t most, above;
    if (digit == 0)
        most = share_of(a.share, bins_sum(hist, lds) + extra);
    else
        most = s.mass_left[digit - 1];
    const uint32_t b = cross_bin(hist, most, extra_bin, extra, &above, lds);
    *key = k0 | b << digit_shift(digit);
    *left = most - above;
    if (keep && threadIdx.x == 0) {
        s.mass_key[digit] = *key;
        s.mass_left[digit] = *left;
    }
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

// Largest keys; clears the row's bins for the passes that follow.
__global__ __launch_bounds__(kBlock) void k_draw_top(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint64_t lds[kWavesPerBlock];
    const Place p = place_of(a, w, block0 + blockIdx.x);
    const uint32_t step = w.stretches * kBlock;
    for (uint32_t b = p.stretch * kBlock + threadIdx.x; b < kDigits * kBins; b += step) {
        w.counts[p.row * kDigits * kBins + b] = 0;
        w.masses[p.row * kDigits * kBins + b] = 0;
    }
    uint32_t top = 0;
    for (int64_t i = p.i0 + threadIdx.x; i < p.i1; i += kBlock) top = umax_(top, score_key(a, p.row * a.stride + i));
    top = group_max<kBlock>(top, lds);
    if (threadIdx.x == 0) w.tops[p.row * w.stretches + p.stretch] = top;
}

template <int DIGIT>
__global__ __launch_bounds__(kBlock) void k_draw_count(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint32_t s_hist[kBins];
    __shared__ uint64_t lds[kWavesPerBlock + 2];
    const Place p = place_of(a, w, block0 + blockIdx.x);
    for (uint32_t b = threadIdx.x; b < kBins; b += kBlock) s_hist[b] = 0;
    uint32_t key = 0, need;
    if (DIGIT > 0) count_digit(a, w, p.row, DIGIT - 1, p.stretch == 0, &key, &need, lds);
    __syncthreads();
    for (int64_t i = p.i0 + threadIdx.x; i < p.i1; i += kBlock) {
        const uint32_t k = score_key(a, p.row * a.stride + i);
        if (same_before(k, key, DIGIT)) atomicAdd(&s_hist[digit_of(k, DIGIT)], 1u);
    }
    __syncthreads();
    uint32_t *out = w.counts + (p.row * kDigits + DIGIT) * kBins;
    for (uint32_t b = threadIdx.x; b < kBins; b += kBlock)
        if (s_hist[b]) atomicAdd(&out[b], s_hist[b]);
}

template <int DIGIT>
__global__ __launch_bounds__(kBlock) void k_draw_mass(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ unsigned long long s_hist[kBins];
    __shared__ uint64_t lds[kWavesPerBlock + 2];
    const Place p = place_of(a, w, block0 + blockIdx.x);
    for (uint32_t b = threadIdx.x; b < kBins; b += kBlock) s_hist[b] = 0;
    const uint32_t top = row_top(w, p.row, lds);
    Kept in;
    if (DIGIT == 0 && a.top_k < (uint32_t)a.n)
        count_digit(a, w, p.row, kDigits - 1, p.stretch == 0, &in.key, &in.ties, lds);
    else
        in = count_kept(a, w, p.row);
    uint32_t key = 0;
    uint64_t left;
    if (DIGIT > 0) mass_digit(a, w, p.row, DIGIT - 1, p.stretch == 0, in, top, &key, &left, lds);
    __syncthreads();
    for (int64_t i = p.i0 + threadIdx.x; i < p.i1; i += kBlock) {
        const uint32_t k = score_key(a, p.row * a.stride + i);
        if (k > in.key && same_before(k, key, DIGIT)) {
            const uint64_t q = mass_of(a, k, top);
            if (q) atomicAdd(&s_hist[digit_of(k, DIGIT)], (unsigned long long)q);
        }
    }
    __syncthreads();
    unsigned long long *out = (unsigned long long *)(w.masses + (p.row * kDigits + DIGIT) * kBins);
    for (uint32_t b = threadIdx.x; b < kBins; b += kBlock)
        if (s_hist[b]) atomicAdd(&out[b], s_hist[b]);
}

// What both filters keep; every workgroup of a row works it out.
__device__ Kept row_kept(const DrawArgs &a, const LongWork &w, int64_t row, uint32_t top, uint64_t *lds) {
    if (a.temperature == 0.0) return Kept{top, 1};
    Kept k{0, 0xFFFFFFFFu};
    if (a.top_k < (uint32_t)a.n) {
        if (a.top_p)
            k = count_kept(a, w, row);
        else
            count_digit(a, w, row, kDigits - 1, false, &k.key, &k.ties, lds);
    }
    if (a.top_p) {
        const Kept in = k;
        uint64_t left;
        mass_digit(a, w, row, kDigits - 1, false, in, top, &k.key, &left, lds);
        const uint64_t q = mass_of(a, k.key, top);
        uint64_t ties = q ? left / q + 1 : 0;
        if (k.key == in.key && ties > in.ties) ties = in.ties;
        k.ties = ties < 0xFFFFFFFFu ? (uint32_t)ties : 0xFFFFFFFFu;
    }
    return k;
}

// Equals of the last key, per stretch.
__global__ __launch_bounds__(kBlock) void k_draw_ties(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint64_t lds[kWavesPerBlock + 2];
    const Place p = place_of(a, w, block0 + blockIdx.x);
    const Kept kept = row_kept(a, w, p.row, row_top(w, p.row, lds), lds);
    uint32_t ties = 0;
    for (int64_t i = p.i0 + threadIdx.x; i < p.i1; i += kBlock)
        ties += score_key(a, p.row * a.stride + i) == kept.key ? 1u : 0u;
    const uint64_t sum = group_sum<kBlock>(ties, lds);
    if (threadIdx.x == 0) w.ties[p.row * w.stretches + p.stretch] = (uint32_t)sum;
}

// Running mass inside the stretch, and its sum. CUT: whether a filter by
// order is on.
template <bool CUT>
__global__ __launch_bounds__(kBlock) void k_draw_run(DrawArgs a, LongWork w, uint64_t block0) {
    __shared__ uint64_t lds[kWavesPerBlock + 2];
    const Place p = place_of(a, w, block0 + blockIdx.x);
    const uint32_t top = row_top(w, p.row, lds);
    Kept kept{0, 0};
    uint64_t place = 0;  // equals before
    if (CUT) {
        kept = row_kept(a, w, p.row, top, lds);
        uint64_t t = 0;
        for (uint32_t c = threadIdx.x; c < p.stretch; c += kBlock) t += w.ties[p.row * w.stretches + c];
        place = group_sum<kBlock>(t, lds);
    }
    uint64_t run = 0;
    for (int64_t t0 = p.i0; t0 < p.i0 + w.stretch && t0 < a.n; t0 += kBlock * kEach) {
        const int64_t j0 = t0 + (int64_t)threadIdx.x * kEach;
        uint64_t q[kEach], mine = 0, total;
        uint32_t key[kEach], ties = 0;
#pragma unroll
        for (int t = 0; t < kEach; ++t) {
            key[t] = j0 + t < p.i1 ? score_key(a, p.row * a.stride + j0 + t) : 0u;
            ties += key[t] == kept.key ? 1u : 0u;
        }
        uint64_t at = 0;
        if (CUT) {
            at = place + group_excl_scan<kBlock>(ties, lds, &total);
            place += total;
        }
#pragma unroll
        for (int t = 0; t < kEach; ++t) {
            bool stays = key[t] > kept.key;
            if (CUT && key[t] == kept.key) stays = at++ < kept.ties;
            q[t] = stays ? mass_of(a, key[t], top) : 0;
            if ((double)q[t] < a.least) q[t] = 0;
            mine += q[t];
        }
        uint64_t r = run + group_excl_scan<kBlock>(mine, lds, &total);
        run += total;
#pragma unroll
        for (int t = 0; t < kEach; ++t) {
            r += q[t];
            if (j0 + t < p.i0 + w.stretch && j0 + t < a.n) w.run[p.row * a.n + j0 + t] = r;
        }
    }
    if (threadIdx.x == 0) w.sums[p.row * w.stretches + p.stretch] = run;
}

// The draws: a workgroup takes kBlock of a row's.
__global__ __launch_bounds__(kBlock) void k_draw_pick(DrawArgs a, LongWork w, uint64_t groups, uint64_t block0) {
    constexpr uint32_t kMine = kStretches / kBlock;
    __shared__ uint64_t s_run[kStretches];
    __shared__ uint64_t lds[kWavesPerBlock];
    const int64_t row = (int64_t)((block0 + blockIdx.x) / groups);
    const int64_t d = (int64_t)((block0 + blockIdx.x) % groups) * kBlock + threadIdx.x;
    uint64_t c[kMine], sum = 0, total;
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) {
        const uint32_t k = threadIdx.x * kMine + j;
        c[j] = k < w.stretches ? w.sums[row * w.stretches + k] : 0;
        sum += c[j];
    }
    uint64_t run = group_excl_scan<kBlock>(sum, lds, &total);
#pragma unroll
    for (uint32_t j = 0; j < kMine; ++j) s_run[threadIdx.x * kMine + j] = run += c[j];
    __syncthreads();
    if (d >= a.draws) return;
    const int64_t at = row * a.draws + d;
    if (total == 0) {
        write_draw(a, at, -1, 0, 1);
        return;
    }
    uint64_t r = share_of(uniform_bits(a.uniform[at]), total);
    uint32_t s = 0, hi = kStretches - 1;
    while (s < hi) {
        const uint32_t mid = (s + hi) / 2;
        if (s_run[mid] > r)
            hi = mid;
        else
            s = mid + 1;
    }
    if (s) r -= s_run[s - 1];
    const int64_t first = (int64_t)s * w.stretch;
    const uint64_t *v = w.run + row * a.n + first;
    uint32_t lo = 0, last = (uint32_t)((first + w.stretch < a.n ? w.stretch : a.n - first) - 1);
    while (lo < last) {
        const uint32_t mid = (lo + last) / 2;
        if (v[mid] > r)
            last = mid;
        else
            lo = mid + 1;
    }
    write_draw(a, at, first + lo, v[lo] - (lo ? v[lo - 1] : 0), total);
}

constexpr int64_t kRowSmall = 512, kRowMiddle = 4096, kRowLarge = 16384;
constexpr uint64_t kBlocksMost = (uint64_t)1 << 23;  // workgroups of a launch (fewer than 2^32 threads)

}  // namespace

size_t draw_work_bytes(int64_t rows, int64_t n, int64_t) {
    return n <= kRowLarge || rows == 0 ? 256 : long_layout(nullptr, rows, n).bytes;
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
    a.temperature = p.temperature;
    int up = 0;
    while (((int64_t)1 << up) < n) ++up;
    a.bits = 62 - up < 52 ? 62 - up : 52;
    a.least = p.min_p * (double)((uint64_t)1 << a.bits);
    a.top_p = p.top_p < 1.0 && p.temperature > 0.0;
    a.share = (uint64_t)(p.top_p * 0x1p53);
    a.top_k = p.top_k > 0 && p.top_k < n && p.temperature > 0.0 ? (uint32_t)p.top_k : 0xFFFFFFFFu;
    a.logits = p.logits != 0;
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
    const LongWork w = long_layout(work, rows, n);
    auto over = [](uint64_t blocks, auto launch) {
        for (uint64_t b = 0; b < blocks; b += kBlocksMost)
            launch(dim3((uint32_t)(blocks - b < kBlocksMost ? blocks - b : kBlocksMost)), b);
    };
    const uint64_t blocks = (uint64_t)rows * w.stretches;
    const dim3 tb(kBlock);
    prof_begin("draw_filter", s);
    over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_top, nb, tb, 0, s, a, w, b); });
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
    const bool cut = a.top_k != 0xFFFFFFFFu || a.top_p || p.temperature == 0.0;
    if (cut) over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_ties, nb, tb, 0, s, a, w, b); });
    prof_end("draw_filter", s);
    prof_begin("draw_pick", s);
    if (cut)
        over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_run<true>, nb, tb, 0, s, a, w, b); });
    else
        over(blocks, [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_run<false>, nb, tb, 0, s, a, w, b); });
    const uint64_t groups = ((uint64_t)draws + kBlock - 1) / kBlock;
    over((uint64_t)rows * groups,
         [&](dim3 nb, uint64_t b) { hipLaunchKernelGGL(k_draw_pick, nb, tb, 0, s, a, w, groups, b); });
    prof_end("draw_pick", s);
    return hipGetLastError();
}

}  // namespace gs
