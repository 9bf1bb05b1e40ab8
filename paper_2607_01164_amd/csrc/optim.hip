// The optimiser step (include/gs_optim.h): AdamW over a list of tensors with
// float32 or MXFP8 moments, the global gradient norm, and moments through a
// densification's source map.
//
// Everything is elementwise or a sum, and bound by HBM: on this part a device
// copy of 1 to 4 GiB moves 4.9 to 5.2 TB/s, an addition of two such arrays 5.5
// to 5.9, a fill 6.9, and these kernels' large lists 6.0 to 6.5. A list is cut
// into pieces ("items") of at most one workgroup's work, and one launch
// covers all tensors: a workgroup reads its item's record (addresses, length,
// rates) with scalar loads and needs nothing else of the list.
#include "optim.h"

#include <cmath>

namespace gs {
namespace {

template <typename T>
using Glob = __attribute__((address_space(1))) T;  // global, not generic, addresses
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
// Vectors at any address that their elements may have: global loads and
// stores need no more.
typedef f4v f4a __attribute__((aligned(4)));
typedef u4v u4a __attribute__((aligned(2)));
typedef u2v u2a __attribute__((aligned(2)));
typedef uint32_t u1a __attribute__((aligned(1)));
typedef uint16_t h1a __attribute__((aligned(1)));

constexpr int kFill = 24;  // tensors whose pieces one launch of k_fill_items writes: 2 KB of arguments
// Neighbouring items that one XCD takes: 267 M elements with 8-bit moments
// take as long with 64, 2 % longer with 256, 3 % without, 5 % with 8; in
// bfloat16 with float32 moments 1 % less with 64, with 256 and without.
constexpr uint32_t kXcdItems = 32;
constexpr int64_t kMaxGrid = 1 << 23;  // workgroups of a launch at most: 2^31 threads

struct FillArgs {
    OptimTensor t[kFill];
    uint32_t first[kFill + 1];       // first item of each, counted from the launch's first
    uint32_t first_norm[kFill + 1];  // the same of its NormItems
    int count;
};

// ---- items ----------------------------------------------------------------

// A thread for each item. Lists are laid out once and used for many steps;
// through arguments rather than a copy, so that the call neither waits nor
// keeps the host's list.
__global__ __launch_bounds__(kBlock) void k_fill_items(FillArgs a, OptimItem *items, NormItem *norms) {
    const uint32_t i = blockIdx.x * kBlock + threadIdx.x;
    if (i < a.first[a.count]) {
        int k = 0;
        while (i >= a.first[k + 1]) ++k;
        const OptimTensor t = a.t[k];
        const int64_t base = (int64_t)(i - a.first[k]) * kOptimChunk;
        const int64_t left = t.n - base;
        OptimItem it;
        const int ps = t.flags & kParamBf16 ? 2 : 4, gs = t.flags & kGradBf16 ? 2 : 4;
        const int ms = t.flags & kMoments8 ? 1 : 4;
        it.p = (char *)t.p + base * ps;
        it.g = (const char *)t.g + base * gs;
        it.m = (char *)t.m + base * ms;
        it.v = (char *)t.v + base * ms;
        it.ms = t.ms ? t.ms + base / 32 : nullptr;
        it.vs = t.vs ? t.vs + base / 32 : nullptr;
        it.base = base;
        it.count = (int32_t)(left < kOptimChunk ? left : kOptimChunk);
        it.place = t.place;
        it.lr = t.lr;
        it.wd = t.wd;
        it.flags = t.flags;
        it.pad = 0;
        items[i] = it;
    }
    if (i < a.first_norm[a.count]) {
        int k = 0;
        while (i >= a.first_norm[k + 1]) ++k;
        const OptimTensor t = a.t[k];
        const int64_t base = (int64_t)(i - a.first_norm[k]) * kNormChunk;
        const int64_t left = t.n - base;
        NormItem it;
        it.g = (const char *)t.g + base * (t.flags & kGradBf16 ? 2 : 4);
        it.count = (int32_t)(left < kNormChunk ? left : kNormChunk);
        it.flags = t.flags;
        norms[i] = it;
    }
}

// Through words and shifts: an item that is read as one object stays in
// memory, which the compiler then moves to LDS.
__device__ __forceinline__ OptimItem load_item(const OptimItem *items, uint32_t i) {
    static_assert(sizeof(OptimItem) == 80, "read as five quarters");
    ConstI4 *p = (ConstI4 *)(items + i);
    const i4v a = p[0], b = p[1], c = p[2], d = p[3], e = p[4];
    const auto address = [](int lo, int hi) { return (uint64_t)(uint32_t)hi << 32 | (uint32_t)lo; };
    OptimItem it;
    it.p = (void *)address(a.x, a.y);
    it.g = (const void *)address(a.z, a.w);
    it.m = (void *)address(b.x, b.y);
    it.v = (void *)address(b.z, b.w);
    it.ms = (uint8_t *)address(c.x, c.y);
    it.vs = (uint8_t *)address(c.z, c.w);
    it.base = (int64_t)address(d.x, d.y);
    it.count = d.z;
    it.place = (uint32_t)d.w;
    it.lr = __builtin_bit_cast(float, (int)e.x);
    it.wd = __builtin_bit_cast(float, (int)e.y);
    it.flags = (uint32_t)e.z;
    return it;
}

__device__ __forceinline__ NormItem load_norm_item(const NormItem *items, uint32_t i) {
    static_assert(sizeof(NormItem) == 16, "read at once");
    return __builtin_bit_cast(NormItem, *(ConstI4 *)(items + i));
}

// ---- element types ----------------------------------------------------------

__device__ __forceinline__ float bf16_to_f32(uint32_t b) { return __builtin_bit_cast(float, b << 16); }

// Loads and stores that keep nothing in the caches (ONCE), or ordinary ones.
// (A template over the vector would drop its alignment.)
#define GS_OPTIM_ACCESS(NAME, VALUE, UNALIGNED)                                         \
    template <bool ONCE>                                                                \
    __device__ __forceinline__ VALUE get_##NAME(const void *base, size_t byte) {        \
        Glob<const UNALIGNED> *p = (Glob<const UNALIGNED> *)((const char *)base + byte); \
        return ONCE ? __builtin_nontemporal_load(p) : *p;                               \
    }                                                                                   \
    template <bool ONCE>                                                                \
    __device__ __forceinline__ void put_##NAME(void *base, size_t byte, VALUE x) {      \
        Glob<UNALIGNED> *p = (Glob<UNALIGNED> *)((char *)base + byte);                  \
        if (ONCE)                                                                       \
            __builtin_nontemporal_store(x, p);                                          \
        else                                                                            \
            *p = x;                                                                     \
    }
GS_OPTIM_ACCESS(f4, f4v, f4a)
GS_OPTIM_ACCESS(u4, u4v, u4a)
GS_OPTIM_ACCESS(u2, u2v, u2a)
GS_OPTIM_ACCESS(u1, uint32_t, u1a)
#undef GS_OPTIM_ACCESS

// Four consecutive elements as float32. FAST: all there. Otherwise the first
// k, and zeros (one by one where k < 4).
template <bool BF16, bool FAST, bool ONCE>
__device__ __forceinline__ void load4(const void *base, int i, int k, float x[4]) {
    if (BF16) {
        Glob<const uint16_t> *p = (Glob<const uint16_t> *)base + i;
        if (FAST || k == 4) {
            const u2v q = get_u2<ONCE>(base, 2 * (size_t)i);
            x[0] = bf16_to_f32(q.x & 0xFFFFu);
            x[1] = bf16_to_f32(q.x >> 16);
            x[2] = bf16_to_f32(q.y & 0xFFFFu);
            x[3] = bf16_to_f32(q.y >> 16);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = j < k ? bf16_to_f32(p[j]) : 0.0f;
        }
    } else {
        Glob<const float> *p = (Glob<const float> *)base + i;
        if (FAST || k == 4) {
            const f4v q = get_f4<ONCE>(base, 4 * (size_t)i);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = q[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = j < k ? p[j] : 0.0f;
        }
    }
}

template <bool FAST, bool ONCE>
__device__ __forceinline__ void store4_f32(void *base, int i, int k, const float x[4]) {
    Glob<float> *p = (Glob<float> *)base + i;
    if (FAST || k == 4) {
        put_f4<ONCE>(base, 4 * (size_t)i, f4v{x[0], x[1], x[2], x[3]});
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < k) p[j] = x[j];
    }
}

template <bool FAST, bool ONCE>
__device__ __forceinline__ void store4_bf16(void *base, int i, int k, const uint32_t x[4]) {
    Glob<uint16_t> *p = (Glob<uint16_t> *)base + i;
    if (FAST || k == 4) {
        put_u2<ONCE>(base, 2 * (size_t)i, u2v{x[0] | x[1] << 16, x[2] | x[3] << 16});
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < k) p[j] = (uint16_t)x[j];
    }
}

template <bool FAST, bool ONCE>
__device__ __forceinline__ uint32_t load4_bytes(const void *base, int i, int k) {
    Glob<const uint8_t> *p = (Glob<const uint8_t> *)base + i;
    if (FAST || k == 4) return get_u1<ONCE>(base, (size_t)i);
    uint32_t x = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < k) x |= (uint32_t)p[j] << (8 * j);
    return x;
}

template <bool FAST, bool ONCE>
__device__ __forceinline__ void store4_bytes(void *base, int i, int k, uint32_t x) {
    Glob<uint8_t> *p = (Glob<uint8_t> *)base + i;
    if (FAST || k == 4) {
        put_u1<ONCE>(base, (size_t)i, x);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < k) p[j] = (uint8_t)(x >> (8 * j));
    }
}

// ---- random bits ------------------------------------------------------------

__device__ __forceinline__ uint32_t mix32(uint32_t x) {
    x ^= x >> 16;
    x *= 0x7feb352du;
    x ^= x >> 15;
    x *= 0x846ca68bu;
    return x ^ (x >> 16);
}

// float32 to bfloat16, up with the odds that 16 random bits give; the place
// of infinities is kept, NaN is NaN whatever its payload.
__device__ __forceinline__ uint32_t to_bf16_random(float x, uint32_t r16) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    return x == x ? (b + r16) >> 16 : 0x7FC0u;
}

// ---- MXFP8 ------------------------------------------------------------------

// 2^e of a scale byte as the conversions take it: they use the exponent's 8
// bits alone, whatever the others are, and read 0 as 2^-127.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

__device__ __forceinline__ void decode4(uint32_t codes, float scale, float x[4]) {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, false);
    const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, true);
    x[0] = a[0];
    x[1] = a[1];
    x[2] = b[0];
    x[3] = b[1];
}

// Maximum over the 8 lanes that hold a block of 32.
__device__ __forceinline__ uint32_t block_max(const uint32_t x[4]) {
    uint32_t top = umax_(umax_(x[0], x[1]), umax_(x[2], x[3]));
    top = umax_(top, dpp_u<0xB1>(top));         // lane ^ 1
    top = umax_(top, dpp_u<0x4E>(top));         // lane ^ 2
    return umax_(top, dpp_u<0x141>(top));       // 7 - lane, within 8
}

// The scale byte of a block: the smallest 2^e >= 2^-126 with |x| <= 448 2^e =
// 1.75 2^(e + 8) for its finite values (8 lanes of 4 elements). Sizes are
// compared as float32 bits; what is not finite, and rare, is taken out where
// it is met. A mantissa above 1.75 carries into the exponent.
__device__ __forceinline__ uint32_t block_scale(const float x[4]) {
    uint32_t b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = __builtin_bit_cast(uint32_t, x[j]) & 0x7FFFFFFFu;
    uint32_t top = block_max(b);
    if (top >= 0x7F800000u) {  // all 8 lanes or none
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = b[j] < 0x7F800000u ? b[j] : 0u;
        top = block_max(b);
    }
    const int byte = (int)((top + 0x1FFFFFu) >> 23) - 8;
    return (uint32_t)(byte > 1 ? byte : 1);
}

// Four numbers to E4M3 codes under a scale. The hardware's stochastic
// rounding adds the upper 20 bits of the seed to the 20 bits below the last
// place kept (denormals too), which with the seed k 2^16 + 2^15 is the
// definition's rounding by (k + 1/2) / 2^16. What is not finite becomes NaN.
template <bool HIGH>
__device__ __forceinline__ uint32_t encode4_random(const float x[4], float scale, const uint32_t bits[4]) {
    uint32_t seed[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) seed[j] = HIGH ? (bits[j] & 0xFFFF0000u) | 0x8000u : bits[j] << 16 | 0x8000u;
    int c = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(0, x[0], seed[0], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(c, x[1], seed[1], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(c, x[2], seed[2], scale, 2);
    return (uint32_t)__builtin_amdgcn_cvt_scalef32_sr_fp8_f32(c, x[3], seed[3], scale, 3);
}

// The same to the nearest, ties to even.
__device__ __forceinline__ uint32_t encode4_nearest(const float x[4], float scale) {
    typedef short s2v __attribute__((ext_vector_type(2)));
    s2v c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s2v{0, 0}, x[0], x[1], scale, false);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, x[2], x[3], scale, true);
    return __builtin_bit_cast(uint32_t, c);
}

// s with every positive value at the grid's smallest, 2^-9 of the scale, or
// above (NaN stays).
__device__ __forceinline__ void keep_positive(float s[4], float scale) {
    const float least = scale * 0x1p-9f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float floor = s[j] == 0.0f ? 0.0f : least;
        s[j] = s[j] < floor ? floor : s[j];
    }
}

// ---- AdamW ------------------------------------------------------------------

struct StepConst {
    float b1, a1, b2, a2;  // beta and 1 - beta
    float eps, clip, rate, second, decay;
    uint64_t t, seed;
};

// One element, its moments in float32; s = sqrt(v) is returned for the 8-bit
// form. The root and the reciprocal are the hardware's, good to an ulp: the
// correctly rounded sequences would be half of the arithmetic, and p's own
// rounding is far above them. The root takes denormals for 0, so they are
// scaled first.
__device__ __forceinline__ float adamw1(const StepConst &c, float g, float &p, float &m, float &v) {
    g = g * c.clip;
    m = fmaf_(m, c.b1, g * c.a1);
    v = fmaf_(v, c.b2, g * c.a2 * g);
    const bool tiny = v < 0x1p-126f;
    float s = __builtin_amdgcn_sqrtf(tiny ? v * 0x1p64f : v);
    s = tiny ? s * 0x1p-32f : s;
    const float u = m * __builtin_amdgcn_rcpf(fmaf_(s, c.second, c.eps));
    p = p - fmaf_(c.rate, u, c.decay * p);
    return s;
}

// The part of an element's random bits that an item has in common.
__device__ __forceinline__ uint32_t random_key(const OptimItem &it, const StepConst &c) {
    uint32_t key = mix32(it.place + 0x9e3779b9u);
    key = mix32(key ^ (uint32_t)c.t);
    key = mix32(key ^ (uint32_t)(c.t >> 32));
    key = mix32(key ^ (uint32_t)c.seed);
    key = mix32(key ^ (uint32_t)(c.seed >> 32));
    return mix32(key ^ (uint32_t)((uint64_t)it.base >> 32));
}

// A thread's four elements of a pass: in memory, m and v are four values or
// four codes with the bytes of their block's scales.
template <bool M8>
struct Quad {
    float p[4], g[4], m[4], v[4];
    uint32_t cm, cv, sm, sv;
};

template <bool PB, bool GB, bool M8, bool FAST, bool ONCE>
__device__ __forceinline__ void load_quad(const OptimItem &it, int i, int k, Quad<M8> &q) {
    load4<PB, FAST, ONCE>(it.p, i, k, q.p);
    load4<GB, FAST, ONCE>(it.g, i, k, q.g);
    if (M8) {
        q.cm = load4_bytes<FAST, ONCE>(it.m, i, k);
        q.cv = load4_bytes<FAST, ONCE>(it.v, i, k);
        q.sm = FAST || k > 0 ? ((Glob<const uint8_t> *)it.ms)[i >> 5] : 0u;
        q.sv = FAST || k > 0 ? ((Glob<const uint8_t> *)it.vs)[i >> 5] : 0u;
    } else {
        load4<false, FAST, ONCE>(it.m, i, k, q.m);
        load4<false, FAST, ONCE>(it.v, i, k, q.v);
    }
}

template <bool PB, bool M8, bool FAST, bool ONCE>
__device__ __forceinline__ void step_quad(const OptimItem &it, const StepConst &c, int i, int k, Quad<M8> &q) {
    float s[4];
    uint32_t bits[4];
    const uint32_t key = M8 || PB ? random_key(it, c) : 0u;
    if (M8) {
        decode4(q.cm, scale_of(q.sm), q.m);
        decode4(q.cv, scale_of(q.sv), q.v);
#pragma unroll
        for (int j = 0; j < 4; ++j) q.v[j] = q.v[j] * q.v[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        s[j] = adamw1(c, q.g[j], q.p[j], q.m[j], q.v[j]);
        // i and the item's first element are multiples of 4
        if (M8 || PB) bits[j] = mix32((((uint32_t)it.base + (uint32_t)i) ^ key) ^ (uint32_t)j);
    }
    if (PB) {
        uint32_t b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = to_bf16_random(q.p[j], (bits[j] * 0x9e3779b1u) >> 16);
        store4_bf16<FAST, ONCE>(it.p, i, k, b);
    } else {
        store4_f32<FAST, ONCE>(it.p, i, k, q.p);
    }
    if (M8) {
        if (!FAST) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j >= k) q.m[j] = s[j] = 0.0f;  // no part in the block's scale
        }
        const uint32_t bm = block_scale(q.m), bs = block_scale(s);
        const float scm = scale_of(bm), scs = scale_of(bs);
        keep_positive(s, scs);
        const uint32_t cm = encode4_random<false>(q.m, scm, bits), cs = encode4_random<true>(s, scs, bits);
        store4_bytes<FAST, ONCE>(it.m, i, k, cm);
        store4_bytes<FAST, ONCE>(it.v, i, k, cs);
        if ((threadIdx.x & 7) == 0 && (FAST || k > 0)) {
            ((Glob<uint8_t> *)it.ms)[i >> 5] = (uint8_t)bm;
            ((Glob<uint8_t> *)it.vs)[i >> 5] = (uint8_t)bs;
        }
    } else {
        store4_f32<FAST, ONCE>(it.m, i, k, q.m);
        store4_f32<FAST, ONCE>(it.v, i, k, q.v);
    }
}

// An item is one pass of the workgroup. In a shorter last one the lanes past
// the end stay: those of its last block take part in the block's maximum. Its
// lanes of four elements take vectors as well: 8000 tensors of 2047 elements
// 82 us, 118 one by one (float32; 100 elements each 10.7, 9.0).
template <bool PB, bool GB, bool M8, bool ONCE>
__device__ __forceinline__ void step_item(const OptimItem &it, const StepConst &c) {
    static_assert(kOptimChunk == 4 * kBlock, "an item is four elements a thread");
    const int i = 4 * (int)threadIdx.x;
    Quad<M8> q;
    if (it.count == kOptimChunk) {
        load_quad<PB, GB, M8, true, ONCE>(it, i, 4, q);
        step_quad<PB, M8, true, ONCE>(it, c, i, 4, q);
    } else {
        const int left = it.count - i;
        const int k = left < 4 ? (left > 0 ? left : 0) : 4;
        load_quad<PB, GB, M8, false, false>(it, i, k, q);
        step_quad<PB, M8, false, false>(it, c, i, k, q);
    }
}

// A workgroup an item of 1024 elements, four a thread, so that every array is
// read and written in whole lines, each byte once, and a block of 32 is 8
// lanes; 7 or 8 workgroups a CU hide the loads, and longer items with the
// next pass loaded ahead were no faster (large lists 2 to 15 % slower).
// float32 moments move 22 to 28 bytes an element, 8-bit ones 10 to 16, for
// about 25 and 50 operations. ONCE (steps that move much, by the rule of the
// caller): loads and stores keep nothing. Measured, a step among others:
//   4096 Gaussians (49 k elements)        2.6 us
//   262144 Gaussians (3.1 M)             13.9 us  6.3 TB/s
//   2097152 Gaussians, 8 bits (25 M)     62.8 us  6.5 TB/s
//   48 tensors (267 M), bf16             971 us   6.0 TB/s
//   the same, float32 with 8 bits        693 us   6.2 TB/s
// so large lists run at the memory's rate; what bounds a small one is the
// launch and two trips to memory, the item's record and the elements.
template <bool CONTROL, bool ONCE>
__global__ __launch_bounds__(kBlock) void k_adamw(const OptimItem *items, StepArgs a, const gs_adamw_control *control) {
    OptimItem it = load_item(items, xcd_group<kXcdItems>(blockIdx.x, gridDim.x));
    StepConst c;
    float first = a.first;
    c.second = a.second;
    c.clip = 1.0f;
    c.t = a.step;
    c.seed = a.seed;
    if (CONTROL) {
        typedef __attribute__((address_space(4))) const gs_adamw_control ConstControl;
        ConstControl *now = (ConstControl *)control;
        // A skipped step has nothing to do; a return here would make the
        // item's loads wait for the control's.
        if (!now->apply) it.count = 0;
        c.t = (uint64_t)now->step;
        first = now->first;
        c.second = now->second;
        c.clip = now->clip;
    }
    c.b1 = a.b1;
    c.a1 = a.a1;
    c.b2 = a.b2;
    c.a2 = a.a2;
    c.eps = a.eps;
    const float lr = it.lr * a.lr_scale;
    c.rate = lr * first;
    c.decay = lr * it.wd;
    switch (it.flags & (kParamBf16 | kGradBf16 | kMoments8)) {
        case 0: step_item<false, false, false, ONCE>(it, c); break;
        case kGradBf16: step_item<false, true, false, ONCE>(it, c); break;
        case kParamBf16 | kGradBf16: step_item<true, true, false, ONCE>(it, c); break;
        case kMoments8: step_item<false, false, true, ONCE>(it, c); break;
        case kMoments8 | kGradBf16: step_item<false, true, true, ONCE>(it, c); break;
        case kMoments8 | kParamBf16 | kGradBf16: step_item<true, true, true, ONCE>(it, c); break;
        default: break;
    }
}

// ---- gradient norm ------------------------------------------------------------

template <int CTRL>
__device__ __forceinline__ double dpp_d(double x) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)dpp_u<CTRL>((uint32_t)(b >> 32)) << 32 | dpp_u<CTRL>((uint32_t)b));
}

__device__ __forceinline__ double readlane_d(double x, int lane) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), lane);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)b, lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Sum over the workgroup, in every thread, in a fixed order.
__device__ __forceinline__ double block_sum(double x, double *lds) {
    x += dpp_d<0xB1>(x);
    x += dpp_d<0x4E>(x);
    x += dpp_d<0x124>(x);
    x += dpp_d<0x128>(x);
    x = (readlane_d(x, 0) + readlane_d(x, 16)) + (readlane_d(x, 32) + readlane_d(x, 48));
    if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = x;
    __syncthreads();
    double r = 0.0;
#pragma unroll
    for (int w = 0; w < kWavesPerBlock; ++w) r += lds[w];
    return r;
}

// beta^t by squaring: its error, t 2^-53 of a number that falls as beta^t,
// is far below float32's.
__device__ __forceinline__ double power(double beta, uint64_t t) {
    double r = 1.0;
    for (; t; t >>= 1, beta *= beta)
        if (t & 1) r *= beta;
    return r;
}

template <bool BF16, bool ONCE>
__device__ __forceinline__ void add_squares(const void *g, int i, double sum[4]) {
    const u4v q = get_u4<ONCE>(g, (size_t)i * (BF16 ? 2 : 4));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t w = q[j];
        if (BF16) {
            const double lo = (double)bf16_to_f32(w & 0xFFFFu);
            const double hi = (double)__builtin_bit_cast(float, w & 0xFFFF0000u);
            sum[j] = __builtin_fma(lo, lo, sum[j]);
            sum[j] = __builtin_fma(hi, hi, sum[j]);
        } else {
            const double x = (double)__builtin_bit_cast(float, w);
            sum[j] = __builtin_fma(x, x, sum[j]);
        }
    }
}

template <bool BF16, bool ONCE>
__device__ __forceinline__ void item_squares(const NormItem &it, double sum[4]) {
    constexpr int kEach = BF16 ? 8 : 4, kPass = kEach * kBlock;
    int i = kEach * (int)threadIdx.x;
#pragma unroll 4
    for (const int end = it.count - kEach; i <= end; i += kPass) add_squares<BF16, ONCE>(it.g, i, sum);
    for (; i < it.count; ++i) {  // the last elements, of one thread
        const double x = BF16 ? (double)bf16_to_f32(((Glob<const uint16_t> *)it.g)[i])
                              : (double)((Glob<const float> *)it.g)[i];
        sum[0] = __builtin_fma(x, x, sum[0]);
    }
}

// Leaves a workgroup's sum and returns whether it is the last one to do so.
// Only operations that are carried out at the device's point of coherence:
// the exchange has its answer before the count is touched, so whoever reads
// the full count finds every sum. (A release in its place writes back the
// XCD's whole L2 for each workgroup, 170 ns one after the other.) Counts from
// all XCDs to one word follow each other, so workgroups count in groups and
// the last of each group in the root. Counters are 0 between launches.
__device__ __forceinline__ bool leave_sum(const NormWork &work, double sum) {
    const uint64_t old = __hip_atomic_exchange((uint64_t *)&work.part[blockIdx.x],
                                               __builtin_bit_cast(uint64_t, sum), __ATOMIC_RELAXED,
                                               __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("" ::"v"(old) : "memory");  // the answer is here
    const uint32_t group = blockIdx.x / kNormGroup, groups = (gridDim.x + kNormGroup - 1) / kNormGroup;
    const uint32_t here = group + 1 < groups ? kNormGroup : gridDim.x - group * kNormGroup;
    uint32_t *mine = work.count + (group + 1) * kNormCounter;
    if (__hip_atomic_fetch_add(mine, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != here - 1) return false;
    __hip_atomic_store(mine, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (groups == 1) return true;
    if (__hip_atomic_fetch_add(work.count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != groups - 1) return false;
    __hip_atomic_store(work.count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}

// sqrt(sum g^2): 2 or 4 bytes an element. Squares are added in float64, four
// sums a thread: their range holds any float32 square, so a finite gradient
// never looks infinite, and the additions cost less than the loads. At most
// 2048 workgroups (all that are resident) go over the items, and the last one
// to finish adds their sums, so the norm is one launch. Measured:
//   4096 Gaussians (49 k elements, float32)    5.4 us
//   524288 Gaussians (6.3 M, float32)          9.2 us    2.7 TB/s
//   48 tensors (267 M, bf16)                  84 us      6.3 TB/s
// Small lists are bound by a chain of trips to memory: item, elements, the
// sum's exchange, the count, the sums.
template <bool ONCE>
__global__ __launch_bounds__(kBlock) void k_grad_norm(const NormItem *items, uint32_t n_items, NormWork work,
                                                      NormArgs a, gs_adamw_control *control) {
    __shared__ double lds[2][kWavesPerBlock];
    __shared__ uint64_t coming;
    __shared__ float corrections[2];
    __shared__ uint32_t last;
    double s4[4] = {0.0, 0.0, 0.0, 0.0};
    for (uint32_t i = blockIdx.x; i < n_items; i += gridDim.x) {
        const NormItem it = load_norm_item(items, i);
        if (it.flags & kGradBf16)
            item_squares<true, ONCE>(it, s4);
        else
            item_squares<false, ONCE>(it, s4);
    }
    // Off the way of the sums, the last wave forms what the coming step needs
    // if it is opened.
    if (threadIdx.x == kBlock - 1) {
        coming = (uint64_t)control->step + 1;
        corrections[0] = (float)(1.0 / (1.0 - power(a.beta1, coming)));
    }
    if (threadIdx.x == kBlock - 2)
        corrections[1] = (float)(1.0 / sqrt(1.0 - power(a.beta2, (uint64_t)control->step + 1)));
    double sum = block_sum((s4[0] + s4[1]) + (s4[2] + s4[3]), lds[0]);
    if (threadIdx.x == 0) last = leave_sum(work, sum);
    __syncthreads();
    if (!last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    // The last workgroup to arrive adds the partial sums, in their order.
    sum = 0.0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += kBlock)
        sum += __hip_atomic_load(&work.part[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sum = block_sum(sum, lds[1]);
    if (threadIdx.x != 0) return;
    const double norm = sqrt(sum);
    control->norm = (float)norm;
    const bool finite = sum < __builtin_inf();
    control->apply = finite;
    if (!finite) {
        control->skipped += 1;
        return;
    }
    control->step = (int64_t)coming;
    control->clip = norm > a.max_norm ? (float)(a.max_norm / norm) : 1.0f;
    control->first = corrections[0];
    control->second = corrections[1];
}

// ---- moments through a densification ------------------------------------------

// 32-bit moments: neighbouring lanes take neighbouring elements, since rows
// of 1, 3 or 4 elements that keep their order lie side by side but on no
// vector's boundary. Every lane gets an address inside the arrays, so that no
// load waits on a branch: elements past the end take the last one's, new rows
// row 0's (there is one: n_in > 0). The scheduler may not put the first use
// of a source before the last of their loads: it did, and each load waited
// alone.
__device__ __forceinline__ void carry_f32(const CarryArray &a, uint32_t n_in, Glob<const int32_t> *source, int64_t base,
                                          int count) {
    constexpr int kEach = 4;
    for (int i = (int)threadIdx.x; i < count; i += kEach * kBlock) {
        float m[kEach], v[kEach];
        if (n_in) {
            uint32_t col[kEach], src[kEach];
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const uint32_t e = i + j * kBlock < count ? i + j * kBlock : count - 1;
                const uint32_t q = __umul24(e, a.over) >> 20;  // e / width
                col[j] = e - __umul24(q, a.width);
                src[j] = (uint32_t)source[q];  // negative: past n_in
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const uint64_t at = (uint64_t)(src[j] < n_in ? src[j] : 0u) * a.width + col[j];
                m[j] = ((Glob<const float> *)a.m)[at];
                v[j] = ((Glob<const float> *)a.v)[at];
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                m[j] = src[j] < n_in ? m[j] : 0.0f;
                v[j] = src[j] < n_in ? v[j] : 0.0f;
            }
        } else {
#pragma unroll
            for (int j = 0; j < kEach; ++j) m[j] = v[j] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int e = i + j * kBlock;
            if (e < count) {
                __builtin_nontemporal_store(m[j], (Glob<float> *)a.m_out + base + e);
                __builtin_nontemporal_store(v[j], (Glob<float> *)a.v_out + base + e);
            }
        }
    }
}

// Four bytes of an array of n from byte `at` on, and the scale bytes of block
// i (the low one) and of the next, of n, as far as they are there.
template <typename U>
__device__ __forceinline__ uint32_t four_bytes(const void *base, U at, U n) {
    if (n >= 4) {
        const U b = at < n - 4 ? at : n - 4;
        return get_u1<false>(base, b) >> (8 * (uint32_t)(at - b));
    }
    Glob<const uint8_t> *p = (Glob<const uint8_t> *)base;
    uint32_t x = 0;
    for (int j = 0; j < 3; ++j)
        if (at + j < n) x |= (uint32_t)p[at + j] << (8 * j);
    return x;
}
template <typename U>
__device__ __forceinline__ uint32_t two_scales(const uint8_t *base, U i, U n) {
    if (n < 2) return *(Glob<const uint8_t> *)base;
    const U b = i < n - 2 ? i : n - 2;
    return (uint32_t) * (Glob<const h1a> *)(base + b) >> (8 * (uint32_t)(i - b));
}

// Rows of 8-bit moments into LDS, a word for each element: m's code and scale
// byte, then v's; zeros for new Gaussians. A thread takes up to four elements
// of a row at a time, with one unaligned word of codes and one pair of scales
// a moment, and four such parts at once: single bytes would be four loads an
// element, which keeps the address units busy, and one part at a time leaves
// too little in flight. Reads stay inside the arrays: the few parts from
// which they would not (of the last block, or any of a short array) are read
// with a look at the end. WHOLE: a row is one part; U: 32 bits where the
// input's elements fit.
template <bool WHOLE, typename U>
__device__ __forceinline__ void rows_to_lds(const CarryArray &a, uint32_t n_in, Glob<const int32_t> *source,
                                            uint32_t rows, uint32_t *lds) {
    constexpr int kEach = 4;
    const U n = (U)n_in * a.width, scales = scale_count(n);
    const U inner = scales > 1 ? (scales - 1) * 32 - 3 : 0;  // parts below it have both words whole
    const uint32_t parts = WHOLE ? 1u : (a.width + 3) >> 2, all = rows * parts;
    for (uint32_t p0 = threadIdx.x; p0 < all; p0 += kEach * kBlock) {
        uint32_t row[kEach], col[kEach], src[kEach], cm[kEach], cv[kEach], sm[kEach], sv[kEach], place[kEach];
        U at[kEach];
        bool outer = false;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const uint32_t p = p0 + j * kBlock < all ? p0 + j * kBlock : all - 1;  // the last one several times
            row[j] = WHOLE ? p : __umul24(p, a.over_parts) >> 20;
            col[j] = WHOLE ? 0u : 4 * (p - __umul24(row[j], parts));
            src[j] = (uint32_t)source[row[j]];  // negative: past n_in
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            at[j] = (U)(src[j] < n_in ? src[j] : 0u) * a.width + col[j];
            place[j] = (uint32_t)at[j] & 31u;
            outer |= at[j] >= inner;
        }
        if (__any(outer)) {
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                cm[j] = four_bytes<U>(a.m, at[j], n);
                cv[j] = four_bytes<U>(a.v, at[j], n);
                sm[j] = two_scales<U>(a.m_scale, at[j] >> 5, scales);
                sv[j] = two_scales<U>(a.v_scale, at[j] >> 5, scales);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                cm[j] = get_u1<false>(a.m, at[j]);
                cv[j] = get_u1<false>(a.v, at[j]);
                sm[j] = *(Glob<const h1a> *)(a.m_scale + (at[j] >> 5));
                sv[j] = *(Glob<const h1a> *)(a.v_scale + (at[j] >> 5));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (src[j] >= n_in) cm[j] = cv[j] = 0u;
            // bytes 1 and 3 of a word: the scales of this block, of the next
            const uint32_t first = __builtin_amdgcn_perm(sv[j], sm[j], 0x040C000Cu);
            const uint32_t next = __builtin_amdgcn_perm(sv[j], sm[j], 0x050C010Cu);
            uint32_t *out = lds + __umul24(row[j], a.width) + col[j];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                if (i >= (WHOLE ? a.width : a.width - col[j])) break;
                // bytes 0 and 2: byte i of cm and of cv
                const uint32_t codes = __builtin_amdgcn_perm(cv[j], cm[j], 0x0C040C00u + i * 0x00010001u);
                out[i] = codes | (place[j] + i > 31u ? next : first);
            }
        }
    }
}

// Four elements' words from LDS to codes under new scales.
__device__ __forceinline__ void requantise(const uint32_t w[4], uint32_t &cm, uint32_t &cv, uint32_t &sm,
                                           uint32_t &sv) {
    float m[4], v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        // scales in bits 30 .. 23
        m[j] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[j], __builtin_bit_cast(float, w[j] << 15), false)[0];
        v[j] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[j], __builtin_bit_cast(float, w[j] >> 1), true)[0];
    }
    sm = block_scale(m);
    sv = block_scale(v);
    cm = encode4_nearest(m, scale_of(sm));
    cv = encode4_nearest(v, scale_of(sv));
    // A positive s stays positive: 1 in every byte that was not 0 and is now.
    // Signs are left out (NaN may have one), so that no byte carries into the
    // next.
    const uint32_t was = __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0C0C0602u),
                                               __builtin_amdgcn_perm(w[1], w[0], 0x0C0C0602u), 0x05040100u);
    const auto not_zero = [](uint32_t x) { return (x & 0x7F7F7F7Fu) + 0x7F7F7F7Fu; };  // in bit 7 of each byte
    cv |= (not_zero(was) & ~not_zero(cv)) >> 7 & 0x01010101u;
}

// 8-bit moments: whole rows, a multiple of 32 of them, go through LDS and are
// taken from there as the step takes its elements, four a lane and a block in
// 8 lanes.
__device__ __forceinline__ void carry_mxfp8(const CarryArray &a, uint32_t n_in, Glob<const int32_t> *source,
                                            uint32_t rows, int64_t base, uint32_t *lds) {
    const int count = (int)(rows * a.width);
    if (n_in == 0) {
        for (int i = (int)threadIdx.x; i < count; i += kBlock) lds[i] = 0u;
    } else if ((uint64_t)n_in * a.width >= 0xFFFFFFFFu) {
        rows_to_lds<false, uint64_t>(a, n_in, source, rows, lds);
    } else if (a.width <= 4) {
        rows_to_lds<true, uint32_t>(a, n_in, source, rows, lds);
    } else {
        rows_to_lds<false, uint32_t>(a, n_in, source, rows, lds);
    }
    __syncthreads();
    uint8_t *m_out = (uint8_t *)a.m_out + base, *v_out = (uint8_t *)a.v_out + base;
    uint8_t *m_scale = a.m_scale_out + (base >> 5), *v_scale = a.v_scale_out + (base >> 5);
    const bool writes = (threadIdx.x & 7) == 0;
    int i = 4 * (int)threadIdx.x;
    for (; i < (count & ~31); i += 4 * kBlock) {
        const u4v q = *(const u4v *)(lds + i);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
        uint32_t cm, cv, sm, sv;
        requantise(w, cm, cv, sm, sv);
        put_u1<true>(m_out, i, cm);
        put_u1<true>(v_out, i, cv);
        if (writes) {
            ((Glob<uint8_t> *)m_scale)[i >> 5] = (uint8_t)sm;
            ((Glob<uint8_t> *)v_scale)[i >> 5] = (uint8_t)sv;
        }
    }
    if (i < count + 31) {  // the last block, if it is a shorter one: all its lanes, as in the step
        const int left = count - i;
        const int k = left < 4 ? (left > 0 ? left : 0) : 4;
        uint32_t w[4], cm, cv, sm, sv;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = j < k ? lds[i + j] : 0u;
        requantise(w, cm, cv, sm, sv);
        store4_bytes<false, false>(m_out, i, k, cm);
        store4_bytes<false, false>(v_out, i, k, cv);
        if (writes && k > 0) {
            ((Glob<uint8_t> *)m_scale)[i >> 5] = (uint8_t)sm;
            ((Glob<uint8_t> *)v_scale)[i >> 5] = (uint8_t)sv;
        }
    }
}

// Rows of all arrays through the source map in one launch, a workgroup some
// rows of one array. 16 bytes an element with float32 moments, 4 with 8-bit
// ones, and the map. The outputs keep nothing in the caches: what is carried
// is read once, and the inputs of neighbouring workgroups share lines (2 M
// Gaussians with 8-bit moments take 1.28 times as long with ordinary stores,
// 1.25 with loads that keep nothing). Measured, a tenth pruned and a fifth
// added:
//   262144 Gaussians, float32 moments     9.7 us  5.3 TB/s
//   2097152 Gaussians, 8-bit moments     33 us    3.5 TB/s of what is needed
// The 8-bit form reads 98 MB and writes 57 for the 113 that it needs, most of
// the rest the map, which the workgroups of each array read again: 4.7 TB/s,
// near a copy's rate. Its arithmetic (32 operations an element) takes no time
// beside that.
__global__ __launch_bounds__(kBlock) void k_carry(CarryArgs a, const int32_t *source) {
    __shared__ alignas(16) uint32_t lds[kCarryMost];
    const uint32_t block = a.block0 + xcd_group<kXcdItems>(blockIdx.x, gridDim.x);
    int k = 0;
#pragma unroll
    for (int j = 1; j < GS_ADAMW_ROWS_MAX; ++j) k = block >= a.first[j] ? j : k;
    const CarryArray r = a.rows[k];
    const int64_t row0 = (int64_t)(block - a.first[k]) * r.rows, left = a.n_out - row0;
    const uint32_t rows = left < r.rows ? (uint32_t)left : r.rows;
    const int64_t base = row0 * r.width;
    Glob<const int32_t> *from = (Glob<const int32_t> *)source + row0;
    if (r.moments8)
        carry_mxfp8(r, (uint32_t)a.n_in, from, rows, base, lds);
    else
        carry_f32(r, (uint32_t)a.n_in, from, base, (int)(rows * r.width));
}

}  // namespace

// ---- host -----------------------------------------------------------------------

hipError_t launch_plan_adamw(const gs_adamw_tensor *tensors, int64_t count, OptimItem *items, NormItem *norms,
                             const NormWork &work, hipStream_t s) {
    const hipError_t e0 = fill_u32(work.count, 0u, kNormCounters * kNormCounter, s);
    if (e0 != hipSuccess) return e0;
    FillArgs a;
    uint64_t done = 0, done_norm = 0;
    int64_t i = 0;
    while (i < count) {
        a.count = 0;
        uint64_t here = 0, here_norm = 0;
        // A tensor's pieces stay in one launch; a launch takes tensors while
        // their pieces fit 31 bits.
        while (i < count && a.count < kFill) {
            const gs_adamw_tensor &t = tensors[i];
            const uint64_t pieces = t.param ? (uint64_t)optim_items(t.n) : 0;
            const uint64_t norm_pieces = (uint64_t)norm_items(t.n);
            if (a.count && here + pieces > 0x7FFFFFFFu) break;
            if (norm_pieces) {
                OptimTensor &o = a.t[a.count];
                o.p = t.param;
                o.g = t.grad;
                o.m = t.m;
                o.v = t.v;
                o.ms = t.moments == GS_MOMENTS_MXFP8 ? t.m_scale : nullptr;
                o.vs = t.moments == GS_MOMENTS_MXFP8 ? t.v_scale : nullptr;
                o.n = t.n;
                o.place = (uint32_t)i;
                o.flags = optim_flags(t);
                o.lr = t.lr;
                o.wd = t.weight_decay;
                a.first[a.count] = (uint32_t)here;
                a.first_norm[a.count++] = (uint32_t)here_norm;
                here += pieces;
                here_norm += norm_pieces;
            }
            ++i;
        }
        if (!a.count) break;
        a.first[a.count] = (uint32_t)here;
        a.first_norm[a.count] = (uint32_t)here_norm;
        const uint64_t most = here > here_norm ? here : here_norm;
        prof_begin("adamw_plan", s);
        hipLaunchKernelGGL(k_fill_items, dim3((uint32_t)((most + kBlock - 1) / kBlock)), dim3(kBlock), 0, s, a,
                           items + done, norms + done_norm);
        prof_end("adamw_plan", s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        done += here;
        done_norm += here_norm;
    }
    return hipSuccess;
}

hipError_t launch_grad_norm(const NormItem *items, int64_t n_items, bool once, const NormWork &work, const NormArgs &a,
                            gs_adamw_control *control, hipStream_t s) {
    const uint32_t blocks = (uint32_t)(n_items < 1 ? 1 : n_items < kNormBlocks ? n_items : kNormBlocks);
    prof_begin("grad_norm", s);
    const auto kernel = once ? k_grad_norm<true> : k_grad_norm<false>;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kBlock), 0, s, items, (uint32_t)n_items, work, a, control);
    prof_end("grad_norm", s);
    return hipGetLastError();
}

hipError_t launch_adamw(const OptimItem *items, int64_t n_items, bool once, const StepArgs &a,
                        const gs_adamw_control *control, hipStream_t s) {
    for (int64_t i = 0; i < n_items; i += kMaxGrid) {
        const int64_t here = n_items - i < kMaxGrid ? n_items - i : kMaxGrid;
        prof_begin("adamw", s);
        const auto kernel = control ? (once ? k_adamw<true, true> : k_adamw<true, false>)
                                    : (once ? k_adamw<false, true> : k_adamw<false, false>);
        hipLaunchKernelGGL(kernel, dim3((uint32_t)here), dim3(kBlock), 0, s, items + i, a, control);
        prof_end("adamw", s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_adamw_carry(const gs_adamw_rows *arrays, int count, int64_t n_in, const int32_t *source,
                              int64_t n_out, hipStream_t s) {
    CarryArgs a;
    a.n_in = n_in;
    a.n_out = n_out;
    uint32_t blocks = 0;
    for (int k = 0; k < GS_ADAMW_ROWS_MAX; ++k) {
        a.first[k] = k < count ? blocks : 0xFFFFFFFFu;
        CarryArray &o = a.rows[k];
        o = CarryArray();
        if (k >= count) continue;
        const gs_adamw_rows &r = arrays[k];
        o.m = r.m;
        o.v = r.v;
        o.m_scale = r.m_scale;
        o.v_scale = r.v_scale;
        o.m_out = r.m_out;
        o.v_out = r.v_out;
        o.m_scale_out = r.m_scale_out;
        o.v_scale_out = r.v_scale_out;
        o.width = (uint32_t)r.width;
        o.over = ((1u << 20) + o.width - 1) / o.width;
        o.over_parts = ((1u << 20) + (o.width + 3) / 4 - 1) / ((o.width + 3) / 4);
        o.rows = carry_rows(o.width, r.moments == GS_MOMENTS_MXFP8);
        o.moments8 = r.moments == GS_MOMENTS_MXFP8;
        blocks += (uint32_t)((n_out + o.rows - 1) / o.rows);
    }
    for (uint32_t b = 0; b < blocks; b += (uint32_t)kMaxGrid) {
        const uint32_t here = blocks - b < (uint32_t)kMaxGrid ? blocks - b : (uint32_t)kMaxGrid;
        a.block0 = b;
        prof_begin("adamw_carry", s);
        hipLaunchKernelGGL(k_carry, dim3(here), dim3(kBlock), 0, s, a, source);
        prof_end("adamw_carry", s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace gs
