// The optimiser step (include/gs_optim.h): AdamW over a list of tensors with
// float32 or MXFP8 moments, the global gradient norm, and moments through a
// densification's source map.
//
// Everything is elementwise or a sum, and bound by HBM. A list is cut into
// pieces ("items") of at most one workgroup's work, and one launch covers
// all tensors: a workgroup reads its item's record (addresses, length, rates)
// with scalar loads and needs nothing else of the list.
#include "optim.h"

#include <cmath>

namespace gs {
namespace {

template <typename T>
using Glob = __attribute__((address_space(1))) T;  // global, not generic, addresses
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));

constexpr int kFill = 24;         // tensors whose pieces one launch of k_fill_items writes
constexpr int64_t kMaxGrid = 1 << 23;  // workgroups of a launch at most: 2^31 threads
constexpr int kNormBlocks = 1024; // workgroups of the norm at most: one partial sum each

struct FillArgs {
    OptimTensor t[kFill];
    uint32_t first[kFill + 1];  // first item of each, counted from the launch's first
    int count;
};

// ---- items ----------------------------------------------------------------

__global__ __launch_bounds__(kBlock) void k_fill_items(FillArgs a, OptimItem *items) {
    const uint32_t i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= a.first[a.count]) return;
    int k = 0;
    while (i >= a.first[k + 1]) ++k;
    const OptimTensor t = a.t[k];
    const int64_t base = (int64_t)(i - a.first[k]) * kOptimChunk;
    const int64_t left = t.n - base;
    OptimItem it;
    const int ps = t.flags & kParamBf16 ? 2 : 4, gs = t.flags & kGradBf16 ? 2 : 4, ms = t.flags & kMoments8 ? 1 : 4;
    it.p = t.p ? (char *)t.p + base * ps : nullptr;
    it.g = (const char *)t.g + base * gs;
    it.m = t.m ? (char *)t.m + base * ms : nullptr;
    it.v = t.v ? (char *)t.v + base * ms : nullptr;
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

__device__ __forceinline__ OptimItem load_item(const OptimItem *items, uint32_t i) {
    static_assert(sizeof(OptimItem) == 80, "read as five quarters");
    union {
        i4v q[5];
        OptimItem it;
    } u;
    ConstI4 *p = (ConstI4 *)(items + i);
#pragma unroll
    for (int k = 0; k < 5; ++k) u.q[k] = p[k];
    return u.it;
}

// ---- element types ----------------------------------------------------------

__device__ __forceinline__ float bf16_to_f32(uint32_t b) { return __builtin_bit_cast(float, b << 16); }

// Four consecutive elements, of which k are there, as float32 bits. Vector
// loads where the arrays allow them, single ones elsewhere.
template <bool BF16>
__device__ __forceinline__ void load4(const void *base, int i, int k, bool vec, float x[4]) {
    if (BF16) {
        Glob<const uint16_t> *p = (Glob<const uint16_t> *)base + i;
        if (vec && k == 4) {
            const u2v q = *(Glob<const u2v> *)p;
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
        if (vec && k == 4) {
            const f4v q = *(Glob<const f4v> *)p;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = q[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = j < k ? p[j] : 0.0f;
        }
    }
}

__device__ __forceinline__ void store4_f32(void *base, int i, int k, bool vec, const float x[4]) {
    Glob<float> *p = (Glob<float> *)base + i;
    if (vec && k == 4) {
        *(Glob<f4v> *)p = f4v{x[0], x[1], x[2], x[3]};
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < k) p[j] = x[j];
    }
}

__device__ __forceinline__ uint32_t load4_bytes(const void *base, int i, int k, bool vec) {
    Glob<const uint8_t> *p = (Glob<const uint8_t> *)base + i;
    if (vec && k == 4) return *(Glob<const uint32_t> *)p;
    uint32_t x = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < k) x |= (uint32_t)p[j] << (8 * j);
    return x;
}

__device__ __forceinline__ void store4_bytes(void *base, int i, int k, bool vec, uint32_t x) {
    Glob<uint8_t> *p = (Glob<uint8_t> *)base + i;
    if (vec && k == 4) {
        *(Glob<uint32_t> *)p = x;
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

// 2^e of a scale byte (byte 0 is 2^-127, a float32 denormal).
__device__ __forceinline__ float scale_of(uint32_t byte) {
    return __builtin_bit_cast(float, umax_(byte << 23, 0x400000u));
}

__device__ __forceinline__ void decode4(uint32_t codes, float scale, float x[4]) {
    typedef float f2v __attribute__((ext_vector_type(2)));
    const f2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false);
    const f2v b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    x[0] = a.x * scale;
    x[1] = a.y * scale;
    x[2] = b.x * scale;
    x[3] = b.y * scale;
}

// The largest finite |x| of a block, as float32 bits: 8 lanes of 4 elements.
__device__ __forceinline__ uint32_t block_top(const float x[4]) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t b = __builtin_bit_cast(uint32_t, x[j]) & 0x7FFFFFFFu;
        top = umax_(top, b < 0x7F800000u ? b : 0u);
    }
    top = umax_(top, dpp_u<0xB1>(top));   // lane ^ 1
    top = umax_(top, dpp_u<0x4E>(top));   // lane ^ 2
    top = umax_(top, dpp_u<0x141>(top));  // 7 - lane, within 8
    return top;
}

// Scale byte of a block with this top: the smallest 2^e >= 2^-126 with
// top <= 448 2^e = 1.75 2^(e + 8). A mantissa above 1.75 carries.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const int s = (int)((top + 0x1FFFFFu) >> 23) - 8;
    return (uint32_t)(s > 1 ? s : 1);
}

// |x| to E4M3 under a scale. x 2^-e 2^-120 puts E4M3's exponent range on
// float32's lowest exponents, denormals on denormals, so the code is the top
// of the float32 bits with 20 bits below it, and `r` of those is added to
// round (2^20 r is the odds of the next code). What is not finite gives 0x7F,
// E4M3's NaN.
__device__ __forceinline__ uint32_t encode1(float x, float inv, uint32_t r) {
    const float y = __builtin_fabsf(x) * inv * 0x1p-120f;
    const uint32_t c = (__builtin_bit_cast(uint32_t, y) + r) >> 20;
    return c < 0x7Fu ? c : 0x7Fu;
}

__device__ __forceinline__ float inverse_scale(uint32_t byte) {
    return __builtin_bit_cast(float, (254u - byte) << 23);
}

__device__ __forceinline__ uint32_t nearest_bits(float x, float inv) {
    const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_fabsf(x) * inv * 0x1p-120f);
    return 0x7FFFFu + ((b >> 20) & 1u);
}

__device__ __forceinline__ uint32_t sign_bit8(float x) { return (__builtin_bit_cast(uint32_t, x) >> 24) & 0x80u; }

// ---- AdamW ------------------------------------------------------------------

struct StepConst {
    float b1, a1, b2, a2;  // beta and 1 - beta
    float eps, clip, rate, second, decay;
    uint32_t key;
};

// One element, its moments in float32; s = sqrt(v) is returned for the 8-bit
// form.
__device__ __forceinline__ float adamw1(const StepConst &c, float g, float &p, float &m, float &v) {
    g = g * c.clip;
    m = m * c.b1 + g * c.a1;
    v = v * c.b2 + g * c.a2 * g;
    const float s = sqrtf(v);
    p = p - (c.rate * (m / (s * c.second + c.eps)) + c.decay * p);
    return s;
}

template <bool PB, bool GB, bool M8>
__device__ __forceinline__ void step_item(const OptimItem &it, const StepConst &c) {
    const bool vec = it.flags & kVectors;
    for (int i = 4 * (int)threadIdx.x; i < it.count + 31; i += 4 * kBlock) {  // whole blocks of lanes
        const int left = it.count - i;
        const int k = left < 4 ? (left > 0 ? left : 0) : 4;
        float p[4], g[4], m[4], v[4], s[4];
        uint32_t bits[4];
        load4<PB>(it.p, i, k, vec, p);
        load4<GB>(it.g, i, k, vec, g);
        if (M8) {
            const uint32_t cm = load4_bytes(it.m, i, k, vec), cv = load4_bytes(it.v, i, k, vec);
            const float sm = k > 0 ? scale_of(((Glob<const uint8_t> *)it.ms)[i >> 5]) : 0.0f;
            const float sv = k > 0 ? scale_of(((Glob<const uint8_t> *)it.vs)[i >> 5]) : 0.0f;
            decode4(cm, sm, m);
            decode4(cv, sv, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = v[j] * v[j];
        } else {
            load4<false>(it.m, i, k, vec, m);
            load4<false>(it.v, i, k, vec, v);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s[j] = adamw1(c, g[j], p[j], m[j], v[j]);
            if (M8 || PB) bits[j] = mix32(((uint32_t)it.base + (uint32_t)(i + j)) ^ c.key);
        }
        if (PB) {
            uint32_t q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] = to_bf16_random(p[j], (bits[j] * 0x9e3779b1u) >> 16);
            Glob<uint16_t> *out = (Glob<uint16_t> *)it.p + i;
            if (vec && k == 4) {
                *(Glob<u2v> *)out = u2v{q[0] | q[1] << 16, q[2] | q[3] << 16};
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < k) out[j] = (uint16_t)q[j];
            }
        } else {
            store4_f32(it.p, i, k, vec, p);
        }
        if (M8) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j >= k) m[j] = s[j] = 0.0f;  // no part in the block's scale
            const uint32_t bm = scale_byte(block_top(m)), bs = scale_byte(block_top(s));
            const float im = inverse_scale(bm), is = inverse_scale(bs);
            uint32_t cm = 0, cs = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = encode1(m[j], im, (bits[j] & 0xFFFFu) * 16u + 8u);
                const uint32_t b = encode1(s[j], is, (bits[j] >> 16) * 16u + 8u);
                cm |= (a | sign_bit8(m[j])) << (8 * j);
                cs |= (s[j] > 0.0f ? umax_(b, 1u) : b) << (8 * j);
            }
            if (k > 0) {
                store4_bytes(it.m, i, k, vec, cm);
                store4_bytes(it.v, i, k, vec, cs);
                if ((threadIdx.x & 7) == 0) {
                    ((Glob<uint8_t> *)it.ms)[i >> 5] = (uint8_t)bm;
                    ((Glob<uint8_t> *)it.vs)[i >> 5] = (uint8_t)bs;
                }
            }
        } else {
            store4_f32(it.m, i, k, vec, m);
            store4_f32(it.v, i, k, vec, v);
        }
    }
}

__global__ __launch_bounds__(kBlock) void k_adamw(const OptimItem *items, StepArgs a, const gs_adamw_control *control) {
    const OptimItem it = load_item(items, blockIdx.x);
    StepConst c;
    uint64_t t = a.step;
    float first = a.first;
    c.second = a.second;
    c.clip = 1.0f;
    if (control) {
        if (!control->apply) return;
        t = (uint64_t)control->step;
        first = control->first;
        c.second = control->second;
        c.clip = control->clip;
    }
    c.b1 = a.b1;
    c.a1 = a.a1;
    c.b2 = a.b2;
    c.a2 = a.a2;
    c.eps = a.eps;
    const float lr = it.lr * a.lr_scale;
    c.rate = lr * first;
    c.decay = lr * it.wd;
    uint32_t key = mix32(it.place + 0x9e3779b9u);
    key = mix32(key ^ (uint32_t)t);
    key = mix32(key ^ (uint32_t)(t >> 32));
    key = mix32(key ^ (uint32_t)a.seed);
    key = mix32(key ^ (uint32_t)(a.seed >> 32));
    c.key = mix32(key ^ (uint32_t)((uint64_t)it.base >> 32));
    switch (it.flags & (kParamBf16 | kGradBf16 | kMoments8)) {
        case 0: step_item<false, false, false>(it, c); break;
        case kGradBf16: step_item<false, true, false>(it, c); break;
        case kParamBf16 | kGradBf16: step_item<true, true, false>(it, c); break;
        case kMoments8: step_item<false, false, true>(it, c); break;
        case kMoments8 | kGradBf16: step_item<false, true, true>(it, c); break;
        case kMoments8 | kParamBf16 | kGradBf16: step_item<true, true, true>(it, c); break;
        default: break;
    }
}

// ---- gradient norm ------------------------------------------------------------

__device__ __forceinline__ double block_sum(double x, double *lds) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
    if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = x;
    __syncthreads();
    double r = 0.0;
#pragma unroll
    for (int w = 0; w < kWavesPerBlock; ++w) r += lds[w];
    return r;
}

template <bool BF16>
__device__ __forceinline__ double item_squares(const OptimItem &it) {
    double sum = 0.0;
    for (int i = 4 * (int)threadIdx.x; i < it.count; i += 4 * kBlock) {
        const int left = it.count - i;
        float g[4];
        load4<BF16>(it.g, i, left < 4 ? left : 4, it.flags & kVectors, g);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum = __builtin_fma((double)g[j], (double)g[j], sum);
    }
    return sum;
}

__global__ __launch_bounds__(kBlock) void k_grad_norm(const OptimItem *items, uint32_t n_items, double *part,
                                                      NormArgs a, gs_adamw_control *control) {
    __shared__ double lds[2][kWavesPerBlock];
    __shared__ uint32_t last;
    double sum = 0.0;
    for (uint32_t i = blockIdx.x; i < n_items; i += gridDim.x) {
        const OptimItem it = load_item(items, i);
        sum += it.flags & kGradBf16 ? item_squares<true>(it) : item_squares<false>(it);
    }
    sum = block_sum(sum, lds[0]);
    if (threadIdx.x == 0) {
        __hip_atomic_store(&part[blockIdx.x], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = __hip_atomic_fetch_add(&control->arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) ==
               gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    // The last workgroup to arrive adds the partial sums, in their order.
    sum = 0.0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += kBlock)
        sum += __hip_atomic_load(&part[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sum = block_sum(sum, lds[1]);
    if (threadIdx.x != 0) return;
    const double norm = sqrt(sum);
    control->arrived = 0;
    control->norm = (float)norm;
    const bool finite = sum < __builtin_inf();
    control->apply = finite;
    if (!finite) {
        control->skipped += 1;
        return;
    }
    const int64_t t = control->step + 1;
    control->step = t;
    control->clip = norm > a.max_norm ? (float)(a.max_norm / norm) : 1.0f;
    control->first = (float)(1.0 / (1.0 - pow(a.beta1, (double)t)));
    control->second = (float)(1.0 / sqrt(1.0 - pow(a.beta2, (double)t)));
}

// ---- moments through a densification ------------------------------------------

template <bool M8>
__device__ __forceinline__ void carry_rows(const gs_adamw_rows &a, int64_t n_in, Glob<const int32_t> *source,
                                           int64_t total, int64_t base) {
    const int64_t row0 = base / a.width;
    const uint32_t col0 = (uint32_t)(base - row0 * a.width);
    const int64_t e0 = base + 4 * (int)threadIdx.x;
    float m[4], v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        m[j] = v[j] = 0.0f;
        if (e0 + j >= total) continue;
        const uint32_t x = col0 + 4 * threadIdx.x + j, q = x / (uint32_t)a.width;
        const int64_t src = source[row0 + q];
        if (src < 0 || src >= n_in) continue;
        const int64_t at = src * a.width + (x - q * (uint32_t)a.width);
        if (M8) {
            float t[4];
            decode4(((Glob<const uint8_t> *)a.m)[at], scale_of(((Glob<const uint8_t> *)a.m_scale)[at >> 5]), t);
            m[j] = t[0];
            decode4(((Glob<const uint8_t> *)a.v)[at], scale_of(((Glob<const uint8_t> *)a.v_scale)[at >> 5]), t);
            v[j] = t[0];
        } else {
            m[j] = ((Glob<const float> *)a.m)[at];
            v[j] = ((Glob<const float> *)a.v)[at];
        }
    }
    const int64_t left = total - e0;
    const int k = left < 4 ? (left > 0 ? (int)left : 0) : 4;
    if (M8) {
        const uint32_t bm = scale_byte(block_top(m)), bs = scale_byte(block_top(v));
        const float im = inverse_scale(bm), is = inverse_scale(bs);
        uint32_t cm = 0, cs = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t p = encode1(m[j], im, nearest_bits(m[j], im));
            const uint32_t q = encode1(v[j], is, nearest_bits(v[j], is));
            cm |= (p | sign_bit8(m[j])) << (8 * j);
            cs |= (v[j] > 0.0f ? umax_(q, 1u) : q) << (8 * j);
        }
        if (k > 0) {
            store4_bytes((uint8_t *)a.m_out + e0, 0, k, false, cm);
            store4_bytes((uint8_t *)a.v_out + e0, 0, k, false, cs);
            if ((threadIdx.x & 7) == 0) {
                ((Glob<uint8_t> *)a.m_scale_out)[e0 >> 5] = (uint8_t)bm;
                ((Glob<uint8_t> *)a.v_scale_out)[e0 >> 5] = (uint8_t)bs;
            }
        }
    } else {
        store4_f32((float *)a.m_out + e0, 0, k, false, m);
        store4_f32((float *)a.v_out + e0, 0, k, false, v);
    }
}

__global__ __launch_bounds__(kBlock) void k_carry(CarryArgs a, const int32_t *source) {
    const uint32_t block = a.block0 + blockIdx.x;
    int k = 0;
    while (block >= a.first[k + 1]) ++k;
    const gs_adamw_rows r = a.rows[k];
    const int64_t base = (int64_t)(block - a.first[k]) * kCarryChunk;
    const int64_t total = a.n_out * r.width;
    if (r.moments == GS_MOMENTS_MXFP8)
        carry_rows<true>(r, a.n_in, (Glob<const int32_t> *)source, total, base);
    else
        carry_rows<false>(r, a.n_in, (Glob<const int32_t> *)source, total, base);
}

}  // namespace

// ---- host -----------------------------------------------------------------------

size_t optim_part_bytes() { return kNormBlocks * sizeof(double); }

hipError_t launch_plan_adamw(const gs_adamw_tensor *tensors, int64_t count, OptimItem *items, hipStream_t s) {
    FillArgs a;
    uint64_t done = 0;
    int64_t i = 0;
    while (i < count) {
        a.count = 0;
        uint64_t here = 0;
        // A tensor's pieces stay in one launch; a launch takes tensors while
        // their pieces fit 31 bits.
        while (i < count && a.count < kFill) {
            const gs_adamw_tensor &t = tensors[i];
            const uint64_t pieces = (uint64_t)optim_items(t.n);
            if (a.count && here + pieces > 0x7FFFFFFFu) break;
            if (pieces) {
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
                a.first[a.count++] = (uint32_t)here;
                here += pieces;
            }
            ++i;
        }
        if (!a.count) break;
        a.first[a.count] = (uint32_t)here;
        prof_begin("adamw_plan", s);
        hipLaunchKernelGGL(k_fill_items, dim3((uint32_t)((here + kBlock - 1) / kBlock)), dim3(kBlock), 0, s, a,
                           items + done);
        prof_end("adamw_plan", s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        done += here;
    }
    return hipSuccess;
}

hipError_t launch_grad_norm(const OptimItem *items, int64_t n_items, double *part, const NormArgs &a,
                            gs_adamw_control *control, hipStream_t s) {
    const uint32_t blocks = (uint32_t)(n_items < 1 ? 1 : n_items < kNormBlocks ? n_items : kNormBlocks);
    prof_begin("grad_norm", s);
    hipLaunchKernelGGL(k_grad_norm, dim3(blocks), dim3(kBlock), 0, s, items, (uint32_t)n_items, part, a, control);
    prof_end("grad_norm", s);
    return hipGetLastError();
}

hipError_t launch_adamw(const OptimItem *items, int64_t n_items, const StepArgs &a, const gs_adamw_control *control,
                        hipStream_t s) {
    for (int64_t i = 0; i < n_items; i += kMaxGrid) {
        const int64_t here = n_items - i < kMaxGrid ? n_items - i : kMaxGrid;
        prof_begin("adamw", s);
        hipLaunchKernelGGL(k_adamw, dim3((uint32_t)here), dim3(kBlock), 0, s, items + i, a, control);
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
    for (int k = 0; k < count; ++k) {
        a.rows[k] = arrays[k];
        a.first[k] = blocks;
        blocks += (uint32_t)((n_out * arrays[k].width + kCarryChunk - 1) / kCarryChunk);
    }
    a.first[count] = blocks;
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
