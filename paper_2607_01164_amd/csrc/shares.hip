// The attention weight that every Gaussian gets from a batch of queries
// (include/gs_budget.h): score_i <- decay score_i + w_i sum_t f_t G_i(p_t).
//
// A lane takes a row of a Gaussian's queries: for grids a row of voxels at
// fixed (y, z), for ordered queries a row of cells, a run of the plan's order,
// both cut to the cutoff ellipsoid as the backward cuts them. Along a row of
// voxels only u0 = U00 dx + c changes, so a pair costs a subtraction, two
// FMAs, the test, one v_exp_f32 and an FMA; there is no search for the row of
// an element, which costs more than the pair itself (the backward's walk, a
// lane an element, has to do it for its longer pairs). A wave takes the rows
// of a few Gaussians, 64 at a time, and adds each Gaussian's lanes with a
// segmented scan: no atomics, an order fixed by the inputs.
#include "budget.h"

#pragma clang fp contract(off)

namespace gs {
namespace {

// Gaussians of a wave (consecutive in gorder), so that their rows fill its
// lanes; one a wave where there are too few to fill the chip otherwise.
constexpr uint32_t kPack = 4;
constexpr int64_t kPackMinGauss = 65536;
constexpr uint32_t kXcdWaves = 4;
// waves of one launch (a launch has fewer than 2^32 threads)
constexpr uint64_t kWavesMost = (uint64_t)1 << 25;

// f of a query: its gain over I, 0 where the field is undefined.
__device__ __forceinline__ float query_factor(const float *influence, const float *gain, int64_t t) {
    const float I = influence[t];
    if (!(I > 0.0f)) return 0.0f;
    return (gain ? gain[t] : 1.0f) / I;
}

__global__ __launch_bounds__(kBlock) void k_shares_stage_grid(int64_t n, const float *__restrict__ influence,
                                                              const float *__restrict__ gain, float *__restrict__ f) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i < n) f[i] = query_factor(influence, gain, i);
}

__global__ __launch_bounds__(kBlock) void k_shares_stage_plan(int64_t n, const uint32_t *__restrict__ order,
                                                              const float4 *__restrict__ pos,
                                                              const float *__restrict__ influence,
                                                              const float *__restrict__ gain,
                                                              float4 *__restrict__ pts) {
    const int64_t k = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (k >= n) return;
    const float4 p = pos[k];
    pts[k] = make_float4(p.x, p.y, p.z, query_factor(influence, gain, order[k]));
}

// Q <= 2 ln(1/tau) from the parameters themselves, in float64.
__device__ __forceinline__ bool within_exact(const SharesExact &x, uint32_t gid, float px, float py, float pz) {
    const float *m = x.mean + 3 * (size_t)gid, *s = x.scale + 3 * (size_t)gid, *q = x.rot + 4 * (size_t)gid;
    const double q0 = q[0], q1 = q[1], q2 = q[2], q3 = q[3];
    const double iq = 1.0 / sqrt(q0 * q0 + q1 * q1 + q2 * q2 + q3 * q3);
    const double w = q0 * iq, a = q1 * iq, b = q2 * iq, c = q3 * iq;
    const double dx = (double)px - m[0], dy = (double)py - m[1], dz = (double)pz - m[2];
    const double u0 = (1.0 - 2.0 * (b * b + c * c)) * dx + 2.0 * (a * b + w * c) * dy + 2.0 * (a * c - w * b) * dz;
    const double u1 = 2.0 * (a * b - w * c) * dx + (1.0 - 2.0 * (a * a + c * c)) * dy + 2.0 * (b * c + w * a) * dz;
    const double u2 = 2.0 * (a * c + w * b) * dx + 2.0 * (b * c - w * a) * dy + (1.0 - 2.0 * (a * a + b * b)) * dz;
    const double e0 = u0 / s[0], e1 = u1 / s[1], e2 = u2 / s[2];
    return e0 * e0 + e1 * e1 + e2 * e2 <= x.cut;
}

// How far the float32 Q' may be off near the cutoff T. The entries of U and
// of d = p - mu are rounded once, u's sums at most three times, so |du| <=
// 5 2^-24 |U| |d| summed by components, at most sqrt(3) kappa |u| 5 2^-24 with
// kappa the largest scale over the smallest; twice |u| |du| and the three
// roundings of |u|^2 stay below 2^-19 kappa Q'.
__device__ __forceinline__ float cutoff_margin(const SharesExact &x, uint32_t gid, float T) {
    const float *s = x.scale + 3 * (size_t)gid;
    const float hi = fmaxf(fmaxf(s[0], s[1]), s[2]), lo = fminf(fminf(s[0], s[1]), s[2]);
    return hi / lo * 0x1p-19f * T;
}

struct SharesArgs {
    QueryParams q;
    GridParams g;
    BwdGeom bg;
    const Record *rec;
    const CellBox *box;
    const uint32_t *gorder;
    int64_t n_gauss;
    const uint32_t *point_off;
    const float4 *pts;
    const float *f;
    SharesExact exact;
    float T, decay;
    float *score;
    uint32_t pack;
    uint64_t wave0;  // the launch's first wave
};

template <bool GRID>
__global__ __launch_bounds__(kWave) void k_shares(SharesArgs a) {
    const uint32_t lane = threadIdx.x;
    const uint64_t first = (a.wave0 + xcd_group<kXcdWaves>(blockIdx.x, gridDim.x)) * a.pack;
    if (first >= (uint64_t)a.n_gauss) return;
    const uint32_t nk = (uint64_t)a.n_gauss - first < a.pack ? (uint32_t)((uint64_t)a.n_gauss - first) : a.pack;
    const float T = a.T;
    // lane i < nk describes Gaussian i of the wave: its rows
    uint32_t mgid = 0, mR = 0, mnx = 0, mny = 1, mx = 0, my = 0, mz = 0;
    if (lane < nk) {
        mgid = a.gorder[first + lane];
        const CellBox b = a.box[mgid];
        if (b.hi.x >= b.lo.x && a.q.n > 0) {
            if (GRID) {
                const GridRows r = grid_rows(a.rec[mgid], b, a.q, a.g, a.bg);
                mx = r.x0;
                mnx = r.x1;
                my = r.y0;
                mny = r.ny;
                mz = r.z0;
                mR = r.ny * r.nz;
            } else {
                mx = (uint32_t)b.lo.x;
                mnx = (uint32_t)(b.hi.x - b.lo.x + 1);
                my = (uint32_t)b.lo.y;
                mny = (uint32_t)(b.hi.y - b.lo.y + 1);
                mz = (uint32_t)b.lo.z;
                mR = mny * (uint32_t)(b.hi.z - b.lo.z + 1);
            }
        }
    }
    const uint32_t mRend = wave_incl_sum(mR);
    const uint32_t Rw = __builtin_amdgcn_readlane(mRend, kWave - 1);
    const bool fdiv = wave_max_uniform(mR) < (1u << 21);
    float mtot = 0.0f;  // lane i < nk: Gaussian i's sum
    for (uint32_t rb = 0; rb < Rw; rb += kWave) {
        // lane l takes row rb + l of the wave's list, of Gaussian i; lanes
        // past the last row have none (the permutes run with every lane)
        const uint32_t gr = rb + lane;
        uint32_t i = 0;
        for (uint32_t t = 0; t < nk; ++t) i += __builtin_amdgcn_readlane(mRend, t) <= gr ? 1u : 0u;
        const uint32_t src = (i < kWave ? i : 0u) << 2;
        auto perm = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_ds_bpermute((int)src, (int)v); };
        const uint32_t gid = perm(mgid), end = perm(mRend), R = perm(mR), nx = perm(mnx), ny = perm(mny);
        const uint32_t x0 = perm(mx), y0 = perm(my), z0 = perm(mz);
        float acc = 0.0f;
        if (gr < Rw) {
            const Record r = a.rec[gid];
            const float margin = cutoff_margin(a.exact, gid, T);
            uint32_t yy, zz, start;
            row_yz(gr - (end - R), ny, fdiv, yy, zz);
            // whether a pair of this Q' at p is within the cutoff
            auto within = [&](float Q, float px, float py, float pz) {
                bool in = Q <= T;
                if (__builtin_fabsf(Q - T) <= margin) in = within_exact(a.exact, gid, px, py, pz);
                return in;
            };
            if (GRID) {
                uint32_t vx;
                float py, pz;
                const uint32_t len = grid_row(r, x0, nx, y0 + yy, z0 + zz, a.q, a.g, a.bg, vx, py, pz);
                const float *f = a.f + ((size_t)vx + (size_t)(uint32_t)a.q.dims[0] *
                                                         ((y0 + yy) + (size_t)(uint32_t)a.q.dims[1] * (z0 + zz)));
                const float dy = py - r.f0.y, dz = pz - r.f0.z;
                const float c0 = fmaf_(r.f1.y, dy, r.f1.z * dz);
                const float u1 = fmaf_(r.f2.x, dy, r.f2.y * dz), u2 = r.f2.z * dz;
                const float c1 = fmaf_(u1, u1, u2 * u2);
                for (uint32_t e = 0; e < len; ++e) {
                    const float px = a.g.lo[0] + ((float)(vx + e) + 0.5f) * a.q.vsz[0];
                    const float u0 = fmaf_(r.f1.x, px - r.f0.x, c0);
                    const float Q = fmaf_(u0, u0, c1);
                    const float v = exp2_hw(-Q) * f[e];
                    acc += within(Q, px, py, pz) ? v : 0.0f;
                }
            } else {
                const uint32_t len = plan_row(r, x0, nx, y0 + yy, z0 + zz, a.g, a.bg, a.point_off, start);
                const float4 *p = a.pts + start;
                for (uint32_t e = 0; e < len; ++e) {
                    const float4 t = p[e];
                    const float Q = record_q(r, t.x, t.y, t.z);
                    const float v = exp2_hw(-Q) * t.w;
                    acc += within(Q, t.x, t.y, t.z) ? v : 0.0f;
                }
            }
        }
        // inclusive sums over the lanes of one Gaussian
#pragma unroll
        for (uint32_t o = 1; o < (uint32_t)kWave; o <<= 1) {
            const float v = __shfl_up(acc, o, kWave);
            const uint32_t j = __shfl_up(i, o, kWave);
            if (lane >= o && j == i) acc += v;
        }
        // the last row of Gaussian `lane` in this batch has its sum
        const uint32_t beg = mRend - mR;
        const uint32_t la = beg > rb ? beg : rb, lb = mRend < rb + kWave ? mRend : rb + kWave;
        const bool some = lane < nk && la < lb;
        const float v = __int_as_float(
            __builtin_amdgcn_ds_bpermute(some ? (int)((lb - 1 - rb) << 2) : 0, __float_as_int(acc)));
        if (some) mtot += v;
    }
    if (lane < nk) {
        const float add = a.rec[mgid].f0.w * mtot;
        a.score[mgid] = a.decay > 0.0f ? fmaf_(a.decay, a.score[mgid], add) : add;
    }
}

size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

SharesWork shares_layout(void *work, int64_t nq, bool grid) {
    SharesWork w;
    const size_t m = (size_t)(nq > 0 ? nq : 1);
    w.pts = grid ? nullptr : (float4 *)work;
    w.f = grid ? (float *)work : nullptr;
    w.bytes = al256(m * (grid ? sizeof(float) : sizeof(float4)));
    return w;
}

hipError_t launch_shares(const QueryParams &q, const GridParams &g, const BwdGeom &bg, const Record *rec,
                         const CellBox *box, const uint32_t *gorder, int64_t n_gauss, const uint32_t *order,
                         const uint32_t *point_off, const float4 *plan_pos, float T, const SharesExact &exact,
                         const float *influence, const float *gain, float decay, float *score,
                         const SharesWork &w, hipStream_t s) {
    if (n_gauss <= 0) return hipSuccess;
    const bool grid = q.kind == 0;
    hipError_t e;
    if (q.n > 0) {
        const dim3 nb((uint32_t)((q.n + kBlock - 1) / kBlock));
        prof_begin("shares_stage", s);
        if (grid)
            hipLaunchKernelGGL(k_shares_stage_grid, nb, dim3(kBlock), 0, s, q.n, influence, gain, w.f);
        else
            hipLaunchKernelGGL(k_shares_stage_plan, nb, dim3(kBlock), 0, s, q.n, order, plan_pos, influence, gain,
                               w.pts);
        prof_end("shares_stage", s);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    SharesArgs a;
    a.q = q;
    a.g = g;
    a.bg = bg;
    a.rec = rec;
    a.box = box;
    a.gorder = gorder;
    a.n_gauss = n_gauss;
    a.point_off = point_off;
    a.pts = w.pts;
    a.f = w.f;
    a.exact = exact;
    a.T = T;
    a.decay = decay;
    a.score = score;
    // a wave's rows are counted in 32 bits
    const int64_t rows = grid ? (int64_t)q.dims[1] * q.dims[2] : (int64_t)g.cells[1] * g.cells[2];
    a.pack = n_gauss < kPackMinGauss || rows > ((int64_t)1 << 31) / kPack ? 1u : kPack;
    const uint64_t waves = ((uint64_t)n_gauss + a.pack - 1) / a.pack;
    prof_begin("shares", s);
    for (a.wave0 = 0; a.wave0 < waves; a.wave0 += kWavesMost) {
        const uint64_t left = waves - a.wave0;
        const dim3 wb((uint32_t)(left < kWavesMost ? left : kWavesMost));
        if (grid)
            hipLaunchKernelGGL(k_shares<true>, wb, dim3(kWave), 0, s, a);
        else
            hipLaunchKernelGGL(k_shares<false>, wb, dim3(kWave), 0, s, a);
    }
    prof_end("shares", s);
    return hipGetLastError();
}

}  // namespace gs
