// The attention weight that every Gaussian gets from a batch of queries
// (include/gs_budget.h): score_i <- decay score_i + w_i sum_t f_t G_i(p_t).
//
// A Gaussian's queries come in rows: of voxels at fixed (y, z) in grids, of the
// plan's cells for ordered queries, both cut to the cutoff ellipsoid as the
// backward cuts them. A wave takes the rows of a few Gaussians, cuts them into
// pieces of one width and walks them with the Gaussian's record in scalars, so
// that a query costs its load and the 24 or so instructions of a pair; lanes
// are added at a Gaussian's end: no atomics, an order fixed by the inputs. The
// bound is the arithmetic over the pairs of the rows, of which the cutoff keeps
// half where rows are of voxels and a fourth to a third where they are of the
// plan's cells: a 128^3 jittered grid and 131072 Gaussians, 54 million pairs, 151
// us. (A lane a row, each with its own record: 583 us.)
#include <type_traits>

#include "budget.h"

#pragma clang fp contract(off)

namespace gs {
namespace {

// Gaussians of a wave (consecutive in gorder), so that their rows fill its
// lanes; fewer where there would be fewer waves than the chip holds (20011
// Gaussians and 100003 points: two a wave 23 us, one 25; 30011 on a 64^3 grid:
// three 29 us, one 33).
constexpr uint32_t kPack = 4;
constexpr int64_t kPackWaves = 8192;
// Waves of an XCD that follow each other, so that neighbours read the same
// queries through one L2 (a jittered 128^3 grid, 131072 Gaussians, all of the
// call: 4 waves some 195 us, 64 166, 128 160, 256 166, 512 172).
constexpr uint32_t kXcdWaves = 128;
// The rows of a Gaussian's queries: voxels of a grid; the plan's cells; voxels
// of a jittered grid, every voxel with its query.
enum { kWalkGrid = 0, kWalkPlan = 1, kWalkVoxels = 2 };
// queries from which a jittered grid is walked by voxels
constexpr int64_t kVoxelsLeast = 4096;
// A Gaussian of more than kRowsMost rows, or that comes to more than kStepsMost
// steps with any of its batches of rows, keeps its wave long after the others
// are done. Where there are queries for such ones, they are left to the launch
// that follows, a workgroup of kTeam waves each. (One Gaussian that reaches all
// of 2 M points or voxels: 5.0 to 10 ms -> 0.73 to 1.5 ms; 9001 Gaussians,
// 300007 crowded points: 114 -> 93 us. Its first batch alone tells little of a
// Gaussian whose rows begin at that batch's end: one behind 60 rows of another
// that reaches all of 1 M points, 3.2 ms by its wave, 0.58 by a team. Without
// such ones the launch costs 4 to 5 us.) They go to kTeamLists lists: counts in
// one place wait for each other.
constexpr uint32_t kStepsMost = 256, kRowsMost = 1024;
constexpr uint32_t kTeam = 8;
constexpr int64_t kTeamQueries = 65536;
constexpr uint32_t kTeamBlocks = 512, kTeamLists = 64;

// How a wave takes its Gaussians: all of every one (calls of fewer than
// kTeamQueries queries); but for those that it leaves to teams; or a team's share
// of one.
enum { kFormAll = 0, kFormLeave = 1, kFormTeam = 2 };
// Steps whose terms a team's lane adds up in float32; its sums of them are held
// in float64, since a Gaussian can have any number of terms, which are alike, and
// so are their roundings (one over 2 M points was 4 10^-5 off in float32, over 16
// M 2 10^-4, now 4 10^-7). The other forms have some 1024 terms a lane at most.
constexpr uint32_t kSettle = 32;

// waves of one launch (a launch has fewer than 2^32 threads)
constexpr uint64_t kWavesMost = (uint64_t)1 << 25;

// The hardware's root, good to an ulp: what it bounds has more slack than that.
__device__ __forceinline__ float sqrt_hw(float x) { return __builtin_amdgcn_sqrtf(x); }

// f of a query: its gain over I, 0 where the field is undefined.
__device__ __forceinline__ float query_factor(const float *influence, const float *gain, int64_t t) {
    const float I = influence[t];
    if (!(I > 0.0f)) return 0.0f;
    return (gain ? gain[t] : 1.0f) / I;
}

__global__ __launch_bounds__(kBlock) void k_shares_stage_grid(int64_t n, const float *__restrict__ influence,
                                                              const float *__restrict__ gain, float *__restrict__ f,
                                                              uint32_t *__restrict__ teams) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i < kTeamLists) teams[i] = 0;
    if (i < n) f[i] = query_factor(influence, gain, i);
}

__global__ __launch_bounds__(kBlock) void k_shares_stage_plan(int64_t n, const uint32_t *__restrict__ order,
                                                              const float4 *__restrict__ pos,
                                                              const float *__restrict__ influence,
                                                              const float *__restrict__ gain,
                                                              float4 *__restrict__ pts,
                                                              uint32_t *__restrict__ teams) {
    const int64_t k = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (k < kTeamLists) teams[k] = 0;
    if (k >= n) return;
    const float4 p = pos[k];
    pts[k] = make_float4(p.x, p.y, p.z, query_factor(influence, gain, order[k]));
}

// Jittered grids whose every voxel has its query: positions in the voxels'
// order, and whether any lies outside its voxel (stray, cleared before).
// Positions that rounding carries over the domain's border are outside.
__global__ __launch_bounds__(kBlock) void k_shares_stage_voxels(QueryParams q, GridParams g,
                                                                const float *__restrict__ influence,
                                                                const float *__restrict__ gain,
                                                                float4 *__restrict__ pts,
                                                                uint32_t *__restrict__ stray,
                                                                uint32_t *__restrict__ teams) {
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i < kTeamLists) teams[i] = 0;
    if (i >= q.n) return;
    float p[3];
    bool valid, in = true, home = true;
    query_position(q, g, (uint32_t)i, p[0], p[1], p[2], valid);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const float u = q.points[3 * i + k];
        home = home && u >= 0.0f && u <= 1.0f;
        in = in && p[k] >= g.lo[k] && p[k] <= g.hi[k];
    }
    pts[i] = make_float4(p[0], p[1], p[2], in ? query_factor(influence, gain, i) : 0.0f);
    if (!home) *stray = 1;
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
// roundings of |u|^2 make (10 sqrt(3) kappa + 3) 2^-24 Q', below 2^-19 kappa Q'.
__device__ __forceinline__ float cutoff_margin(const SharesExact &x, uint32_t gid, float T) {
    const float *s = x.scale + 3 * (size_t)gid;
    const float hi = fmaxf(fmaxf(s[0], s[1]), s[2]), lo = fminf(fminf(s[0], s[1]), s[2]);
    return hi * __builtin_amdgcn_rcpf(lo) * 0x1p-19f * T;
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
    const uint32_t *order;
    const float4 *pts;
    const float *f;
    const uint32_t *stray;
    SharesExact exact;
    float T, decay;
    float *score;
    uint32_t *teams;  // Gaussians left to teams: the lists' counts, then the lists (null: none are left)
    uint32_t team_room;
    uint32_t pack;
    uint64_t wave0;  // the launch's first wave
};

// A grid's voxel: its number in x, its centre's y and z.
struct Voxel {
    uint32_t x;
    float y, z;
};

// The voxels of a jittered grid that a Gaussian can reach: a row (y, z) of
// voxels holds points of the slab [y, y + 1] x [z, z + 1]. With e the part of
// u = U d that depends on y and z alone, |e| over the slab is at least its value
// at the slab's centre less `reach`, the largest |e| of half a voxel; so is Q
// >= |e|^2. In x the row's centre moves by at most `shift` over the slab. (The
// slab is widened by what rounding moves a position.)
struct VoxelReach {
    float reach, shift;
};
__device__ __forceinline__ VoxelReach voxel_reach(const Record &r, const QueryParams &q, const BwdGeom &bg) {
    const float hy = (0.5f + bg.vslack[1]) * q.vsz[1], hz = (0.5f + bg.vslack[2]) * q.vsz[2];
    const float e1 = fabsf(r.f2.x) * hy + fabsf(r.f2.y) * hz, e2 = fabsf(r.f2.z) * hz;
    VoxelReach v;
    v.reach = sqrt_hw(fmaf_(e1, e1, e2 * e2)) * (1.0f + 0x1p-10f);
    v.shift = (fabsf(r.f1.y) * hy + fabsf(r.f1.z) * hz) / fabsf(r.f1.x);
    return v;
}

// Rows y0 .. y0 + ny - 1, z0 .. z0 + nz - 1 of voxels that meet the ellipsoid's box.
__device__ __forceinline__ void voxel_rows(const Record &r, const QueryParams &q, const GridParams &g,
                                           const BwdGeom &bg, uint32_t &y0, uint32_t &ny, uint32_t &z0,
                                           uint32_t &nz) {
    const float rt = sqrt_hw(bg.T2);
    const float t = r.f2.y / r.f2.z;
    const float hy = rt * sqrt_hw(fmaf_(t, t, 1.0f)) / r.f2.x, hz = rt / r.f2.z;
    auto cut = [](float mu, float h, float lo, float iv, float slack, int32_t dim, uint32_t &first, uint32_t &n) {
        n = clip_range(floorf((mu - h - lo) * iv - slack), floorf((mu + h - lo) * iv + slack), 0u, (uint32_t)dim - 1u,
                       first);
    };
    cut(r.f0.y, hy, g.lo[1], bg.ivsz[1], bg.vslack[1], q.dims[1], y0, ny);
    cut(r.f0.z, hz, g.lo[2], bg.ivsz[2], bg.vslack[2], q.dims[2], z0, nz);
}

// The voxels of row (vy, vz) that the cutoff T2 can reach: first and number.
__device__ __forceinline__ uint32_t voxel_row(const Record &r, const VoxelReach &v, uint32_t vy, uint32_t vz,
                                              const QueryParams &q, const GridParams &g, const BwdGeom &bg,
                                              uint32_t &first) {
    const float dy = g.lo[1] + ((float)vy + 0.5f) * q.vsz[1] - r.f0.y;
    const float dz = g.lo[2] + ((float)vz + 0.5f) * q.vsz[2] - r.f0.z;
    const float e1 = fmaf_(r.f2.x, dy, r.f2.y * dz), e2 = r.f2.z * dz;
    const float e = fmaxf(sqrt_hw(fmaf_(e1, e1, e2 * e2)) * (1.0f - 0x1p-10f) - v.reach, 0.0f);
    const float left = bg.T2 - e * e;
    first = 0;
    if (!(left >= 0.0f)) return 0;
    const float iu = __builtin_amdgcn_rcpf(r.f1.x);
    const float w = sqrt_hw(left) * iu * (1.0f + 0x1p-10f) + v.shift;
    const float c = r.f0.x - fmaf_(r.f1.y, dy, r.f1.z * dz) * iu;
    const float m = (fabsf(r.f0.x) + fabsf(c) + w) * 0x1p-20f;
    return clip_range(floorf((c - w - m - g.lo[0]) * bg.ivsz[0] - bg.vslack[0]),
                      floorf((c + w + m - g.lo[0]) * bg.ivsz[0] + bg.vslack[0]), 0u, (uint32_t)q.dims[0] - 1u, first);
}

// A wave takes `pack` Gaussians (consecutive in gorder). Their rows are listed
// one Gaussian after the other and set up 64 at a time, a lane a row; the rows
// with queries go to LDS, in up to kPieces pieces of 2^k queries. Then each
// Gaussian's are walked with its record in scalars: 2^k lanes a piece, the
// pieces next to each other, so that short rows share a step and a load reads
// whole stretches of memory, and kAhead steps at a time, all their loads under
// way before the first is used.
constexpr uint32_t kAhead = 2;
constexpr uint32_t kPieces = 4;
constexpr uint32_t kEntries = kPieces * kWave + kAhead * 16;  // the last steps read past their rows

// The sums of a wave's Gaussians, lane i < nk Gaussian i's (mgid). part of
// parts: of the steps, or of the rows where there are many, this wave takes its
// share. kFormLeave: Gaussians of too many rows or steps are left out, in `left` by
// bit.
template <int WALK, int FORM>
__device__ __forceinline__ float walk(const SharesArgs &a, uint32_t mgid, uint32_t nk, uint32_t part, uint32_t parts,
                                      uint32_t &left, uint2 *s_row, float2 *s_yz, uint32_t *s_x) {
    constexpr bool LEAVE = FORM == kFormLeave, TEAM = FORM == kFormTeam;
    const uint32_t lane = threadIdx.x % kWave;
    const float T = a.T;
    // positions that leave their voxels: the plan's rows, through its order
    const bool voxels = WALK == kWalkVoxels && *a.stray == 0;
    left = 0;
    // lane i < nk describes Gaussian i of the wave: its rows
    uint32_t mR = 0, mnx = 0, mny = 1, mx = 0, my = 0, mz = 0;
    VoxelReach mreach{0.0f, 0.0f};
    if (lane < nk) {
        const CellBox b = a.box[mgid];
        if (b.hi.x >= b.lo.x && a.q.n > 0) {
            if (WALK == kWalkGrid) {
                const GridRows r = grid_rows(a.rec[mgid], b, a.q, a.g, a.bg);
                mx = r.x0;
                mnx = r.x1;
                my = r.y0;
                mny = r.ny;
                mz = r.z0;
                mR = r.ny * r.nz;
            } else if (voxels) {
                const Record r = a.rec[mgid];
                uint32_t nz;
                voxel_rows(r, a.q, a.g, a.bg, my, mny, mz, nz);
                mR = mny * nz;
                mreach = voxel_reach(r, a.q, a.bg);
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
    if (LEAVE) {
        left = (uint32_t)__ballot(mR > kRowsMost);  // (lanes from nk on have none)
        mR = mR > kRowsMost ? 0u : mR;
    }
    const uint32_t mRend = wave_incl_sum(mR);
    const uint32_t Rw = __builtin_amdgcn_readlane(mRend, kWave - 1);
    const bool fdiv = wave_max_uniform(mR) < (1u << 21);
    float mtot = 0.0f;  // lane i < nk: Gaussian i's sum
    float acc = 0.0f;   // of the Gaussian being walked
    double held = 0.0;  // and a team's after every kSettle steps
    auto settle = [&]() {
        held += (double)acc;
        acc = 0.0f;
    };
    // where a loop of steps from `at` to `end`, `apart` from each other, settles
    auto stop_of = [&](uint32_t at, uint32_t end, uint32_t apart) {
        return !TEAM || end - at <= kSettle * apart ? end : at + kSettle * apart;
    };
    uint32_t cur = ~0u, cgid = 0;
    uint32_t steps = 0;  // of it, so far
    Record c = {};
    float margin = 0.0f;
    auto finish = [&]() {
        float t = row16_sum(TEAM ? (float)(held + (double)acc) : acc);
        t += swz_xor16(t);
        t += perm_xor32(t, lane);
        if (lane == cur) mtot = t;
        acc = 0.0f;
        held = 0.0;
    };
    // the parts share the batches of 64 rows; where those are fewer, several
    // parts share a batch's steps
    const uint32_t batches = Rw / kWave + (Rw % kWave ? 1u : 0u);
    const uint32_t groups = batches < parts ? (batches ? batches : 1u) : parts;
    const uint32_t sub = part / groups, subs = parts / groups;
    const uint32_t rb0 = sub < subs ? part % groups * kWave : Rw;
    const uint32_t stride = groups * kWave;
    for (uint32_t rb = rb0; rb < Rw; rb = Rw - rb > stride ? rb + stride : Rw) {  // (rb + stride may pass 2^32)
        // lane l sets up row rb + l of the wave's list, of Gaussian i (the
        // permutes run with every lane)
        const uint32_t gr = rb + lane;
        uint32_t i = 0;
        for (uint32_t t = 0; t < nk; ++t) i += __builtin_amdgcn_readlane(mRend, t) <= gr ? 1u : 0u;
        const uint32_t src = (i < kWave ? i : 0u) << 2;
        auto perm = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_ds_bpermute((int)src, (int)v); };
        const uint32_t gid = perm(mgid), end = perm(mRend), R = perm(mR), nx = perm(mnx), ny = perm(mny);
        const uint32_t x0 = perm(mx), y0 = perm(my), z0 = perm(mz);
        VoxelReach reach{0.0f, 0.0f};
        if (voxels) {
            reach.reach = __uint_as_float(perm(__float_as_uint(mreach.reach)));
            reach.shift = __uint_as_float(perm(__float_as_uint(mreach.shift)));
        }
        uint32_t start = 0, len = 0, vx = 0;
        float py = 0.0f, pz = 0.0f;
        if (gr < Rw) {
            const Record r = a.rec[gid];
            uint32_t yy, zz;
            row_yz(gr - (end - R), ny, fdiv, yy, zz);
            const uint32_t vy = y0 + yy, vz = z0 + zz;
            if (WALK == kWalkGrid)
                len = grid_row(r, x0, nx, vy, vz, a.q, a.g, a.bg, vx, py, pz);
            else if (voxels)
                len = voxel_row(r, reach, vy, vz, a.q, a.g, a.bg, vx);
            else
                len = plan_row(r, x0, nx, vy, vz, a.g, a.bg, a.point_off, start);
            if (WALK == kWalkGrid || voxels)
                start = (uint32_t)a.q.dims[0] * (vy + (uint32_t)a.q.dims[1] * vz) + vx;
        }
        // queries of a piece: a power of two, kPieces of them the longest row
        const uint32_t longest = wave_max_uniform(len);
        const bool whole = longest > kPieces * kWave;  // rows that stay in one piece
        const uint32_t shift = longest > 128u ? 6u : longest > 64u ? 5u : longest > 32u ? 4u : longest > 16u ? 3u : 2u;
        const uint32_t wide = 1u << shift, mine = lane & (wide - 1), own = lane >> shift;
        const uint32_t pieces = whole ? (len > 0 ? 1u : 0u) : (len + wide - 1) >> shift;
        const uint32_t upto = wave_incl_sum(pieces);  // pieces of the batch's rows up to this one's
        __builtin_amdgcn_wave_barrier();
        for (uint32_t k = 0; k < pieces; ++k) {
            const uint32_t at = upto - pieces + k, from = k << shift;
            s_row[at] = make_uint2(start + from, whole ? len : len - from);
            if (WALK == kWalkGrid) {
                s_yz[at] = make_float2(py, pz);
                s_x[at] = vx + from;
            }
        }
        __builtin_amdgcn_wave_barrier();
        const uint32_t nrows = Rw - rb < (uint32_t)kWave ? Rw - rb : (uint32_t)kWave;
        const uint32_t ia = __builtin_amdgcn_readlane(i, 0), ib = __builtin_amdgcn_readlane(i, nrows - 1);
        for (uint32_t gi = ia; gi <= ib; ++gi) {
            const uint32_t gend = __builtin_amdgcn_readlane(mRend, gi), gR = __builtin_amdgcn_readlane(mR, gi);
            if (gR == 0) continue;
            // its rows in this batch, and their pieces
            const uint32_t la = gend - gR > rb ? gend - gR - rb : 0u;
            const uint32_t lb = gend - rb < nrows ? gend - rb : nrows;
            const uint32_t ra = la ? __builtin_amdgcn_readlane(upto, la - 1) : 0u;
            const uint32_t rz = lb ? __builtin_amdgcn_readlane(upto, lb - 1) : 0u;
            if (gi != cur) {
                if (cur != ~0u) finish();
                cur = gi;
                steps = 0;
                cgid = __builtin_amdgcn_readlane(mgid, gi);
                c = load_record_uniform(a.rec, cgid);
                margin = readfirst_f(cutoff_margin(a.exact, cgid, T));
            }
            if (LEAVE) {
                if (whole) {
                    const uint32_t all = wave_incl_sum(lane >= la && lane < lb ? len : 0u);
                    steps += __builtin_amdgcn_readlane(all, kWave - 1) / kWave;
                } else {
                    steps += (rz - ra) >> (6u - shift);
                }
                if (steps > kStepsMost) {  // the team walks all of it
                    left |= 1u << gi;
                    acc = 0.0f;
                    continue;
                }
            }
            // kAhead queries of a lane: query k[u] if on[u], at voxel x[u] of
            // its row in grids
            auto add = [&](const uint32_t k[kAhead], const bool on[kAhead], const Voxel v[kAhead]) {
                float px[kAhead], py[kAhead], pz[kAhead], f[kAhead];
#pragma unroll
                for (uint32_t u = 0; u < kAhead; ++u) {
                    const uint32_t q = on[u] ? k[u] : 0u;
                    if (WALK == kWalkGrid) {
                        f[u] = a.f[q];
                    } else {
                        const float4 t = a.pts[WALK == kWalkVoxels && !voxels ? a.order[q] : q];
                        px[u] = t.x;
                        py[u] = t.y;
                        pz[u] = t.z;
                        f[u] = t.w;
                    }
                }
                bool in[kAhead], near[kAhead], any = false;
                float e[kAhead];
#pragma unroll
                for (uint32_t u = 0; u < kAhead; ++u) {
                    if (WALK == kWalkGrid) {
                        px[u] = a.g.lo[0] + ((float)v[u].x + 0.5f) * a.q.vsz[0];
                        py[u] = v[u].y;
                        pz[u] = v[u].z;
                    }
                    const float Q = record_q(c, px[u], py[u], pz[u]);
                    in[u] = on[u] && Q <= T;
                    near[u] = on[u] && __builtin_fabsf(Q - T) <= margin;
                    any = any || near[u];
                    e[u] = exp2_hw(-Q) * f[u];
                }
                if (any) {
#pragma unroll
                    for (uint32_t u = 0; u < kAhead; ++u)
                        if (near[u]) in[u] = within_exact(a.exact, cgid, px[u], py[u], pz[u]);
                }
#pragma unroll
                for (uint32_t u = 0; u < kAhead; ++u) acc += in[u] ? e[u] : 0.0f;
            };
            if (!whole) {
                const uint32_t rows = (uint32_t)kWave >> shift;  // of a step
                const uint32_t apart = subs * kAhead * rows;
                for (uint32_t r0 = ra + sub * kAhead * rows; r0 < rz;) {
                    const uint32_t stop = stop_of(r0, rz, apart);
                    for (; r0 < stop; r0 += apart) {
                        uint32_t k[kAhead];
                        bool on[kAhead];
                        Voxel v[kAhead] = {};
#pragma unroll
                        for (uint32_t u = 0; u < kAhead; ++u) {
                            const uint32_t row = r0 + u * rows + own;
                            const uint2 w = s_row[row];
                            on[u] = row < rz && mine < w.y;
                            k[u] = w.x + mine;
                            if (WALK == kWalkGrid) {
                                const float2 yz = s_yz[row];
                                v[u] = Voxel{s_x[row] + mine, yz.x, yz.y};
                            }
                        }
                        add(k, on, v);
                    }
                    if (!TEAM) break;
                    settle();
                }
            } else {
                for (uint32_t row = ra; row < rz; ++row) {
                    const uint2 w = s_row[row];
                    uint32_t x0 = 0;
                    float2 yz = make_float2(0.0f, 0.0f);
                    if (WALK == kWalkGrid) {
                        x0 = s_x[row];
                        yz = s_yz[row];
                    }
                    const uint32_t apart = subs * kAhead * kWave;
                    for (uint32_t e0 = sub * kAhead * kWave; e0 < w.y;) {
                        const uint32_t stop = stop_of(e0, w.y, apart);
                        for (; e0 < stop; e0 += apart) {
                            uint32_t k[kAhead];
                            bool on[kAhead];
                            Voxel v[kAhead];
#pragma unroll
                            for (uint32_t u = 0; u < kAhead; ++u) {
                                const uint32_t e = e0 + u * kWave + lane;
                                on[u] = e < w.y;
                                k[u] = w.x + e;
                                v[u] = Voxel{x0 + e, yz.x, yz.y};
                            }
                            add(k, on, v);
                        }
                        if (!TEAM) break;
                        settle();
                    }
                }
            }
        }
    }
    if (cur != ~0u) finish();
    return mtot;
}

__device__ __forceinline__ void add_score(const SharesArgs &a, uint32_t gid, float sum) {
    const float add = a.rec[gid].f0.w * sum;
    a.score[gid] = a.decay > 0.0f ? fmaf_(a.decay, a.score[gid], add) : add;
}

// Waves of a SIMD, to which registers are held: waits for loads and LDS are
// filled by other waves (6, then 7 or 8 of them: a jittered 128^3 grid 167 -> 156
// us, 2 M points 172 -> 155; grids lose by it, 120 -> 124 us).
constexpr int waves_of(int walk) { return walk == kWalkPlan ? 8 : walk == kWalkVoxels ? 7 : 6; }
template <int WALK, int FORM>
__global__ __launch_bounds__(kWave, waves_of(WALK)) void k_shares(SharesArgs a) {
    __shared__ uint2 s_row[kEntries];   // first query, queries
    __shared__ float2 s_yz[WALK == kWalkGrid ? kEntries : 1];   // grids: y and z, first voxel in x
    __shared__ uint32_t s_x[WALK == kWalkGrid ? kEntries : 1];
    const uint32_t lane = threadIdx.x;
    const uint64_t first = (a.wave0 + xcd_group<kXcdWaves>(blockIdx.x, gridDim.x)) * a.pack;
    if (first >= (uint64_t)a.n_gauss) return;
    const uint32_t nk = (uint64_t)a.n_gauss - first < a.pack ? (uint32_t)((uint64_t)a.n_gauss - first) : a.pack;
    const uint32_t gid = lane < nk ? a.gorder[first + lane] : 0u;
    uint32_t left;
    const float sum = walk<WALK, FORM>(a, gid, nk, 0, 1, left, s_row, s_yz, s_x);
    if (lane >= nk) return;
    if (FORM == kFormLeave && (left >> lane & 1u)) {
        const uint32_t list = (uint32_t)((a.wave0 + blockIdx.x) % kTeamLists);
        a.teams[kTeamLists + (size_t)list * a.team_room + atomicAdd(&a.teams[list], 1u)] = gid;
    } else
        add_score(a, gid, sum);
}

// The Gaussians that k_shares left, a workgroup each.
template <int WALK>
__global__ __launch_bounds__(kTeam * kWave) void k_shares_team(SharesArgs a) {
    __shared__ uint2 s_row[kTeam][kEntries];
    __shared__ float2 s_yz[WALK == kWalkGrid ? kTeam : 1][WALK == kWalkGrid ? kEntries : 1];
    __shared__ uint32_t s_x[WALK == kWalkGrid ? kTeam : 1][WALK == kWalkGrid ? kEntries : 1];
    __shared__ float s_sum[kTeam];
    const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const uint32_t list = blockIdx.x % kTeamLists, count = a.teams[list];
    for (uint32_t i = blockIdx.x / kTeamLists; i < count; i += gridDim.x / kTeamLists) {
        const uint32_t gid = a.teams[kTeamLists + (size_t)list * a.team_room + i];
        uint32_t left;
        const float sum = walk<WALK, kFormTeam>(a, gid, 1, wave, kTeam, left, s_row[wave],
                                            s_yz[WALK == kWalkGrid ? wave : 0], s_x[WALK == kWalkGrid ? wave : 0]);
        if (lane == 0) s_sum[wave] = sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            float all = 0.0f;
#pragma unroll
            for (uint32_t w = 0; w < kTeam; ++w) all += s_sum[w];
            add_score(a, gid, all);
        }
        __syncthreads();
    }
}

bool has_teams(int64_t nq) { return nq >= kTeamQueries; }

size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

bool walks_voxels(const QueryParams &q) { return q.kind == 3 && !q.voxel_ids && q.n >= kVoxelsLeast; }

SharesWork shares_layout(void *work, int64_t n_gauss, int64_t nq, bool grid) {
    SharesWork w;
    const size_t m = (size_t)(nq > 0 ? nq : 1);
    char *b = (char *)work;
    w.stray = (uint32_t *)b;
    w.teams = b ? (uint32_t *)(b + 256) : nullptr;
    const size_t room = has_teams(nq) ? (size_t)n_gauss + kTeamLists * kPack : 0;
    const size_t head = 256 + al256(sizeof(uint32_t) * (kTeamLists + room));
    w.pts = grid || !b ? nullptr : (float4 *)(b + head);
    w.f = grid && b ? (float *)(b + head) : nullptr;
    w.bytes = head + al256(m * (grid ? sizeof(float) : sizeof(float4)));
    return w;
}

hipError_t launch_shares(const QueryParams &q, const GridParams &g, const BwdGeom &bg, const Record *rec,
                         const CellBox *box, const uint32_t *gorder, int64_t n_gauss, const uint32_t *order,
                         const uint32_t *point_off, const float4 *plan_pos, float T, const SharesExact &exact,
                         const float *influence, const float *gain, float decay, float *score,
                         const SharesWork &w, hipStream_t s) {
    if (n_gauss <= 0) return hipSuccess;
    const int kind = q.kind == 0 ? kWalkGrid : walks_voxels(q) ? kWalkVoxels : kWalkPlan;
    hipError_t e;
    if (q.n > 0) {
        const dim3 nb((uint32_t)((q.n + kBlock - 1) / kBlock));
        prof_begin("shares_stage", s);
        if (kind == kWalkGrid) {
            hipLaunchKernelGGL(k_shares_stage_grid, nb, dim3(kBlock), 0, s, q.n, influence, gain, w.f, w.teams);
        } else if (kind == kWalkVoxels) {
            if ((e = fill_u32(w.stray, 0u, 1, s)) != hipSuccess) return e;
            hipLaunchKernelGGL(k_shares_stage_voxels, nb, dim3(kBlock), 0, s, q, g, influence, gain, w.pts, w.stray,
                               w.teams);
        } else {
            hipLaunchKernelGGL(k_shares_stage_plan, nb, dim3(kBlock), 0, s, q.n, order, plan_pos, influence, gain,
                               w.pts, w.teams);
        }
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
    a.order = order;
    a.pts = w.pts;
    a.f = w.f;
    a.stray = w.stray;
    a.exact = exact;
    a.T = T;
    a.decay = decay;
    a.score = score;
    // a wave's rows are counted in 32 bits
    const int64_t rows = kind == kWalkPlan ? (int64_t)g.cells[1] * g.cells[2] : (int64_t)q.dims[1] * q.dims[2];
    const int64_t most = n_gauss / kPackWaves < (int64_t)kPack ? n_gauss / kPackWaves : (int64_t)kPack;
    a.pack = most < 1 || rows > ((int64_t)1 << 31) / kPack ? 1u : (uint32_t)most;
    const uint64_t waves = ((uint64_t)n_gauss + a.pack - 1) / a.pack;
    a.teams = has_teams(q.n) ? w.teams : nullptr;
    a.team_room = (uint32_t)((waves + kTeamLists - 1) / kTeamLists * a.pack);
    prof_begin("shares", s);
    for (a.wave0 = 0; a.wave0 < waves; a.wave0 += kWavesMost) {
        const uint64_t left = waves - a.wave0;
        const dim3 wb((uint32_t)(left < kWavesMost ? left : kWavesMost));
        auto launch = [&](auto walk, auto form) {
            hipLaunchKernelGGL((k_shares<decltype(walk)::value, decltype(form)::value>), wb, dim3(kWave), 0, s, a);
        };
        auto each = [&](auto form) {
            if (kind == kWalkGrid)
                launch(std::integral_constant<int, kWalkGrid>(), form);
            else if (kind == kWalkVoxels)
                launch(std::integral_constant<int, kWalkVoxels>(), form);
            else
                launch(std::integral_constant<int, kWalkPlan>(), form);
        };
        if (a.teams)
            each(std::integral_constant<int, kFormLeave>());
        else
            each(std::integral_constant<int, kFormAll>());
    }
    prof_end("shares", s);
    if (a.teams) {
        const dim3 tb(kTeamBlocks), tt(kTeam * kWave);
        prof_begin("shares_team", s);
        if (kind == kWalkGrid)
            hipLaunchKernelGGL(k_shares_team<kWalkGrid>, tb, tt, 0, s, a);
        else if (kind == kWalkVoxels)
            hipLaunchKernelGGL(k_shares_team<kWalkVoxels>, tb, tt, 0, s, a);
        else
            hipLaunchKernelGGL(k_shares_team<kWalkPlan>, tb, tt, 0, s, a);
        prof_end("shares_team", s);
    }
    return hipGetLastError();
}

}  // namespace gs
