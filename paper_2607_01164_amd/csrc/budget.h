// Internal declarations of the budget operators (include/gs_budget.h):
// shares.hip, evict.hip, draw.hip and their launchers.
#pragma once

#include "../../include/gs_budget.h"
#include "internal.h"

namespace gs {

// Accumulated attention weight (shares.hip).
struct SharesWork {
    float4 *pts;      // ordered queries, in the plan's or the voxels' order: position and f
    float *f;         // grids: f of every voxel
    uint32_t *stray;  // jittered grids: whether a position lies outside its voxel
    uint32_t *teams;  // Gaussians left to teams of waves: the lists' counts, then the lists
    size_t bytes;
};
SharesWork shares_layout(void *work, int64_t n_gauss, int64_t nq, bool grid);
// The Gaussians as the caller holds them, for the pairs near the cutoff.
struct SharesExact {
    const float *mean, *scale, *rot;
    double cut;  // 2 ln(1 / tau)
};
hipError_t launch_shares(const QueryParams &q, const GridParams &g, const BwdGeom &bg, const Record *rec,
                         const CellBox *box, const uint32_t *gorder, int64_t n_gauss, const uint32_t *order,
                         const uint32_t *point_off, const float4 *plan_pos, float T, const SharesExact &exact,
                         const float *influence, const float *gain, float decay, float *score,
                         const SharesWork &w, hipStream_t s);

// Eviction and copies (evict.hip).
size_t evict_work_bytes(int64_t n);
hipError_t launch_evict(const gs_params &in, int64_t n, const float *score, const uint8_t *pinned, int64_t keep,
                        const gs_params &out, int32_t *source, float *score_out, void *work, hipStream_t s);
hipError_t launch_split(const gs_params &set, int64_t n, const int32_t *ids, int64_t count, int32_t *source,
                        float *score, uint32_t *copies, hipStream_t s);

// Draws (draw.hip).
size_t draw_work_bytes(int64_t rows, int64_t n, int64_t draws);
hipError_t launch_draw(int64_t rows, int64_t n, const void *scores, int64_t stride, const int32_t *lengths,
                       const gs_draw_params &p, int64_t draws, const double *uniform, int32_t *ids, float *prob,
                       void *work, hipStream_t s);

}  // namespace gs
