// What the front end and the kernels of the paged cache share.
#pragma once
#include "../../include/ws_synapse.h"
#include "ws_internal.h"

namespace ws {

constexpr int kMaxAxes = 4;

// Sizes for the attention's workspace: partial rows of the splits, statistics of every query head, and with weights the logits.
constexpr int kPagedSplitTarget = 1024;     // workgroups a launch aims at
constexpr int kPagedUnit = 128;             // rows of the smallest split

static inline int paged_splits(int S, int Hkv, int cap)
{
    const long long pairs = (long long)S * Hkv;
    const long long want = (kPagedSplitTarget + pairs - 1) / pairs, most = (cap + kPagedUnit - 1) / kPagedUnit;
    return (int)(want < most ? want : most);
}

struct PagedAttendSpace {
    size_t partial, stats, logits, bytes;   // offsets, total
};
static inline PagedAttendSpace paged_attend_space(int S, int Hkv, int Hq, int cap, int d, bool weights)
{
    PagedAttendSpace p;
    const size_t rows = (size_t)S * Hq;
    p.partial = 0;
    p.stats = round_up(rows * paged_splits(S, Hkv, cap) * (d + 2) * sizeof(float), 256);
    p.logits = p.stats + round_up(rows * sizeof(float), 256);
    p.bytes = p.logits + (weights ? round_up(rows * cap * sizeof(float), 256) : 0);
    return p;
}
static inline size_t paged_attend_workspace_bytes(int S, int Hkv, int Hq, int cap, int d, bool weights)
{
    return paged_attend_space(S, Hkv, Hq, cap, d, weights).bytes;
}

// Per KV head of a sequence: how many rows move, and from where to where.
static inline int paged_evict_moves(int cap, int keep) { return keep >= cap ? 1 : (keep < cap - keep ? keep : cap - keep); }
static inline size_t paged_evict_workspace_bytes(int S, int Hkv, int cap, int keep)
{
    const size_t pairs = (size_t)S * Hkv;
    return round_up(pairs * sizeof(int32_t), 256) + round_up(pairs * paged_evict_moves(cap, keep) * 2 * sizeof(int32_t), 256);
}

// turns per unit of position of every pair, and the axis it goes by
struct RotaryTable {
    double turns[64];
    unsigned char axis[64];
};

hipError_t launch_paged_append(const ws_paged_cache &c, const ws_rows &k, const ws_rows &v, int T, const int32_t *first,
                               const int32_t *pos, const RotaryTable &rot, const ws_rows *q, int Hq, void *q_out, const int32_t *seen,
                               int32_t *stamp, float *mass, hipStream_t st);
hipError_t launch_paged_attend(const ws_paged_cache &c, const void *Q, int Hq, float scale, float *O, float *lse, float decay,
                               const float *mass_in, float *mass_out, void *ws, hipStream_t st);
hipError_t launch_paged_evict(const ws_paged_cache &c, int keep, int sinks, int recent, const int32_t *seen, const float *mass_in,
                              float *mass_out, const int32_t *stamp_in, int32_t *stamp_out, int32_t *len_out, int32_t *kept,
                              void *ws, hipStream_t st);

#ifdef __HIPCC__
// Rows of a sequence that count: what `len` says, within the table.
__device__ __forceinline__ int paged_rows(int n, int cap) { return n < 0 ? 0 : (n > cap ? cap : n); }
// First row of head h in page number `p`, counted in rows of the pool; a number outside the pool stands for page 0.
__device__ __forceinline__ long long paged_base(int p, int pages, int Hkv, int h, int page)
{
    const int q = (unsigned)p < (unsigned)pages ? p : 0;
    return ((long long)q * Hkv + h) * page;
}
#endif

}  // namespace ws
