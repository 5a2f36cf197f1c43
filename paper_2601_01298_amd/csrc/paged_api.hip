// C-ABI front end of the paged cache: argument validation on the host, then the kernel launchers.
#include <cmath>

#include "paged_internal.h"

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int kMaxRows = 1 << 24;

ws_status check_cache(const ws_paged_cache *c)
{
    if (!c) return WS_ERR_INVALID_ARG;
    if (c->dt != WS_F32 && c->dt != WS_BF16) return WS_ERR_UNSUPPORTED;
    if (c->d != 64 && c->d != 128) return WS_ERR_UNSUPPORTED;
    if (!c->K || !c->V || !c->table || !c->len || c->pages < 1 || c->Hkv < 1 || c->S < 1 || c->per_seq < 1) return WS_ERR_INVALID_ARG;
    if (!aligned(c->K, 16) || !aligned(c->V, 16) || !aligned(c->table, 4) || !aligned(c->len, 4)) return WS_ERR_INVALID_ARG;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128 && c->page != 256) return WS_ERR_UNSUPPORTED;
    if ((long long)c->per_seq * c->page >= kMaxRows) return WS_ERR_UNSUPPORTED;
    // (sequence, head) pairs index the launches
    if ((long long)c->S * c->Hkv > (1 << 20)) return WS_ERR_UNSUPPORTED;
    return WS_OK;
}

ws_status check_rows(const ws_rows *r, int es)
{
    if (!r || !r->x || !aligned(r->x, 16) || r->token < 0 || r->head < 0) return WS_ERR_INVALID_ARG;
    if ((r->token % (16 / es)) != 0 || (r->head % (16 / es)) != 0) return WS_ERR_INVALID_ARG;
    return WS_OK;
}

ws_status check_ws(const void *ws, size_t have, size_t need)
{
    if (need == 0) return WS_OK;
    return ws == nullptr || !aligned(ws, 256) || have < need ? WS_ERR_WORKSPACE : WS_OK;
}

}  // namespace

extern "C" {

ws_status ws_synapse_paged_append(const ws_paged_cache *cache, const ws_rows *k, const ws_rows *v, int T, const int32_t *first,
                                  const int32_t *pos, int axes, const int *pairs_host, float base, const ws_rows *q, int Hq,
                                  void *q_out, const int32_t *seen, int32_t *stamp, float *mass, ws_stream stream)
{
    ws_status s = check_cache(cache);
    if (s != WS_OK) return s;
    const int es = cache->dt == WS_BF16 ? 2 : 4, half = cache->d / 2;
    if ((s = check_rows(k, es)) != WS_OK || (s = check_rows(v, es)) != WS_OK) return s;
    if (q && (s = check_rows(q, es)) != WS_OK) return s;
    if (T < 1 || !first || !aligned(first, 4) || !aligned(pos, 4) || !aligned(stamp, 4) || !aligned(mass, 4) || !aligned(seen, 4))
        return WS_ERR_INVALID_ARG;
    if (stamp && !seen) return WS_ERR_INVALID_ARG;
    if (q && (Hq < 1 || !q_out || !aligned(q_out, 16))) return WS_ERR_INVALID_ARG;
    if (q && Hq > (1 << 16)) return WS_ERR_UNSUPPORTED;
    if (T >= kMaxRows) return WS_ERR_UNSUPPORTED;
    ws::RotaryTable rot = {};
    if (pos) {
        if (!pairs_host || !(base > 0.0f) || !std::isfinite(base)) return WS_ERR_INVALID_ARG;
        if (axes < 1 || axes > ws::kMaxAxes) return WS_ERR_UNSUPPORTED;
        // base^(-2c/d) turns / (2 pi) pair by pair; 64 products in 64 bits of mantissa are off by less than half a step of the result
        const long double step = std::pow((long double)base, -2.0L / cache->d);
        long double turns = 1.0L / 6.283185307179586476925286766559L;
        int c = 0;
        for (int a = 0; a < axes; ++a) {
            if (pairs_host[a] < 0 || pairs_host[a] > half - c) return WS_ERR_INVALID_ARG;
            for (int i = 0; i < pairs_host[a]; ++i, ++c) {
                rot.axis[c] = (unsigned char)a;
                rot.turns[c] = (double)turns;
                turns *= step;
            }
        }
        if (c != half) return WS_ERR_INVALID_ARG;
    }
    const hipError_t e = ws::launch_paged_append(*cache, *k, *v, T, first, pos, rot, q, Hq, q_out, seen, stamp, mass,
                                                 (hipStream_t)stream);
    return e == hipSuccess ? WS_OK : WS_ERR_HIP;
}

ws_status ws_synapse_paged_attend(const ws_paged_cache *cache, const void *Q, int Hq, float scale, float *O, float *lse, float decay,
                                  const float *mass_in, float *mass_out, void *workspace, size_t workspace_bytes, ws_stream stream)
{
    ws_status s = check_cache(cache);
    if (s != WS_OK) return s;
    if (!Q || !O || Hq < 1 || Hq % cache->Hkv != 0 || !std::isfinite(scale)) return WS_ERR_INVALID_ARG;
    if (!aligned(Q, 16) || !aligned(O, 16) || !aligned(lse, 4) || !aligned(mass_in, 4) || !aligned(mass_out, 4)) return WS_ERR_INVALID_ARG;
    if (mass_in && !mass_out) return WS_ERR_INVALID_ARG;
    if (mass_out && !(decay >= 0.0f && std::isfinite(decay))) return WS_ERR_INVALID_ARG;
    if ((long long)cache->S * Hq > (1 << 20)) return WS_ERR_UNSUPPORTED;
    const int cap = cache->per_seq * cache->page;
    const bool bf16 = cache->dt == WS_BF16;
    if (ws::paged_most_tiles(bf16, cache->S, cache->Hkv, Hq, cap) > 0x7FFFFFFFLL) return WS_ERR_UNSUPPORTED;
    if (mass_out && !ws::paged_logits_fit(Hq / cache->Hkv, cap)) return WS_ERR_UNSUPPORTED;
    s = check_ws(workspace, workspace_bytes, ws::paged_attend_workspace_bytes(bf16, cache->S, cache->Hkv, Hq, cap, cache->d, mass_out != nullptr));
    if (s != WS_OK) return s;
    if (scale <= 0.0f) scale = 1.0f / std::sqrt((float)cache->d);
    const hipError_t e = ws::launch_paged_attend(*cache, Q, Hq, scale, O, lse, decay, mass_in, mass_out, workspace, (hipStream_t)stream);
    return e == hipSuccess ? WS_OK : WS_ERR_HIP;
}

ws_status ws_synapse_paged_evict(const ws_paged_cache *cache, int keep, int sinks, int recent, const int32_t *seen,
                                 const float *mass_in, float *mass_out, const int32_t *stamp_in, int32_t *stamp_out,
                                 int32_t *len_out, int32_t *kept, void *workspace, size_t workspace_bytes, ws_stream stream)
{
    ws_status s = check_cache(cache);
    if (s != WS_OK) return s;
    if (!seen || !mass_in || !mass_out || !stamp_in || !stamp_out || !len_out) return WS_ERR_INVALID_ARG;
    if (keep < 1 || sinks < 0 || recent < 0 || (long long)sinks + recent > keep) return WS_ERR_INVALID_ARG;
    if (!aligned(seen, 4) || !aligned(mass_in, 4) || !aligned(mass_out, 4) || !aligned(stamp_in, 4) || !aligned(stamp_out, 4) ||
        !aligned(len_out, 4) || !aligned(kept, 4))
        return WS_ERR_INVALID_ARG;
    if (keep >= kMaxRows) return WS_ERR_UNSUPPORTED;
    const int cap = cache->per_seq * cache->page;
    s = check_ws(workspace, workspace_bytes, ws::paged_evict_workspace_bytes(cache->S, cache->Hkv, cap, keep));
    if (s != WS_OK) return s;
    const hipError_t e = ws::launch_paged_evict(*cache, keep, sinks, recent, seen, mass_in, mass_out, stamp_in, stamp_out, len_out, kept,
                                                workspace, (hipStream_t)stream);
    return e == hipSuccess ? WS_OK : WS_ERR_HIP;
}

}  // extern "C"
