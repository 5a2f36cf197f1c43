// What the front end and the kernels of the paged cache share.
#pragma once
#include "../../include/ws_synapse.h"
#include "ws_internal.h"

namespace ws {

constexpr int kMaxAxes = 4;

// How a launch of the attention is shared out.  The rows of all (sequence, KV head, up to 16 of its query heads) are counted off in
// tiles, and every workgroup takes an equal run of tiles, across the borders of heads and sequences.
constexpr int kPagedGroups = 512;           // most workgroups of a launch
constexpr int kPagedQueries = 16;           // query heads a workgroup serves from one reading of the rows: the matrix tile's width
static inline int paged_tile_rows(bool bf16) { return bf16 ? 32 : 16; }
static inline int paged_query_tiles(int g) { return (g + kPagedQueries - 1) / kPagedQueries; }
// most tiles there can be (the lengths are on the device)
static inline long long paged_most_tiles(bool bf16, int S, int Hkv, int Hq, int cap)
{
    const int tr = paged_tile_rows(bf16);
    return (long long)S * Hkv * paged_query_tiles(Hq / Hkv) * ((cap + tr - 1) / tr);
}
// One workgroup of four waves per compute unit keeps the memory busiest (8 heads of 131072 rows, d = 128: 84 us with 256, 88 with 512, 90
// with 768; 256 heads of 32768 rows, d = 64: 309, 325, 328).  Where a tile is only 4 KB and a workgroup has few of them, two hide more of
// the way from one head to the next (128 heads of up to 4000 rows, bf16, d = 64: 21.5 us with 256, 18.7 with 512; 72 heads of up to 4100,
// fp32, d = 64: 17.6, 16.3; but 64 heads of 2048, d = 128: 19.4, 20.2).  fp32 at d = 128, tiles of 8 KB as bf16: 8 heads of 131072 rows 179,
// 182; 128 heads of 2048 51, 51; 72 of up to 4100 37, 37; for 128 heads of lengths spread in their logarithm up to 16384, 89 and 78, where
// bf16 takes 51 and 51.
static inline int paged_groups(bool bf16, int S, int Hkv, int Hq, int cap, int d)
{
    const long long tiles = paged_most_tiles(bf16, S, Hkv, Hq, cap), want = (tiles + 3) / 4;     // four waves, a tile each
    const int most = d == 128 || tiles >= 256 * 256 ? 256 : kPagedGroups;
    return (int)(want < most ? want : most);
}

// whole tiles of logits per query head
__host__ __device__ static inline int logit_rows(int cap) { return (cap + 31) / 32 * 32; }

// their offsets within a head travel in 32 bits
static inline bool paged_logits_fit(int g, int cap) { return (long long)logit_rows(cap) * g < (1LL << 29); }

// Whether every (sequence, KV head) goes to one workgroup that does all of it, in one launch.  Short caches, where the second launch costs
// more than a few tiles one after the other (2 heads of 200 rows: 3.9 us against 9.5; 8 of 700: 12.8 against 11.2; 8 of 2000: 29.5
// against 10.7), and so many heads that they fill the chip as they are, up to a width of the tables at which the longest head there
// may be does not keep one compute unit busy long after the others: the lengths are on the device.  A row costs its workgroup 8 ns at
// d = 64, 14 ns at 128; a batch of one long sequence among short ones ends with it.  us, one workgroup per head / equal runs, bf16 at
// d = 128, g = 1, with all sequences as long as the table, spread evenly in their logarithm, and one that long among ones of 64 rows:
//                                 rows   equal        log-spread   one long
//     512 heads, no weights       1216    51 / 54      36 / 40      21 / 14
//                                 1536    63 / 66      34 / 43      25 / 15
//                                 2048    83 / 85      40 / 46      32 / 14
//                                 5120   203 / 200     89 / 72      72 / 19
//     1600 heads, no weights      1536   203 / 194     66 / 112     30 / 28
//                                 2048   270 / 254     90 / 99      39 / 29
//                                 5120   675 / 613    185 / 185     79 / 36
//     512 heads, weights          1216    53 / 60      23 / 42      22 / 16
//                                 2048    87 / 93      47 / 52      33 / 17
//                                 2560   108 / 116     63 / 70      39 / 19
//                                 4096   173 / 186     68 / 65      60 / 19
//     1600 heads, weights         2048   295 / 299     84 / 146     36 / 36
//                                 4096   593 / 597    167 / 206     65 / 42
// (d = 64 and fp32 alike.)  Behind 1536 rows one workgroup per head gains nothing without weights.  With them, whose logits then stay in
// LDS, it gains up to 15 % (512 heads of 4096 rows, d = 64: 88 / 104) where all are as long as their table, and takes three times as
// long where one is.
constexpr int kWholeRows = 512, kWholePairs = 512, kWholePairRows = 1536, kWholePairRowsWeights = 2048;
constexpr int kWholeLogits = 5120;          // 20 KB beside the merge area
static inline bool paged_whole_heads(int S, int Hkv, int Hq, int cap, bool weights)
{
    const int g = Hq / Hkv;
    if (weights && (g > kPagedQueries || (long long)(logit_rows(cap) + 4) * g > kWholeLogits)) return false;
    return cap <= kWholeRows || ((long long)S * Hkv >= kWholePairs && cap <= (weights ? kWholePairRowsWeights : kWholePairRows));
}

struct PagedAttendSpace {
    size_t start, stats, slot_stats, slots, logits, bytes;   // offsets, total; the first 256 bytes hold the number of tiles
};
static inline PagedAttendSpace paged_attend_space(bool bf16, int S, int Hkv, int Hq, int cap, int d, bool weights)
{
    PagedAttendSpace p;
    const int g = Hq / Hkv, gt = g < kPagedQueries ? g : kPagedQueries;
    const size_t slots = 2 * (size_t)paged_groups(bf16, S, Hkv, Hq, cap, d);
    p.start = 256;
    p.stats = p.start + round_up((size_t)S * Hkv * paged_query_tiles(g) * sizeof(int32_t), 256);
    p.slot_stats = p.stats + round_up((size_t)S * Hq * sizeof(float), 256);
    p.slots = p.slot_stats + round_up(slots * gt * 2 * sizeof(float), 256);
    p.logits = p.slots + round_up(slots * gt * d * sizeof(float), 256);
    p.bytes = p.logits + (weights ? round_up((size_t)S * Hq * logit_rows(cap) * sizeof(float), 256) : 0);
    return p;
}
static inline size_t paged_attend_workspace_bytes(bool bf16, int S, int Hkv, int Hq, int cap, int d, bool weights)
{
    return paged_whole_heads(S, Hkv, Hq, cap, weights) ? 0 : paged_attend_space(bf16, S, Hkv, Hq, cap, d, weights).bytes;
}

// Per KV head of a sequence: how many rows move, and from where to where.
static inline int paged_evict_moves(int cap, int keep) { return keep >= cap ? 1 : (keep < cap - keep ? keep : cap - keep); }
// Rows of a head whose choice one workgroup makes: as many as its registers hold.  us, so / by workgroups of kChunk rows, bf16, d = 64, to
// half and to 97 % of the rows:
//     heads        2                         16                        128                       1600
//     2048 rows    14 / 27,  10 / 25         15 / 27,  11 / 26         18 / 33,  11 / 28         106 / 168,  27 / 100
//     8192         16 / 27,  18 / 28         18 / 29,  18 / 28         45 / 58,  20 / 36         472 / 512, 145 / 228
//     16384        24 / 28,  25 / 29         29 / 33,  26 / 31         81 / 93,  33 / 48         946 / 1026, 295 / 463
constexpr int kPickRows = 16384;
constexpr int kChunk = 4096;                // rows per workgroup of longer ones
// (one more than the rows fill, because no chunk has rows on both sides of `keep`)
static inline int paged_evict_chunks(int cap) { return cap <= kPickRows ? 0 : (cap + kChunk - 1) / kChunk + 1; }
struct PagedEvictSpace {
    size_t moves, keys, hist, cells, above, bytes;           // offsets, total; the counts of moves lie at 0
};
static inline PagedEvictSpace paged_evict_space(int S, int Hkv, int cap, int keep)
{
    PagedEvictSpace p;
    const size_t pairs = (size_t)S * Hkv, chunks = pairs * paged_evict_chunks(cap);
    p.moves = round_up(pairs * sizeof(int32_t), 256);
    p.keys = p.moves + round_up(pairs * paged_evict_moves(cap, keep) * 2 * sizeof(int32_t), 256);
    p.hist = p.keys + (chunks ? round_up(pairs * cap * sizeof(uint32_t), 256) : 0);
    p.cells = p.hist + chunks * 3 * 2048 * sizeof(uint16_t);
    p.above = p.cells + (chunks ? round_up(pairs * 2 * 8, 256) : 0);
    p.bytes = p.above + round_up(chunks * 4, 256);
    return p;
}
static inline size_t paged_evict_workspace_bytes(int S, int Hkv, int cap, int keep) { return paged_evict_space(S, Hkv, cap, keep).bytes; }

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
