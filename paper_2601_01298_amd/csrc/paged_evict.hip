// Eviction by accumulated attention weight.
//
// Every row's account becomes a 32-bit key that orders like it (protected rows above all numbers, a NaN below).  The keep-th
// largest key of a head is found in three digits from the top, 11, 11 and 10 bits: count the values of a digit among the keys
// that agree so far, and take the value at which the counts from above reach what is left to keep.  Who has a larger key
// stays, and of equal ones the lowest rows; then the rows that became free below `keep` and those that stay behind it are
// listed in order, and row i of one list goes to row i of the other.
//
//   evict_pick   one workgroup per head, keys in registers: up to kPickRows rows.  With few moves it makes them too.
//   evict_chunks (four times)   the same over workgroups of kChunk rows each, for longer heads: a step
//                that needs all chunks of a head (the counts of a digit, the rows listed before a chunk's) starts with a new
//                launch and adds up what the chunks left, so nothing waits inside a kernel and nothing is added atomically
//                between workgroups.
//   evict_move   copies the rows of K and V, accounts and stamps from and to where the lists say.
// Bound: HBM (the moved rows: 8 heads of 131072 rows to 32768, 201 MB in 45 us, 4.4 TB/s); for short heads the chain of barriers of evict_pick
// (1600 heads of 1056 rows to 1024: 21 us, 59 MB), for long ones the launches (7.2, 7.6, 7.7
// and 12.5 us).
#include <type_traits>

#include "paged_internal.h"

namespace ws {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

namespace {

constexpr int kDigits[3] = {11, 11, 10};
constexpr int kBins = 2048;                 // room for a digit's counts

struct EvictArgs {
    void *K, *V;
    const int32_t *table, *len;
    int pages, H, page_shift, S, per_seq, row_bytes;
    int keep, sinks, recent;
    const int32_t *seen, *stamp_in;
    const float *mass_in;
    float *mass_out;
    int32_t *stamp_out, *len_out, *kept;
    int32_t *count, *moves;                 // [pairs], [pairs][2][most]
    int most, chunks;
    uint32_t *keys;                         // [pairs][cap]
    uint16_t *hist;                         // [3][pairs][chunks][kBins]
    uint2 *cells;                           // [2][pairs]: the digits found so far, and how many rows with exactly them are kept
    int32_t *above;                         // [pairs][chunks]: keys above all that start with the first two digits
    __device__ int rows_of(int s) const { return paged_rows(len[s], per_seq << page_shift); }
    __device__ int cap() const { return per_seq << page_shift; }
    __device__ uint16_t *hist_of(int digit, int pair, int chunk) const
    {
        return hist + (((long long)digit * S * H + pair) * chunks + chunk) * kBins;
    }
};

// Orders as the accounts do: NaN least, protected rows above all numbers.
__device__ __forceinline__ uint32_t key_of(float mass, int stamp, int sinks, long long fresh)
{
    if (stamp < sinks || stamp >= fresh) return 0xFFFFFFFFu;
    if (mass != mass) return 0u;
    const uint32_t u = __float_as_uint(mass + 0.0f);             // -0 is 0
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ uint32_t wave_scan(uint32_t v)       // inclusive
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(v, o);
        if ((int)(threadIdx.x & 63) >= o) v += y;
    }
    return v;
}

__device__ __forceinline__ int below(unsigned long long mask)   // set bits of lower lanes
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// The digit at which counts from the largest value down reach `left`.  Thread t holds PER counts, of the values PER (THREADS - 1 - t)
// and up.  Returned to all: the digit, and `left` less what lies above it.  Two barriers.
template <int THREADS, int PER>
__device__ __forceinline__ int find_digit(const uint32_t (&c)[PER], uint32_t &left, uint32_t *wave_sum, uint32_t *found)
{
    const int tid = threadIdx.x;
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) mine += c[i];
    const uint32_t upto = wave_scan(mine);
    if ((tid & 63) == 63) wave_sum[tid >> 6] = upto;
    __syncthreads();
    uint32_t above = upto - mine;
#pragma unroll
    for (int w = 0; w < THREADS / 64 - 1; ++w)
        if (w < tid >> 6) above += wave_sum[w];
    if (above < left && left <= above + mine) {
        int digit = PER * (THREADS - 1 - tid);
        uint32_t over = above;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i) {
            if (above < left && left <= above + c[i]) {
                digit += i;
                over = above;
            }
            above += c[i];
        }
        found[0] = (uint32_t)digit;
        found[1] = left - over;
    }
    __syncthreads();
    left = found[1];
    return (int)found[0];
}

// Copies move j .. of a head with the threads of a group of `pieces`: rows of K and V 16 bytes a thread, U moves at a time, and by the
// first thread the account, the stamp and the note of where the row came from.
template <int U>
__device__ __forceinline__ void move_rows(const EvictArgs &a, int pair, const int32_t *free_rows, const int32_t *movers, int count, int group,
                                          int groups, int piece)
{
    const int s = pair / a.H, h = pair % a.H, pmask = (1 << a.page_shift) - 1;
    const int32_t *table = a.table + (long long)s * a.per_seq;
    const long long at = (long long)pair * a.cap();
    for (int j0 = group; j0 < count; j0 += groups * U) {
        int to[U], from[U], to_page[U], from_page[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = min(j0 + u * groups, count - 1);
            to[u] = free_rows[j];
            from[u] = movers[j];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            to_page[u] = table[to[u] >> a.page_shift];
            from_page[u] = table[from[u] >> a.page_shift];
        }
        u32x4_t k[U], v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long src = (paged_base(from_page[u], a.pages, a.H, h, 1 << a.page_shift) + (from[u] & pmask)) * a.row_bytes + piece * 16;
            k[u] = *reinterpret_cast<const u32x4_t *>(reinterpret_cast<const char *>(a.K) + src);
            v[u] = *reinterpret_cast<const u32x4_t *>(reinterpret_cast<const char *>(a.V) + src);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool there = j0 + u * groups < count;
            if (there && (unsigned)to_page[u] < (unsigned)a.pages) {
                const long long dst = (paged_base(to_page[u], a.pages, a.H, h, 1 << a.page_shift) + (to[u] & pmask)) * a.row_bytes + piece * 16;
                __builtin_nontemporal_store(k[u], reinterpret_cast<u32x4_t *>(reinterpret_cast<char *>(a.K) + dst));
                __builtin_nontemporal_store(v[u], reinterpret_cast<u32x4_t *>(reinterpret_cast<char *>(a.V) + dst));
            }
            if (there && piece == 0) {
                a.mass_out[at + to[u]] = a.mass_in[at + from[u]];
                a.stamp_out[at + to[u]] = a.stamp_in[at + from[u]];
                if (a.kept != nullptr) a.kept[(long long)pair * a.keep + to[u]] = from[u];
            }
        }
    }
}

// A row that stays where it is: its account and stamp where they are wanted elsewhere.
__device__ __forceinline__ void leave_row(const EvictArgs &a, int pair, int i, float mass, int stamp)
{
    const long long at = (long long)pair * a.cap() + i;
    if (a.mass_out != a.mass_in) a.mass_out[at] = mass;
    if (a.stamp_out != a.stamp_in) a.stamp_out[at] = stamp;
    if (a.kept != nullptr) a.kept[(long long)pair * a.keep + i] = i;
}

constexpr int kMoveRows = 4;                // rows a thread of evict_move has on their way at once
// Moves of a head that evict_pick makes itself.  us, in the same launch / in one of their own, heads of 2016 rows, bf16:
//     moves               32           64           128          256          512
//     2 heads, d = 64      9 / 12      10 / 13      12 / 13      12 / 13      16 / 14
//     128 heads, d = 64   10 / 13      10 / 13      12 / 15      16 / 15      20 / 17
//     128, d = 128        11 / 13      12 / 14      16 / 15      22 / 17      31 / 22
//     1600, d = 128       26 / 33      37 / 42      55 / 58     103 / 104    168 / 154
constexpr int kInlineMoves = 128;

// Wave w has rows 64 KPT w and up, KPT runs of 64: the order of rows is the order of waves, runs and lanes.
template <int THREADS, int KPT, bool MOVE>
__global__ void __launch_bounds__(THREADS)
evict_pick(EvictArgs a)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ __attribute__((aligned(16))) uint32_t hist[kBins];
    __shared__ uint32_t wave_sum[WAVES], found[2];
    __shared__ int wave_ties[WAVES], wave_free[WAVES], wave_move[WAVES];
    __shared__ int32_t lists[2][MOVE ? kInlineMoves : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int pair = blockIdx.x, s = pair / a.H;
    const int n = a.rows_of(s);
    if (MOVE && pair % a.H == 0 && tid == 0 && a.len_out != a.len) a.len_out[s] = min(n, a.keep);
    const int row0 = wave * 64 * KPT + lane;
    const long long at = (long long)pair * a.cap(), fresh = (long long)a.seen[s] - a.recent;
    float mass[KPT];
    int stamp[KPT];
#pragma unroll
    for (int k = 0; k < KPT; ++k) {
        const int i = max(0, min(row0 + k * 64, n - 1));
        mass[k] = a.mass_in[at + i];
        stamp[k] = a.stamp_in[at + i];
    }
    if (n <= a.keep) {
        if (!MOVE && tid == 0) a.count[pair] = 0;
#pragma unroll
        for (int k = 0; k < KPT; ++k)
            if (row0 + k * 64 < n) leave_row(a, pair, row0 + k * 64, mass[k], stamp[k]);
        return;
    }
    for (int i = tid; i < kBins; i += THREADS) hist[i] = 0;
    __syncthreads();
    uint32_t key[KPT];
#pragma unroll
    for (int k = 0; k < KPT; ++k) key[k] = key_of(mass[k], stamp[k], a.sinks, fresh);
    uint32_t prefix = 0, left = (uint32_t)a.keep;
    int shift = 32;
#pragma unroll
    for (int digit = 0; digit < 3; ++digit) {
        const uint32_t known = digit == 0 ? 0u : 0xFFFFFFFFu << shift;
        shift -= kDigits[digit];
#pragma unroll
        for (int k = 0; k < KPT; ++k)
            if (row0 + k * 64 < n && (key[k] & known) == prefix) atomicAdd(&hist[(key[k] >> shift) & ((1 << kDigits[digit]) - 1)], 1u);
        __syncthreads();
        constexpr int PER = kBins / THREADS;
        uint32_t c[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            c[i] = hist[PER * (THREADS - 1 - tid) + i];
            hist[PER * (THREADS - 1 - tid) + i] = 0;             // for the next digit, which waits for find_digit's barriers
        }
        prefix |= (uint32_t)find_digit<THREADS, PER>(c, left, wave_sum, found) << shift;
    }
    // rows with a larger key stay, and of those with this one the first `left`
    int ties = 0;
#pragma unroll
    for (int k = 0; k < KPT; ++k) ties += __popcll(__ballot(row0 + k * 64 < n && key[k] == prefix));
    if (lane == 0) wave_ties[wave] = ties;
    __syncthreads();
    ties = 0;
#pragma unroll
    for (int w = 0; w < WAVES - 1; ++w)
        if (w < wave) ties += wave_ties[w];
    uint32_t stays = 0;                                          // bit k: row k of this lane
    int nfree = 0, nmove = 0;
#pragma unroll
    for (int k = 0; k < KPT; ++k) {
        const int i = row0 + k * 64;
        const bool tie = i < n && key[k] == prefix;
        const unsigned long long mask = __ballot(tie);
        const bool stay = i < n && (key[k] > prefix || (tie && ties + below(mask) < (int)left));
        ties += __popcll(mask);
        if (stay) stays |= 1u << k;
        nfree += __popcll(__ballot(i < a.keep && !stay));
        nmove += __popcll(__ballot(i >= a.keep && stay));
    }
    if (lane == 0) {
        wave_free[wave] = nfree;
        wave_move[wave] = nmove;
    }
    __syncthreads();
    int all = 0;
    nfree = nmove = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) {
            nfree += wave_free[w];
            nmove += wave_move[w];
        }
        all += wave_free[w];
    }
    int32_t *free_rows = MOVE ? lists[0] : a.moves + (long long)pair * 2 * a.most, *movers = MOVE ? lists[1] : free_rows + a.most;
#pragma unroll
    for (int k = 0; k < KPT; ++k) {
        const int i = row0 + k * 64;
        const bool stay = (stays >> k) & 1u, is_free = i < a.keep && !stay, moves = i >= a.keep && stay;
        const unsigned long long fm = __ballot(is_free), mm = __ballot(moves);
        if (is_free) free_rows[nfree + below(fm)] = i;
        if (moves) movers[nmove + below(mm)] = i;
        nfree += __popcll(fm);
        nmove += __popcll(mm);
        if (stay && !moves) leave_row(a, pair, i, mass[k], stamp[k]);
    }
    if constexpr (MOVE) {
        __syncthreads();
        const int pieces = a.row_bytes / 16;
        move_rows<2>(a, pair, free_rows, movers, all, tid / pieces, THREADS / pieces, tid % pieces);
    } else {
        if (tid == 0) a.count[pair] = all;
    }
}

__global__ void __launch_bounds__(256)
evict_lengths(EvictArgs a)
{
    const int s = blockIdx.x * 256 + threadIdx.x;
    if (s < a.S) a.len_out[s] = min(a.rows_of(s), a.keep);
}

// ---- heads of more rows: a workgroup per chunk ------------------------------------------------------------------------------
constexpr int kChunkKeys = kChunk / 256;    // per thread

// The rows of a head in chunks: first those below `keep`, then those behind, so that a chunk has rows of one kind only.
struct Chunks {
    int n, keep, low, all;                  // chunks below `keep`, chunks
    __device__ __forceinline__ Chunks(int rows, int k)
        : n(rows), keep(k), low((min(rows, k) + kChunk - 1) / kChunk), all(low + (max(0, rows - k) + kChunk - 1) / kChunk)
    {
    }
    __device__ __forceinline__ int base(int c) const { return c < low ? c * kChunk : keep + (c - low) * kChunk; }
    __device__ __forceinline__ int end(int c) const { return min(c < low ? min(keep, n) : n, base(c) + kChunk); }
};
// Row k of a thread in the chunk that starts at `base`: the order of rows is the order of waves, runs of 64 and lanes.
__device__ __forceinline__ int chunk_row(int base, int k) { return base + (threadIdx.x >> 6) * (kChunk / 4) + k * 64 + (threadIdx.x & 63); }

// The value of digit `d` from the counts that all chunks of the head left; `left` as in find_digit.
template <int BINS>
__device__ __forceinline__ int digit_of_chunks(const EvictArgs &a, int d, int pair, int chunks, uint32_t &left, uint32_t *wave_sum, uint32_t *found)
{
    constexpr int PER = BINS / 256;
    const uint16_t *h = a.hist_of(d, pair, 0) + PER * (255 - (int)threadIdx.x);
    uint32_t c[PER] = {};
#pragma unroll 8
    for (int i = 0; i < chunks; ++i) {
        uint32_t w[PER / 2];
        if constexpr (PER == 8) {
            const uint4 x = *reinterpret_cast<const uint4 *>(h + (long long)i * kBins);
            w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
        } else {
            const uint2 x = *reinterpret_cast<const uint2 *>(h + (long long)i * kBins);
            w[0] = x.x, w[1] = x.y;
        }
#pragma unroll
        for (int j = 0; j < PER / 2; ++j) {
            c[2 * j] += w[j] & 0xFFFFu;
            c[2 * j + 1] += w[j] >> 16;
        }
    }
    return find_digit<256, PER>(c, left, wave_sum, found);
}

template <int DIGIT>
__device__ __forceinline__ void digit_of_chunk(const EvictArgs &a, int pair, const Chunks &chunks, int chunk)
{
    __shared__ uint32_t hist[kBins];
    __shared__ uint32_t wave_sum[4], found[2];
    __shared__ int wave_above[4];
    const int tid = threadIdx.x, base = chunks.base(chunk), end = chunks.end(chunk);
    const long long at = (long long)pair * a.cap();
    if (chunks.n <= a.keep) {
        if (DIGIT == 0)
#pragma unroll 8
            for (int k = 0; k < kChunkKeys; ++k) {
                const int i = chunk_row(base, k);
                if (i < end) leave_row(a, pair, i, a.mass_in[at + i], a.stamp_in[at + i]);
            }
        return;
    }
    uint32_t key[kChunkKeys];
    if constexpr (DIGIT == 0) {
        const long long fresh = (long long)a.seen[pair / a.H] - a.recent;
        float mass[kChunkKeys];
        int stamp[kChunkKeys];
#pragma unroll
        for (int k = 0; k < kChunkKeys; ++k) {
            const int i = min(chunk_row(base, k), end - 1);
            mass[k] = a.mass_in[at + i];
            stamp[k] = a.stamp_in[at + i];
        }
#pragma unroll
        for (int k = 0; k < kChunkKeys; ++k) key[k] = key_of(mass[k], stamp[k], a.sinks, fresh);
    } else {
#pragma unroll
        for (int k = 0; k < kChunkKeys; ++k) key[k] = a.keys[at + min(chunk_row(base, k), end - 1)];
    }
    for (int i = tid; i < kBins; i += 256) hist[i] = 0;
    uint32_t prefix = 0, left = (uint32_t)a.keep;
    if constexpr (DIGIT > 0) {
        if constexpr (DIGIT == 2) {
            const uint2 cell = a.cells[pair];
            prefix = cell.x, left = cell.y;
        }
        prefix |= (uint32_t)digit_of_chunks<kBins>(a, DIGIT - 1, pair, chunks.all, left, wave_sum, found) << (DIGIT == 1 ? 21 : 10);
        if (chunk == 0 && tid == 0) a.cells[(long long)(DIGIT - 1) * a.S * a.H + pair] = make_uint2(prefix, left);
    }
    __syncthreads();
    constexpr int SHIFT = DIGIT == 0 ? 21 : DIGIT == 1 ? 10 : 0;
    constexpr uint32_t KNOWN = DIGIT == 0 ? 0u : DIGIT == 1 ? 0xFFFFFFFFu << 21 : 0xFFFFFFFFu << 10;
#pragma unroll
    for (int k = 0; k < kChunkKeys; ++k)
        if (chunk_row(base, k) < end) {
            if (DIGIT == 0) a.keys[at + chunk_row(base, k)] = key[k];
            if ((key[k] & KNOWN) == prefix) atomicAdd(&hist[(key[k] >> SHIFT) & ((1 << kDigits[DIGIT]) - 1)], 1u);
        }
    if constexpr (DIGIT == 2) {
        int more = 0;
#pragma unroll
        for (int k = 0; k < kChunkKeys; ++k) more += __popcll(__ballot(chunk_row(base, k) < end && key[k] > (prefix | 1023u)));
        if ((tid & 63) == 0) wave_above[tid >> 6] = more;
    }
    __syncthreads();
    if (DIGIT == 2 && tid == 0) a.above[(long long)pair * a.chunks + chunk] = wave_above[0] + wave_above[1] + wave_above[2] + wave_above[3];
    uint32_t *out = reinterpret_cast<uint32_t *>(a.hist_of(DIGIT, pair, chunk));
    for (int i = tid; i < (1 << kDigits[DIGIT]) / 2; i += 256) out[i] = hist[2 * i] | hist[2 * i + 1] << 16;
}

// Who stays, the lists of free rows and of rows that move, in order, and the accounts of those that are neither.  Of the chunks before
// this one no more is needed than how many of their keys lie above the threshold and how many at it: of the latter the first `left` of the
// head stay, so min(left, how many there were) of them have.
__device__ __forceinline__ void place_chunk(const EvictArgs &a, int pair, const Chunks &chunks, int chunk)
{
    __shared__ uint32_t wave_sum[4], found[2];
    __shared__ int sums[4][4], wave_ties[4], wave_listed[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, base = chunks.base(chunk), end = chunks.end(chunk);
    if (chunks.n <= a.keep) {
        if (chunk == 0 && tid == 0) a.count[pair] = 0;
        return;
    }
    const bool low = chunk < chunks.low, elsewhere = a.mass_out != a.mass_in || a.stamp_out != a.stamp_in;
    const long long at = (long long)pair * a.cap();
    uint32_t key[kChunkKeys];
    float mass[kChunkKeys];
    int stamp[kChunkKeys];
#pragma unroll
    for (int k = 0; k < kChunkKeys; ++k) key[k] = a.keys[at + min(chunk_row(base, k), end - 1)];
    if (low && elsewhere)
#pragma unroll
        for (int k = 0; k < kChunkKeys; ++k) {
            const int i = min(chunk_row(base, k), end - 1);
            mass[k] = a.mass_in[at + i];
            stamp[k] = a.stamp_in[at + i];
        }
    const uint2 cell = a.cells[(long long)a.S * a.H + pair];
    uint32_t left = cell.y;
    const int digit = digit_of_chunks<kBins / 2>(a, 2, pair, chunks.all, left, wave_sum, found);
    const uint32_t threshold = cell.x | (uint32_t)digit;
    // keys above the threshold and at it in the chunks before this one, and in those below `keep`
    int before[2] = {0, 0}, lower[2] = {0, 0};                   // of this lane's values of the last digit
#pragma unroll 4
    for (int c = wave; c < max(chunk, chunks.low); c += 4) {
        const uint16_t *h = a.hist_of(2, pair, c);
        int over = lane == 0 ? a.above[(long long)pair * a.chunks + c] : 0, equal = 0;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint4 x = reinterpret_cast<const uint4 *>(h)[2 * lane + half];
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int bin = 16 * lane + 8 * half + i, n = (int)((w[i / 2] >> (16 * (i & 1))) & 0xFFFFu);
                if (bin > digit) over += n;
                if (bin == digit) equal += n;
            }
        }
        if (c < chunk) before[0] += over, before[1] += equal;
        if (c < chunks.low) lower[0] += over, lower[1] += equal;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        before[0] += __shfl_xor(before[0], o);
        before[1] += __shfl_xor(before[1], o);
        lower[0] += __shfl_xor(lower[0], o);
        lower[1] += __shfl_xor(lower[1], o);
    }
    int ties = 0;
#pragma unroll
    for (int k = 0; k < kChunkKeys; ++k) ties += __popcll(__ballot(chunk_row(base, k) < end && key[k] == threshold));
    if (lane == 0) {
        sums[wave][0] = before[0], sums[wave][1] = before[1], sums[wave][2] = lower[0], sums[wave][3] = lower[1];
        wave_ties[wave] = ties;
    }
    __syncthreads();
    int sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = sums[0][i] + sums[1][i] + sums[2][i] + sums[3][i];
    const int kept_before = sum[0] + min((int)left, sum[1]), kept_low = sum[2] + min((int)left, sum[3]);
    if (chunk == 0 && tid == 0) a.count[pair] = a.keep - kept_low;
    ties = sum[1];
#pragma unroll
    for (int w = 0; w < 3; ++w)
        if (w < wave) ties += wave_ties[w];
    uint32_t stays = 0;                                          // bit k: row k of this lane
    int listed = 0;
#pragma unroll
    for (int k = 0; k < kChunkKeys; ++k) {
        const bool there = chunk_row(base, k) < end, tie = there && key[k] == threshold;
        const unsigned long long mask = __ballot(tie);
        const bool stay = there && (key[k] > threshold || (tie && ties + below(mask) < (int)left));
        ties += __popcll(mask);
        if (stay) stays |= 1u << k;
        listed += __popcll(__ballot(there && stay != low));
    }
    if (lane == 0) wave_listed[wave] = listed;
    __syncthreads();
    // a chunk below `keep` lists those that go, a chunk behind it those that stay
    listed = low ? chunk * kChunk - kept_before : kept_before - kept_low;
#pragma unroll
    for (int w = 0; w < 3; ++w)
        if (w < wave) listed += wave_listed[w];
    int32_t *list = a.moves + ((long long)pair * 2 + (low ? 0 : 1)) * a.most;
#pragma unroll
    for (int k = 0; k < kChunkKeys; ++k) {
        const int i = chunk_row(base, k);
        const bool there = i < end, stay = (stays >> k) & 1u, mine = there && stay != low;
        const unsigned long long mask = __ballot(mine);
        if (mine) list[listed + below(mask)] = i;
        listed += __popcll(mask);
        if (low && stay) leave_row(a, pair, i, mass[k], stamp[k]);
    }
}

// The steps over chunks.  The lengths are on the device, so a grid made for the longest cache there can be would be mostly empty: a head has
// gridDim.x workgroups, which take its chunks in turn.  STEP 0 to 2: the digits, 3: who stays, and the lists.
template <int STEP>
__global__ void __launch_bounds__(256)
evict_chunks(EvictArgs a)
{
    const int pair = blockIdx.y + blockIdx.z * gridDim.y;
    if (pair >= a.S * a.H) return;
    const Chunks chunks(a.rows_of(pair / a.H), a.keep);
    if (STEP == 3 && chunks.all == 0 && blockIdx.x == 0 && threadIdx.x == 0) a.count[pair] = 0;
    for (int chunk = blockIdx.x; chunk < chunks.all; chunk += gridDim.x) {
        if constexpr (STEP < 3) digit_of_chunk<STEP>(a, pair, chunks, chunk);
        else place_chunk(a, pair, chunks, chunk);
        if (chunk + (int)gridDim.x < chunks.all) __syncthreads();
    }
}

__global__ void __launch_bounds__(256)
evict_move(EvictArgs a)
{
    const int pair = blockIdx.y + blockIdx.z * gridDim.y;
    if (pair >= a.S * a.H) return;
    // (nothing else here looks at the lengths: len_out may be where they came from)
    if (blockIdx.x == 0 && pair % a.H == 0 && threadIdx.x == 0) a.len_out[pair / a.H] = min(a.rows_of(pair / a.H), a.keep);
    const int32_t *free_rows = a.moves + (long long)pair * 2 * a.most;
    const int pieces = a.row_bytes / 16, per = 256 / pieces;
    move_rows<kMoveRows>(a, pair, free_rows, free_rows + a.most, a.count[pair], blockIdx.x * per + threadIdx.x / pieces, gridDim.x * per,
                 threadIdx.x % pieces);
}

}  // namespace

hipError_t launch_paged_evict(const ws_paged_cache &c, int keep, int sinks, int recent, const int32_t *seen, const float *mass_in,
                              float *mass_out, const int32_t *stamp_in, int32_t *stamp_out, int32_t *len_out, int32_t *kept,
                              void *ws, hipStream_t st)
{
    const int cap = c.per_seq * c.page, pairs = c.S * c.Hkv;
    const PagedEvictSpace sp = paged_evict_space(c.S, c.Hkv, cap, keep);
    char *base = reinterpret_cast<char *>(ws);
    EvictArgs a = {};
    a.K = c.K, a.V = c.V, a.table = c.table, a.len = c.len;
    a.pages = c.pages, a.H = c.Hkv, a.page_shift = __builtin_ctz((unsigned)c.page), a.S = c.S, a.per_seq = c.per_seq;
    a.row_bytes = c.d * (c.dt == WS_BF16 ? 2 : 4);
    a.keep = keep, a.sinks = sinks, a.recent = recent;
    a.seen = seen, a.stamp_in = stamp_in, a.mass_in = mass_in;
    a.mass_out = mass_out, a.stamp_out = stamp_out, a.len_out = len_out, a.kept = kept;
    a.most = paged_evict_moves(cap, keep), a.chunks = paged_evict_chunks(cap);
    a.count = reinterpret_cast<int32_t *>(base);
    a.moves = reinterpret_cast<int32_t *>(base + sp.moves);
    a.keys = reinterpret_cast<uint32_t *>(base + sp.keys);
    a.hist = reinterpret_cast<uint16_t *>(base + sp.hist);
    a.cells = reinterpret_cast<uint2 *>(base + sp.cells);
    a.above = reinterpret_cast<int32_t *>(base + sp.above);
    const int y = pairs < 32768 ? pairs : 32768, z = (pairs + y - 1) / y;
    if (cap <= kPickRows) {
        const bool move = a.most <= kInlineMoves;
        const dim3 grid((unsigned)pairs);
        auto pick = [&](auto threads, auto keys) {
            constexpr int T = decltype(threads)::value, N = decltype(keys)::value;
            if (move) hipLaunchKernelGGL((evict_pick<T, N, true>), grid, dim3(T), 0, st, a);
            else hipLaunchKernelGGL((evict_pick<T, N, false>), grid, dim3(T), 0, st, a);
        };
        using std::integral_constant;
        if (cap <= 2048) pick(integral_constant<int, 256>(), integral_constant<int, 8>());
        else if (cap <= 8192) pick(integral_constant<int, 1024>(), integral_constant<int, 8>());
        else pick(integral_constant<int, 1024>(), integral_constant<int, 16>());
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (move) {
            // where the new lengths replace the old ones they wait until every head has read them
            if (len_out == c.len) hipLaunchKernelGGL(evict_lengths, dim3((unsigned)((c.S + 255) / 256)), dim3(256), 0, st, a);
            return hipGetLastError();
        }
    } else {
        const int share = 4096 / pairs > 1 ? 4096 / pairs : 1;
        const dim3 grid((unsigned)(a.chunks < share ? a.chunks : share), (unsigned)y, (unsigned)z), block(256);
        hipLaunchKernelGGL((evict_chunks<0>), grid, block, 0, st, a);
        hipLaunchKernelGGL((evict_chunks<1>), grid, block, 0, st, a);
        hipLaunchKernelGGL((evict_chunks<2>), grid, block, 0, st, a);
        hipLaunchKernelGGL((evict_chunks<3>), grid, block, 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int per = 256 / (a.row_bytes / 16) * kMoveRows;
    const long long want = (a.most + per - 1) / per, share = 8192 / pairs > 1 ? 8192 / pairs : 1;
    hipLaunchKernelGGL(evict_move, dim3((unsigned)(want < share ? want : share), (unsigned)y, (unsigned)z), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace ws
