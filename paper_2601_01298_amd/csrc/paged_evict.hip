// Eviction by accumulated attention weight.
//
// evict_pick: one workgroup per KV head of a sequence.  Every row's account becomes a 32-bit number that orders like it (protected
// rows above all); the keep-th largest is found digit by digit from the top (counts of the 256 values of a digit among the rows
// that agree so far), then one ordered pass tells who stays, who of those has to move (it lies at `keep` or behind) and which
// rows became free, and writes the accounts and stamps.  evict_move: copies the rows of K and V from and to where evict_pick says.
#include "paged_internal.h"

namespace ws {

namespace {

constexpr int kPick = 1024;

struct EvictArgs {
    void *K, *V;
    const int32_t *table, *len;
    int pages, H, page, S, per_seq, row_bytes;
    int keep, sinks, recent;
    const int32_t *seen, *stamp_in;
    const float *mass_in;
    float *mass_out;
    int32_t *stamp_out, *len_out, *kept;
    int32_t *count, *moves;      // [pairs], [pairs][2][most]
    int most;
};

// Orders as the accounts do: NaN least, protected rows above all numbers.
__device__ __forceinline__ uint32_t rank_of(float mass, int stamp, int sinks, long long fresh)
{
    if (stamp < sinks || stamp >= fresh) return 0xFFFFFFFFu;
    if (mass != mass) return 0u;
    const uint32_t u = __float_as_uint(mass + 0.0f);             // -0 is 0
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Exclusive sum over the workgroup of v; `total` is the whole.  Two barriers.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *wave_sum, uint32_t &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    if (lane == 63) wave_sum[wave] = x;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (int w = 0; w < kPick / 64; ++w) {
        const uint32_t c = wave_sum[w];
        if (w < wave) before += c;
        all += c;
    }
    __syncthreads();
    total = all;
    return before + x - v;
}

__global__ void __launch_bounds__(kPick)
evict_pick(EvictArgs a)
{
    __shared__ uint32_t hist[256];
    __shared__ uint32_t wave_sum[kPick / 64];
    __shared__ uint32_t found[2];
    const int tid = threadIdx.x, pair = blockIdx.x, s = pair / a.H;
    const int cap = a.per_seq * a.page;
    const int n = paged_rows(a.len[s], cap);
    const float *mass = a.mass_in + (long long)pair * cap;
    const int32_t *stamp = a.stamp_in + (long long)pair * cap;
    float *mass_out = a.mass_out + (long long)pair * cap;
    int32_t *stamp_out = a.stamp_out + (long long)pair * cap;
    int32_t *kept = a.kept != nullptr ? a.kept + (long long)pair * a.keep : nullptr;
    if (n <= a.keep) {
        if (tid == 0) a.count[pair] = 0;
        for (int i = tid; i < n; i += kPick) {
            mass_out[i] = mass[i];
            stamp_out[i] = stamp[i];
            if (kept != nullptr) kept[i] = i;
        }
        return;
    }
    const long long fresh = (long long)a.seen[s] - a.recent;
    uint32_t prefix = 0, left = (uint32_t)a.keep;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        const uint32_t known = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
        for (int i = tid; i < n; i += kPick) {
            const uint32_t key = rank_of(mass[i], stamp[i], a.sinks, fresh);
            if ((key & known) == prefix) atomicAdd(&hist[(key >> shift) & 255], 1u);
        }
        __syncthreads();
        // thread t < 256 holds digit 255 - t, so that sums run from the largest down
        const uint32_t c = tid < 256 ? hist[255 - tid] : 0u;
        uint32_t total;
        const uint32_t above = block_scan(c, wave_sum, total);
        if (tid < 256 && above < left && left <= above + c) {
            found[0] = 255 - tid;
            found[1] = above;
        }
        __syncthreads();
        prefix |= found[0] << shift;
        left -= found[1];
        __syncthreads();
    }
    // rows above the threshold stay, and of those at it the first `left`
    int32_t *free_rows = a.moves + (long long)pair * 2 * a.most, *movers = free_rows + a.most;
    uint32_t ties = 0, nfree = 0, nmove = 0;
    for (int i0 = 0; i0 < n; i0 += kPick) {
        const int i = i0 + tid;
        float m = 0.0f;
        int st = 0;
        uint32_t key = 0;
        if (i < n) {
            m = mass[i];
            st = stamp[i];
            key = rank_of(m, st, a.sinks, fresh);
        }
        const bool tie = i < n && key == prefix;
        uint32_t total;
        const uint32_t rank = block_scan(tie ? 1u : 0u, wave_sum, total);
        const bool stays = i < n && (key > prefix || (tie && ties + rank < left));
        ties += total;
        const bool hole = i < n && i < a.keep && !stays, mover = stays && i >= a.keep;
        const uint32_t at = block_scan((hole ? 1u : 0u) | (mover ? 0x10000u : 0u), wave_sum, total);
        if (hole) free_rows[nfree + (at & 0xFFFFu)] = i;
        if (mover) movers[nmove + (at >> 16)] = i;
        nfree += total & 0xFFFFu;
        nmove += total >> 16;
        if (stays && i < a.keep) {
            mass_out[i] = m;
            stamp_out[i] = st;
            if (kept != nullptr) kept[i] = i;
        }
    }
    __syncthreads();
    for (uint32_t j = tid; j < nfree; j += kPick) {
        const int to = free_rows[j], from = movers[j];
        mass_out[to] = mass[from];
        stamp_out[to] = stamp[from];
        if (kept != nullptr) kept[to] = from;
    }
    if (tid == 0) a.count[pair] = (int)nfree;
}

__global__ void __launch_bounds__(256)
evict_move(EvictArgs a)
{
    const int pair = blockIdx.y + blockIdx.z * gridDim.y;
    if (pair >= a.S * a.H) return;
    const int s = pair / a.H, h = pair % a.H;
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) a.len_out[s] = min(paged_rows(a.len[s], a.per_seq * a.page), a.keep);
    const int count = a.count[pair];
    const int32_t *free_rows = a.moves + (long long)pair * 2 * a.most, *movers = free_rows + a.most;
    const int32_t *table = a.table + (long long)s * a.per_seq;
    const int pieces = a.row_bytes / 16;
    for (long long i = blockIdx.x * 256 + threadIdx.x; i < (long long)count * 2 * pieces; i += (long long)gridDim.x * 256) {
        const int j = (int)(i / (2 * pieces)), w = (int)(i % (2 * pieces));
        const int to = free_rows[j], from = movers[j];
        const int to_page = table[to / a.page];
        if ((unsigned)to_page >= (unsigned)a.pages) continue;
        char *pool = reinterpret_cast<char *>(w < pieces ? a.K : a.V);
        const long long src = paged_base(table[from / a.page], a.pages, a.H, h, a.page) + from % a.page;
        const long long dst = paged_base(to_page, a.pages, a.H, h, a.page) + to % a.page;
        *reinterpret_cast<uint4 *>(pool + dst * a.row_bytes + (w % pieces) * 16) =
            *reinterpret_cast<const uint4 *>(pool + src * a.row_bytes + (w % pieces) * 16);
    }
}

}  // namespace

hipError_t launch_paged_evict(const ws_paged_cache &c, int keep, int sinks, int recent, const int32_t *seen, const float *mass_in,
                              float *mass_out, const int32_t *stamp_in, int32_t *stamp_out, int32_t *len_out, int32_t *kept,
                              void *ws, hipStream_t st)
{
    const int cap = c.per_seq * c.page, pairs = c.S * c.Hkv;
    EvictArgs a = {};
    a.K = c.K, a.V = c.V, a.table = c.table, a.len = c.len;
    a.pages = c.pages, a.H = c.Hkv, a.page = c.page, a.S = c.S, a.per_seq = c.per_seq;
    a.row_bytes = c.d * (c.dt == WS_BF16 ? 2 : 4);
    a.keep = keep, a.sinks = sinks, a.recent = recent;
    a.seen = seen, a.stamp_in = stamp_in, a.mass_in = mass_in;
    a.mass_out = mass_out, a.stamp_out = stamp_out, a.len_out = len_out, a.kept = kept;
    a.most = paged_evict_moves(cap, keep);
    a.count = reinterpret_cast<int32_t *>(ws);
    a.moves = reinterpret_cast<int32_t *>(reinterpret_cast<char *>(ws) + round_up((size_t)pairs * sizeof(int32_t), 256));
    hipLaunchKernelGGL(evict_pick, dim3((unsigned)pairs), dim3(kPick), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const long long work = ((long long)a.most * 2 * (a.row_bytes / 16) + 255) / 256;
    const long long share = 4096 / pairs > 1 ? 4096 / pairs : 1;
    const int y = pairs < 32768 ? pairs : 32768, z = (pairs + y - 1) / y;
    hipLaunchKernelGGL(evict_move, dim3((unsigned)(work < share ? work : share), (unsigned)y, (unsigned)z), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace ws
