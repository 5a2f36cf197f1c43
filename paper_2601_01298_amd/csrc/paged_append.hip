// The rows of new tokens join the paged cache: keys and queries rotated to their positions, values copied, the rows' stamps and
// accounts started.
//
// One workgroup per token.  Its d/2 angles are formed once, one per thread (position times frequency in float64, in turns, less
// the whole turns, then the fp32 sine and cosine of half-turns), and wait in LDS for all heads of the token; then a thread
// takes 16 bytes of the lower half of a head's row and the 16 bytes they pair with.  Bound: HBM for prompts (32768 tokens, 8 key and
// 32 query heads of 128, bf16: 808 MB in 137 us, 5.9 TB/s of reads and writes), the launch for a decode step (100 tokens: 4.5 us).
#include "paged_internal.h"

namespace ws {

namespace {

struct AppendArgs {
    void *K, *V;
    const int32_t *table, *len;
    int pages, H, page, S, per_seq;
    const char *k, *v, *q;
    long long k_token, k_head, v_token, v_head, q_token, q_head;     // bytes
    int T, Hq;
    const int32_t *first, *pos, *seen;
    char *q_out;
    int32_t *stamp;
    float *mass;
};

// Past the caches: a prompt is larger than they are (144 us with ordinary stores, 137 with these), and what reads a decode step's rows next
// runs on other dies.
__device__ __forceinline__ void store16(char *p, const uint4 &x)
{
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
    const u32x4_t v = {x.x, x.y, x.z, x.w};
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t *>(p));
}

template <bool BF16>
__device__ __forceinline__ void rotate16(uint4 &lo, uint4 &hi, const float2 *cs)
{
    constexpr int PER = BF16 ? 8 : 4;
    float x0[PER], x1[PER];
    const uint32_t a[4] = {lo.x, lo.y, lo.z, lo.w}, b[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (BF16) {
            x0[2 * j] = __uint_as_float(a[j] << 16);
            x0[2 * j + 1] = __uint_as_float(a[j] & 0xFFFF0000u);
            x1[2 * j] = __uint_as_float(b[j] << 16);
            x1[2 * j + 1] = __uint_as_float(b[j] & 0xFFFF0000u);
        } else {
            x0[j] = __uint_as_float(a[j]);
            x1[j] = __uint_as_float(b[j]);
        }
    }
    float y0[PER], y1[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        y0[e] = x0[e] * cs[e].x - x1[e] * cs[e].y;
        y1[e] = x1[e] * cs[e].x + x0[e] * cs[e].y;
    }
    uint32_t wl[4], wh[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (BF16) {
            wl[j] = bf16_rne(y0[2 * j]) | (bf16_rne(y0[2 * j + 1]) << 16);
            wh[j] = bf16_rne(y1[2 * j]) | (bf16_rne(y1[2 * j + 1]) << 16);
        } else {
            wl[j] = __float_as_uint(y0[j]);
            wh[j] = __float_as_uint(y1[j]);
        }
    }
    lo = make_uint4(wl[0], wl[1], wl[2], wl[3]);
    hi = make_uint4(wh[0], wh[1], wh[2], wh[3]);
}

template <bool BF16, int D>
__global__ void __launch_bounds__(256)
append_tokens(AppendArgs a, RotaryTable rot)
{
    constexpr int ES = BF16 ? 2 : 4, PER = 16 / ES, HALF = D / 2, PP = HALF / PER;     // PP: piece pairs per row
    __shared__ float2 cs[HALF];
    const int t = blockIdx.x, tid = threadIdx.x;
    // the sequence: the last s with first[s] <= t
    int lo = 0, hi = a.S;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.first[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int s = lo, end = a.first[s + 1];
    if (t < a.first[s] || t >= end) return;                  // behind the last sequence
    if (a.pos != nullptr && tid < HALF) {
        const double turns = (double)a.pos[(size_t)rot.axis[tid] * a.T + t] * rot.turns[tid];
        float sn, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn, &c);
        cs[tid] = make_float2(c, sn);
    }
    __syncthreads();
    const long long cap = (long long)a.per_seq * a.page;
    const long long row = (long long)a.len[s] - (end - t);
    const bool there = row >= 0 && row < cap;
    const int page = there ? a.table[(size_t)s * a.per_seq + row / a.page] : -1;
    const bool write = (unsigned)page < (unsigned)a.pages;
    const int rotated = write ? a.H : 0;
    const int nq = a.q != nullptr ? a.Hq : 0;
    for (int i = tid; i < (rotated + nq) * PP; i += 256) {
        const int h = i / PP, p = i % PP;
        const bool key = h < rotated;
        const char *src = key ? a.k + t * a.k_token + h * a.k_head : a.q + t * a.q_token + (h - rotated) * a.q_head;
        char *dst = key ? reinterpret_cast<char *>(a.K) + (paged_base(page, a.pages, a.H, h, a.page) + row % a.page) * (D * ES)
                        : a.q_out + ((long long)t * a.Hq + (h - rotated)) * (D * ES);
        uint4 x = *reinterpret_cast<const uint4 *>(src + p * 16), y = *reinterpret_cast<const uint4 *>(src + HALF * ES + p * 16);
        if (a.pos != nullptr) rotate16<BF16>(x, y, cs + p * PER);
        store16(dst + p * 16, x);
        store16(dst + HALF * ES + p * 16, y);
    }
    if (!write) return;
    for (int i = tid; i < a.H * 2 * PP; i += 256) {
        const int h = i / (2 * PP), p = i % (2 * PP);
        char *dst = reinterpret_cast<char *>(a.V) + (paged_base(page, a.pages, a.H, h, a.page) + row % a.page) * (D * ES);
        store16(dst + p * 16, *reinterpret_cast<const uint4 *>(a.v + t * a.v_token + h * a.v_head + p * 16));
    }
    for (int h = tid; h < a.H; h += 256) {
        const long long at = ((long long)s * a.H + h) * cap + row;
        if (a.stamp != nullptr) a.stamp[at] = a.seen[s] - (end - t);
        if (a.mass != nullptr) a.mass[at] = 0.0f;
    }
}

}  // namespace

hipError_t launch_paged_append(const ws_paged_cache &c, const ws_rows &k, const ws_rows &v, int T, const int32_t *first,
                               const int32_t *pos, const RotaryTable &rot, const ws_rows *q, int Hq, void *q_out, const int32_t *seen,
                               int32_t *stamp, float *mass, hipStream_t st)
{
    const bool bf16 = c.dt == WS_BF16;
    const long long es = bf16 ? 2 : 4;
    AppendArgs a = {};
    a.K = c.K, a.V = c.V, a.table = c.table, a.len = c.len;
    a.pages = c.pages, a.H = c.Hkv, a.page = c.page, a.S = c.S, a.per_seq = c.per_seq;
    a.k = reinterpret_cast<const char *>(k.x), a.k_token = k.token * es, a.k_head = k.head * es;
    a.v = reinterpret_cast<const char *>(v.x), a.v_token = v.token * es, a.v_head = v.head * es;
    if (q) a.q = reinterpret_cast<const char *>(q->x), a.q_token = q->token * es, a.q_head = q->head * es, a.Hq = Hq;
    a.q_out = reinterpret_cast<char *>(q_out);
    a.T = T, a.first = first, a.pos = pos, a.seen = seen, a.stamp = stamp, a.mass = mass;
    const dim3 grid((unsigned)T), block(256);
    if (bf16 && c.d == 64) hipLaunchKernelGGL((append_tokens<true, 64>), grid, block, 0, st, a, rot);
    else if (bf16) hipLaunchKernelGGL((append_tokens<true, 128>), grid, block, 0, st, a, rot);
    else if (c.d == 64) hipLaunchKernelGGL((append_tokens<false, 64>), grid, block, 0, st, a, rot);
    else hipLaunchKernelGGL((append_tokens<false, 128>), grid, block, 0, st, a, rot);
    return hipGetLastError();
}

}  // namespace ws
