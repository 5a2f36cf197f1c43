// Attention of one new token of every sequence over its paged cache.
//     z[q,r] = scale Q[q].K[r],  O[q] = sum_r exp(z - m) V[r] / sum_r exp(z - m)
//
// paged_split: a workgroup takes one KV head of one sequence and one of `splits` equal ranges of its rows, in tiles of 64 rows with
// the softmax's running maximum and sum, and leaves maximum, sum and unnormalised output per query head; paged_join: one wave
// per query head brings the splits to their common maximum; paged_weights: adds the rows' weights, from the logits that
// paged_split left, to their accounts.  Logits are kept in units of log2.
#include "paged_internal.h"

namespace ws {

namespace {

constexpr int kTile = 64;

struct AttendArgs {
    const void *K, *V, *Q;
    const int32_t *table, *len;
    int pages, H, page, S, per_seq, Hq, splits;
    float scale_log2;
    float *partial, *stats, *logits;
    float *O, *lse;
    const float *mass_in;
    float *mass_out;
    float decay;
};

template <bool BF16>
__device__ __forceinline__ float element(const void *p, long long i)
{
    if constexpr (BF16) return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(p)[i] << 16);
    else return reinterpret_cast<const float *>(p)[i];
}

__device__ __forceinline__ void split_range(int n, int splits, int sp, int &r0, int &r1)
{
    const int per = ((n + splits - 1) / splits + kTile - 1) / kTile * kTile;
    r0 = min(n, sp * per);
    r1 = min(n, r0 + per);
}

template <bool BF16, int D>
__global__ void __launch_bounds__(256)
paged_split(AttendArgs a)
{
    __shared__ float z[kTile];
    __shared__ float part[256];
    const int tid = threadIdx.x;
    const int sp = blockIdx.x % a.splits, pair = blockIdx.x / a.splits;
    const int s = pair / a.H, h = pair % a.H, g = a.Hq / a.H;
    const int cap = a.per_seq * a.page;
    const int n = paged_rows(a.len[s], cap);
    int r0, r1;
    split_range(n, a.splits, sp, r0, r1);
    for (int j = 0; j < g; ++j) {
        const int qh = h * g + j;
        float m = -__builtin_inff(), l = 0.0f, acc = 0.0f;
        for (int t0 = r0; t0 < r1; t0 += kTile) {
            const int rows = min(kTile, r1 - t0);
            // four threads per row
            const int r = tid >> 2, lane = tid & 3;
            float dot = 0.0f;
            if (r < rows) {
                const int row = t0 + r;
                const long long base = paged_base(a.table[(long long)s * a.per_seq + row / a.page], a.pages, a.H, h, a.page) + row % a.page;
                for (int e = lane; e < D; e += 4)
                    dot = fmaf(element<BF16>(a.Q, ((long long)s * a.Hq + qh) * D + e), element<BF16>(a.K, base * D + e), dot);
            }
            dot = lane_group_sum<4>(dot);
            __syncthreads();
            if (lane == 0) z[r] = r < rows ? dot * a.scale_log2 : -__builtin_inff();
            __syncthreads();
            float top = m;
            for (int i = 0; i < rows; ++i) top = fmaxf(top, z[i]);
            const float fade = exp2f(m - top);
            m = top;
            if (a.logits != nullptr && tid < rows) a.logits[((long long)s * a.Hq + qh) * cap + t0 + tid] = z[tid];
            l *= fade;
            acc *= fade;
            for (int i = 0; i < rows; ++i) l += exp2f(z[i] - m);
            // 256 / D threads per output element, each every so many rows
            for (int i = tid / D; i < rows; i += 256 / D) {
                const int row = t0 + i;
                const long long base = paged_base(a.table[(long long)s * a.per_seq + row / a.page], a.pages, a.H, h, a.page) + row % a.page;
                acc = fmaf(exp2f(z[i] - m), element<BF16>(a.V, base * D + tid % D), acc);
            }
        }
        __syncthreads();
        part[tid] = acc;
        __syncthreads();
        if (tid < D) {
            float sum = 0.0f;
            for (int i = 0; i < 256 / D; ++i) sum += part[i * D + tid];
            float *out = a.partial + (((long long)s * a.Hq + qh) * a.splits + sp) * (D + 2);
            out[2 + tid] = sum;
            if (tid == 0) {
                out[0] = m;
                out[1] = l;
            }
        }
        __syncthreads();
    }
}

template <int D>
__global__ void __launch_bounds__(64)
paged_join(AttendArgs a)
{
    const long long row = blockIdx.x;
    const float *p = a.partial + row * a.splits * (D + 2);
    const int lane = threadIdx.x;
    float m = -__builtin_inff();
    for (int i = 0; i < a.splits; ++i) m = fmaxf(m, p[i * (D + 2)]);
    float l = 0.0f, acc[D / 64] = {};
    for (int i = 0; i < a.splits; ++i) {
        const float *q = p + (long long)i * (D + 2);
        if (q[1] == 0.0f) continue;                  // a split of no rows
        const float f = exp2f(q[0] - m);
        l += q[1] * f;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) acc[e] = fmaf(q[2 + e * 64 + lane], f, acc[e]);
    }
#pragma unroll
    for (int e = 0; e < D / 64; ++e) a.O[row * D + e * 64 + lane] = l > 0.0f ? acc[e] / l : 0.0f;
    if (lane == 0) {
        const float all = l > 0.0f ? m + log2f(l) : -__builtin_inff();
        a.stats[row] = all;
        if (a.lse != nullptr) a.lse[row] = all * 0.693147180559945309f;
    }
}

__global__ void __launch_bounds__(256)
paged_weights(AttendArgs a)
{
    const int cap = a.per_seq * a.page;
    const int pair = blockIdx.y + blockIdx.z * gridDim.y;
    if (pair >= a.S * a.H) return;
    const int s = pair / a.H, h = pair % a.H, g = a.Hq / a.H;
    const int r = blockIdx.x * 256 + threadIdx.x;
    if (r >= paged_rows(a.len[s], cap)) return;
    const long long at = (long long)pair * cap + r;
    float w = a.mass_in != nullptr ? a.decay * a.mass_in[at] : 0.0f;
    for (int j = 0; j < g; ++j) {
        const long long q = (long long)s * a.Hq + h * g + j;
        w += exp2f(a.logits[q * cap + r] - a.stats[q]);
    }
    a.mass_out[at] = w;
}

}  // namespace

hipError_t launch_paged_attend(const ws_paged_cache &c, const void *Q, int Hq, float scale, float *O, float *lse, float decay,
                               const float *mass_in, float *mass_out, void *ws, hipStream_t st)
{
    const int cap = c.per_seq * c.page;
    const PagedAttendSpace sp = paged_attend_space(c.S, c.Hkv, Hq, cap, c.d, mass_out != nullptr);
    AttendArgs a = {};
    a.K = c.K, a.V = c.V, a.Q = Q, a.table = c.table, a.len = c.len;
    a.pages = c.pages, a.H = c.Hkv, a.page = c.page, a.S = c.S, a.per_seq = c.per_seq, a.Hq = Hq;
    a.splits = paged_splits(c.S, c.Hkv, cap);
    a.scale_log2 = scale * 1.4426950408889634f;
    char *base = reinterpret_cast<char *>(ws);
    a.partial = reinterpret_cast<float *>(base + sp.partial);
    a.stats = reinterpret_cast<float *>(base + sp.stats);
    a.logits = mass_out ? reinterpret_cast<float *>(base + sp.logits) : nullptr;
    a.O = O, a.lse = lse, a.mass_in = mass_in, a.mass_out = mass_out, a.decay = decay;
    const dim3 grid((unsigned)(c.S * c.Hkv * a.splits)), block(256);
    if (c.dt == WS_BF16 && c.d == 64) hipLaunchKernelGGL((paged_split<true, 64>), grid, block, 0, st, a);
    else if (c.dt == WS_BF16) hipLaunchKernelGGL((paged_split<true, 128>), grid, block, 0, st, a);
    else if (c.d == 64) hipLaunchKernelGGL((paged_split<false, 64>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((paged_split<false, 128>), grid, block, 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (c.d == 64) hipLaunchKernelGGL((paged_join<64>), dim3((unsigned)(c.S * Hq)), dim3(64), 0, st, a);
    else hipLaunchKernelGGL((paged_join<128>), dim3((unsigned)(c.S * Hq)), dim3(64), 0, st, a);
    e = hipGetLastError();
    if (e != hipSuccess || !mass_out) return e;
    const int pairs = c.S * c.Hkv, y = pairs < 32768 ? pairs : 32768;
    hipLaunchKernelGGL(paged_weights, dim3((unsigned)((cap + 255) / 256), (unsigned)y, (unsigned)((pairs + y - 1) / y)), dim3(256), 0,
                       st, a);
    return hipGetLastError();
}

}  // namespace ws
