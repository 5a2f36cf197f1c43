// Attention of one new token of every sequence over its paged cache.
//     z[q,r] = scale Q[q].K[r],  O[q] = sum_r exp(z - m) V[r] / sum_r exp(z - m)
//
// paged_split reads the cache once for every 16 query heads of a KV head.  The rows of all (sequence, KV head) pairs are counted off in
// tiles of TR rows, and every workgroup takes an equal run of tiles across the borders of pairs, so that a batch of unequal lengths
// keeps the whole chip busy.
// Inside its part of a pair the four waves take tiles in turn; a wave does
//     S^T = K_tile . Q^T    (rows of the result: cache rows, columns: up to 16 query heads)
//     O^T += V_tile^T . P^T (rows: head dimensions, columns: query heads)
// with 16x16 matrix instructions.  Both results hold one query head per lane (lane & 15), so maximum, sum and rescaling are plain
// per-lane arithmetic, and the weights leave the softmax in the lane and order the second product's operand wants: the order of the
// rows within a contraction is free as long as V is fetched in the same one.  A lane's block of V is rows x head dimensions, which
// the product wants the other way round; eight rows of bf16 are turned in registers by one byte permutation per pair.  Nothing of K, V
// or P goes through LDS.  Bound: HBM (g flop per byte against 250): 8 heads of 131072 rows, d = 128, bf16: 537 MB in 80 us, 6.7 TB/s, matrix
// cores 8 % busy.  With weights, 256 heads of 32768 rows under 8 query heads each: 4.6 GB in 879 us, 5.2 TB/s; the logits, 6 % of the
// bytes, cost 261 us, because they are written to HBM in between the reads (10 of it with all stores on a kilobyte per head).
//
// paged_join brings the parts of a pair that several workgroups shared to their common maximum; paged_weights adds the rows'
// weights, from the logits that paged_split left, to their accounts.  Logits and maxima are in units of log2.
#include <type_traits>

#include "paged_internal.h"

namespace ws {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

namespace {

// What no kernel here writes and every lane of a wave reads alike is read through the scalar cache.
typedef const __attribute__((address_space(4))) int32_t *scalar_i32;
__device__ __forceinline__ scalar_i32 as_scalar(const int32_t *p) { return (scalar_i32)(uintptr_t)p; }

// With up to 16 query heads per KV head the cache's rows are read once: marked as such they leave the chip's caches to everything else
// (8 heads of 131072 rows, d = 128, bf16: 83 us against 95 with ordinary loads).  With more they are read again for the next 16, and the
// mark would keep them from being found (32 query heads per KV head, the same rows: 131 us with it, 108 without; 100 x 8 heads of
// 1200 rows: 176, 142; fp32, 64 query heads, 8 heads of 131072 rows: 614, 356).
template <bool ONCE, typename T>
__device__ __forceinline__ T load_rows(const void *p)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const T *>(p));
    else return *reinterpret_cast<const T *>(p);
}
template <bool ONCE>
__device__ __forceinline__ uint4 load16(const void *p)
{
    const u32x4_t v = load_rows<ONCE, u32x4_t>(p);
    return make_uint4(v[0], v[1], v[2], v[3]);
}

struct AttendArgs {
    const void *K, *V, *Q;
    const int32_t *table, *len;
    int pages, H, page_shift, S, per_seq, Hq, tiles_q;
    float scale_log2;
    int32_t *total, *start;                  // [1] tiles in all; [S,H,tiles_q] first tile of every pair
    float *stats;                            // [S,Hq] log2 of the sum of all weights
    float *slot_stats, *slots;               // [2 * groups][gt][2], [2 * groups][gt][D]
    float *logits;                           // [S,H][logit_rows(cap) / 16][g][16] or NULL: what a wave stores at once lies together
    float *O, *lse;
    const float *mass_in;
    float *mass_out;
    float decay;
    int aligned;                             // the accounts can be read and written 16 bytes at a time
};

// An equal share of `total` tiles for each of `groups`: group b's run starts at ...
__device__ __forceinline__ int share_start(int total, int groups, int b)
{
    const int per = total / groups, rest = total % groups;
    return b * per + min(b, rest);
}
// ... and tile t is in the run of group
__device__ __forceinline__ int share_owner(int total, int groups, int t)
{
    const int per = total / groups, rest = total % groups;
    return t < (per + 1) * rest ? t / (per + 1) : rest + (t - (per + 1) * rest) / per;
}

// A workgroup's run of units of UNIT rows, counted through all sequences and the `pairs` heads of each: units [from, to) of `total`, the
// sequence s that holds unit `from`, and that sequence's first unit.  Every wave finds it for itself: a lane counts the units of some
// consecutive sequences, a scan over the lanes gives where each lane's begin.
struct Run {
    int total, from, to, s, first;
    template <int UNIT>
    __device__ __forceinline__ void find(const AttendArgs &a, int pairs, int groups, int b)
    {
        const int lane = threadIdx.x & 63, cap = a.per_seq << a.page_shift, each = (a.S + 63) / 64;
        if (a.S == 1) {                                  // nothing to look for: 0.5 to 1 us of a call
            s = first = 0;
            total = (paged_rows(as_scalar(a.len)[0], cap) + UNIT - 1) / UNIT * pairs;
            from = share_start(total, groups, b);
            to = share_start(total, groups, b + 1);
            return;
        }
        int mine = 0;
        for (int i = 0; i < each; ++i) {
            const int q = lane * each + i;
            if (q < a.S) mine += (paged_rows(a.len[q], cap) + UNIT - 1) / UNIT;
        }
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(upto, o);
            if (lane >= o) upto += y;
        }
        total = __builtin_amdgcn_readlane(upto, 63) * pairs;
        from = share_start(total, groups, b);
        to = share_start(total, groups, b + 1);
        if (from >= to) return;
        const int l = __builtin_ctzll(__ballot((long long)upto * pairs > from));        // the lane that reaches beyond `from`
        s = l * each;
        first = (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l)) * pairs;
        skip<UNIT>(a, pairs, from);
    }
    // On to the sequence that holds unit t, which is not before s.
    template <int UNIT>
    __device__ __forceinline__ int skip(const AttendArgs &a, int pairs, int t)
    {
        for (;;) {
            const int n = paged_rows(as_scalar(a.len)[s], a.per_seq << a.page_shift), units = (n + UNIT - 1) / UNIT;
            if (t < first + units * pairs) return n;
            first += units * pairs;
            ++s;
        }
    }
};

template <bool BF16, int D>
struct Shape {
    static constexpr int TR = BF16 ? 32 : 16;            // rows of a tile
    static constexpr int RB = D * (BF16 ? 2 : 4);        // bytes of a row
    static constexpr int HV = TR / 16;                   // 16-row halves of a tile
    static constexpr int NK = RB / 64;                   // 16-byte loads of K per lane and half
    static constexpr int C = D / 16;                     // head dimensions per lane: a lane's block of V is rows x C
    static constexpr int VW = C * (BF16 ? 2 : 4) / 4;    // 32-bit words of them
    static constexpr int NV = 4 * HV;                    // rows of V per lane
};

template <bool BF16, int D>
struct Tile {
    uint4 k[Shape<BF16, D>::HV][Shape<BF16, D>::NK];
    uint32_t v[Shape<BF16, D>::NV][Shape<BF16, D>::VW];
};

constexpr int kNowhere = 0, kToMemory = 1, kToLds = 2;       // where the logits go, for the rows' weights

// Room for the four waves' parts of a result; a row's length shifts the banks from query to query.
template <int D>
struct alignas(16) Merge {
    float part[4][kPagedQueries][D + 4];
    float m[4][kPagedQueries], l[4][kPagedQueries];
    // the four parts of query q brought to their maximum: that, their sum of weights, and element e
    __device__ __forceinline__ void query(int q, int e, float &top, float &lsum, float &sum) const
    {
        top = fmaxf(fmaxf(m[0][q], m[1][q]), fmaxf(m[2][q], m[3][q]));
        sum = lsum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(m[w][q] - top);
            sum = fmaf(part[w][q][e], f, sum);
            lsum = fmaf(l[w][q], f, lsum);
        }
    }
};

// One wave's way through tiles of a (sequence, KV head, query heads).  begin() says which and asks for the first tile, run() goes through
// them, leave() puts the wave's part into LDS; begin() of the next ones may come before leave(), so that their first tile is on its
// way while the waves' parts are put together.
template <bool BF16, int D, int SINK, bool ONCE>
struct Sweep {
    using P = Shape<BF16, D>;
    static constexpr int TR = P::TR, RB = P::RB, HV = P::HV, NK = P::NK, C = P::C, VW = P::VW, NV = P::NV;
    const AttendArgs &a;
    const int lane, wave, lq, lj, pmask, g;
    const unsigned koff, voff;
    float *const kept;                                   // kToLds: [g][kept_stride]
    const int kept_stride;
    // which tiles
    int s, h, q0, n, t, tb, gt, last16;
    scalar_i32 table;
    __amdgpu_buffer_rsrc_t logits;
    // the tile on its way, the pages of the next one, the queries
    Tile<BF16, D> x;
    int id[HV];
    uint4 qf[NK];
    // what is there: maximum and sum (of the lane's rows) of query lq, output
    float m, l;
    f32x4_t acc[C];

    __device__ __forceinline__ Sweep(const AttendArgs &args, float *k, int stride)
        : a(args), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), lq(lane & 15), lj(lane >> 4),
          pmask((1 << args.page_shift) - 1), g(args.Hq / args.H), koff(lq * RB + lj * 16), voff(4 * lj * RB + lq * VW * 4), kept(k),
          kept_stride(stride)
    {
    }

    __device__ __forceinline__ void pages_of(int tile, int (&to)[HV]) const
    {
#pragma unroll
        for (int hf = 0; hf < HV; ++hf) to[hf] = table[min(tile * TR + 16 * hf, last16) >> a.page_shift];
    }
    __device__ __forceinline__ unsigned long long half_base(int tile, int hf, int page) const    // where a half starts in the pools
    {
        const int r = min(tile * TR + 16 * hf, last16);
        return (unsigned long long)(paged_base(page, a.pages, a.H, h, 1 << a.page_shift) + (r & pmask)) * RB;
    }
    __device__ __forceinline__ void load_k(int tile)
    {
#pragma unroll
        for (int hf = 0; hf < HV; ++hf) {
            const char *p = reinterpret_cast<const char *>(a.K) + half_base(tile, hf, id[hf]);
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) x.k[hf][kk] = load16<ONCE>(p + koff + kk * 64);
        }
    }
    __device__ __forceinline__ void load_v(int tile)
    {
#pragma unroll
        for (int hf = 0; hf < HV; ++hf) {
            const char *p = reinterpret_cast<const char *>(a.V) + half_base(tile, hf, id[hf]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (VW == 2) {
                    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
                    const u32x2_t w = load_rows<ONCE, u32x2_t>(p + voff + i * RB);
                    x.v[4 * hf + i][0] = w[0], x.v[4 * hf + i][1] = w[1];
                } else {
#pragma unroll
                    for (int j = 0; j < VW / 4; ++j) {
                        const uint4 w = load16<ONCE>(p + voff + i * RB + 16 * j);
                        x.v[4 * hf + i][4 * j] = w.x, x.v[4 * hf + i][4 * j + 1] = w.y;
                        x.v[4 * hf + i][4 * j + 2] = w.z, x.v[4 * hf + i][4 * j + 3] = w.w;
                    }
                }
            }
        }
    }

    // Tiles [ta, to) of sequence s_'s head h_ (n_ > 0 rows), for its query heads q0_ ..
    __device__ __forceinline__ void begin(int s_, int h_, int q0_, int n_, int ta, int to)
    {
        s = s_, h = h_, q0 = q0_, n = n_, t = ta + wave, tb = to;
        gt = min(kPagedQueries, g - q0);
        last16 = (n - 1) & ~15;                          // a tile's second half may not exist: it reads this one instead
        table = as_scalar(a.table) + (long long)s * a.per_seq;
        if constexpr (SINK == kToMemory) {
            // the logits of this head's query heads, from the first one of this tile of them on
            const int rows = logit_rows(a.per_seq << a.page_shift);
            float *p = a.logits + ((long long)(s * a.H + h) * rows * g + q0 * 16);
            logits = __builtin_amdgcn_make_buffer_rsrc(p, 0, (rows * g - q0 * 16) * 4, 0x00020000);
        }
        if (t >= tb) return;
        pages_of(t, id);
        load_k(t);
        // the lane's part of query lq's row, in the order of the K loads; heads that do not exist are zero
        const char *q = reinterpret_cast<const char *>(a.Q) + ((long long)s * a.Hq + h * g + q0 + lq) * RB + lj * 16;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
            qf[kk] = make_uint4(0, 0, 0, 0);
            if (lq < gt) qf[kk] = *reinterpret_cast<const uint4 *>(q + kk * 64);
        }
        load_v(t);
        pages_of(t + 4, id);
    }

    // One tile, held in x.  MORE: the wave's next tile, t + 4, is loaded behind the last use of K and of V (so one of the two is always
    // on its way), and the pages of the one after it are looked up; a tile with another one behind it is whole.
    template <bool MORE>
    __device__ __forceinline__ void tile()
    {
        int id2[HV];
        if constexpr (MORE) pages_of(t + 8, id2);
        // scores of rows 16 hf + 4 lj + i for query lq
        f32x4_t z[HV];
#pragma unroll
        for (int hf = 0; hf < HV; ++hf) {
            z[hf] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) {
                if constexpr (BF16) {
                    z[hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x.k[hf][kk]),
                                                                   __builtin_bit_cast(bf16x8_t, qf[kk]), z[hf], 0, 0, 0);
                } else {
                    const uint32_t kw[4] = {x.k[hf][kk].x, x.k[hf][kk].y, x.k[hf][kk].z, x.k[hf][kk].w};
                    const uint32_t qw[4] = {qf[kk].x, qf[kk].y, qf[kk].z, qf[kk].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        z[hf] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[e]), __uint_as_float(qw[e]), z[hf], 0, 0, 0);
                }
            }
        }
        if constexpr (MORE) load_k(t + 4);
        const int r0 = t * TR + 4 * lj;              // the lane's first row
        float top = -__builtin_inff();
#pragma unroll
        for (int hf = 0; hf < HV; ++hf)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[hf][i] *= a.scale_log2;
                // rows behind the sequence's last one hold anything: their score is replaced, and so is their V below
                if (!MORE && r0 + 16 * hf + i >= n) z[hf][i] = -__builtin_inff();
                top = fmaxf(top, z[hf][i]);
            }
        if constexpr (SINK == kToMemory) {
            // Lanes of heads that do not exist store out of the buffer's range, which the hardware drops: behind a branch the
            // compiler could not count these stores, and every tile would wait for the K it has just asked for.
            const unsigned to = (unsigned)((t * HV * g + lq) * 16 + 4 * lj) * 4u;
#pragma unroll
            for (int hf = 0; hf < HV; ++hf) {
                const bool there = lq < gt && (MORE || r0 + 16 * hf < n);
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, z[hf]), logits, there ? to + 64u * g * hf : 0xFFFFFFF0u, 0, 0);
            }
        }
        if constexpr (SINK == kToLds) {
            if (lq < gt)
#pragma unroll
                for (int hf = 0; hf < HV; ++hf)
                    if (MORE || r0 + 16 * hf < n) *reinterpret_cast<f32x4_t *>(kept + lq * kept_stride + r0 + 16 * hf) = z[hf];
        }
        // the reference is moved only when a score exceeds it by more than 2^8: weights stay far from overflow, and the
        // accumulator is rescaled a few times per pass instead of once per tile.  (All four lanes of a query agree.)
        if (__any(top > m + 8.0f)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float to = fmaxf(m, top);
            const float fade = __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= fade;
#pragma unroll
            for (int c = 0; c < C; ++c) acc[c] *= fade;
        }
        float p[HV][4];
#pragma unroll
        for (int hf = 0; hf < HV; ++hf)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[hf][i] = __builtin_amdgcn_exp2f(z[hf][i] - m);
                l += p[hf][i];
            }
        if constexpr (!MORE) {
#pragma unroll
            for (int e = 0; e < NV; ++e)
#pragma unroll
                for (int w = 0; w < VW; ++w) x.v[e][w] = r0 + (e >> 2) * 16 + (e & 3) >= n ? 0u : x.v[e][w];
        }
        // O^T += V^T P^T
        if constexpr (BF16) {
            // a weight as the sum of three bf16 numbers, all its 24 bits: one alone would cost 2^-9 of it, two 2^-17, which
            // shows in the output (the matrix cores have the time)
            uint32_t part[3][4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                f32x2_t pv;
                pv[0] = p[w >> 1][2 * (w & 1)];
                pv[1] = p[w >> 1][2 * (w & 1) + 1];
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    const uint32_t two = __builtin_bit_cast(uint32_t, __builtin_convertvector(pv, bf16x2_t));
                    part[k][w] = two;
                    pv[0] -= __uint_as_float(two << 16);
                    pv[1] -= __uint_as_float(two & 0xFFFF0000u);
                }
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                uint32_t vt[4];
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    vt[w] = __builtin_amdgcn_perm(x.v[2 * w + 1][c >> 1], x.v[2 * w][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
                const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, make_uint4(vt[0], vt[1], vt[2], vt[3]));
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        vf, __builtin_bit_cast(bf16x8_t, make_uint4(part[k][0], part[k][1], part[k][2], part[k][3])), acc[c], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < C; ++c)
                    acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.v[i][c]), p[0][i], acc[c], 0, 0, 0);
        }
        if constexpr (MORE) {
            load_v(t + 4);
#pragma unroll
            for (int hf = 0; hf < HV; ++hf) id[hf] = id2[hf];
        }
    }

    __device__ __forceinline__ void run()
    {
        m = -__builtin_inff(), l = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        if (t >= tb) return;
        for (; t + 4 < tb; t += 4) tile<true>();
        tile<false>();
    }

    // Lane (lq, lj) holds head dimensions 4 C lj .. 4 C (lj + 1) - 1 of query lq, of `queries` there are.
    __device__ __forceinline__ void leave(Merge<D> &red, int queries)
    {
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (lq >= queries) return;
        if (lj == 0) {
            red.m[wave][lq] = m;
            red.l[wave][lq] = l;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < C; c += 4)
                *reinterpret_cast<f32x4_t *>(&red.part[wave][lq][(4 * lj + i) * C + c]) =
                    f32x4_t{acc[c][i], acc[c + 1][i], acc[c + 2][i], acc[c + 3][i]};
    }
};

template <bool BF16, int D, bool WEIGHTS, bool ONCE>
__global__ void __launch_bounds__(256, 3)
paged_split(AttendArgs a)
{
    constexpr int TR = Shape<BF16, D>::TR;
    __shared__ Merge<D> red;
    const int tid = threadIdx.x, b = blockIdx.x, groups = gridDim.x;
    const int pairs = a.H * a.tiles_q, g = a.Hq / a.H;   // pairs: of one sequence

    Run run;
    run.template find<TR>(a, pairs, groups, b);
    if (b == 0 && tid == 0) *a.total = run.total;
    int t0 = run.from, s = run.s, first = run.first;
    const int t1 = run.to;
    if (t0 >= t1) return;
    // ---- its parts of pairs, one after the other; a part's first tile is asked for before the one before it is put together
    const int run0 = t0;
    Sweep<BF16, D, WEIGHTS ? kToMemory : kNowhere, ONCE> w(a, nullptr, 0);
    int pair, pair0, ts;                                 // the part at t0: its pair within the sequence, the pair's first tile, its tiles
    auto begin = [&]() {
        const int n = run.template skip<TR>(a, pairs, t0);
        s = run.s, first = run.first, ts = (n + TR - 1) / TR;
        pair = (t0 - first) / ts;
        pair0 = first + pair * ts;
        w.begin(s, pair / a.tiles_q, pair % a.tiles_q * kPagedQueries, n, t0 - pair0, min(ts, t1 - pair0));
    };
    begin();
    for (;;) {
        w.run();
        const long long qrow = (long long)s * a.Hq + w.h * g + w.q0;
        const int gt = w.gt, end = min(pair0 + ts, t1);
        const bool all = t0 == pair0 && end == pair0 + ts;       // nobody else has a part of this pair
        const int slot = 2 * b + (t0 == run0 ? 0 : 1);
        if (t0 == pair0 && tid == 0) a.start[(long long)s * pairs + pair] = pair0;
        t0 = end;
        const bool more = t0 < t1;
        if (more) begin();
        w.leave(red, gt);
        __syncthreads();
        for (int i = tid; i < gt * D; i += 256) {
            const int q = i / D, e = i % D;
            float top, lsum, sum;
            red.query(q, e, top, lsum, sum);
            if (all) {
                a.O[(qrow + q) * D + e] = sum / lsum;
                if (e == 0) {
                    const float z = top + __builtin_amdgcn_logf(lsum);
                    a.stats[qrow + q] = z;
                    if (a.lse != nullptr) a.lse[qrow + q] = z * 0.693147180559945309f;
                }
            } else {
                const int gs = min(kPagedQueries, g);
                a.slots[((long long)slot * gs + q) * D + e] = sum;
                if (e == 0) {
                    a.slot_stats[(slot * gs + q) * 2] = top;
                    a.slot_stats[(slot * gs + q) * 2 + 1] = lsum;
                }
            }
        }
        if (!more) return;
        __syncthreads();
    }
}

// decay * mass_in + w of four rows, to mass_out.
__device__ __forceinline__ void account(const AttendArgs &a, long long at, int r, int n, const f32x4_t &w)
{
    at += r;
    if (r + 4 <= n && a.aligned) {
        f32x4_t x = w;
        if (a.mass_in != nullptr) {
            const f32x4_t old = *reinterpret_cast<const f32x4_t *>(a.mass_in + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = fmaf(a.decay, old[i], w[i]);
        }
        *reinterpret_cast<f32x4_t *>(a.mass_out + at) = x;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r + i < n) a.mass_out[at + i] = a.mass_in != nullptr ? fmaf(a.decay, a.mass_in[at + i], w[i]) : w[i];
    }
}

// Short caches: one workgroup has all rows of its (sequence, KV head, query heads), so nothing is left to join, and the logits, kept
// in LDS, become weights in the same launch.
template <bool BF16, int D, bool WEIGHTS, bool ONCE>
__global__ void __launch_bounds__(256, 3)
paged_whole(AttendArgs a, int kept_stride)
{
    constexpr int TR = Shape<BF16, D>::TR;
    __shared__ Merge<D> red;
    __shared__ float stat[kPagedQueries];
    extern __shared__ __attribute__((aligned(16))) float kept[];     // [g][kept_stride] logits
    const int tid = threadIdx.x;
    const int cap = a.per_seq << a.page_shift, g = a.Hq / a.H;
    const int qt = blockIdx.x % a.tiles_q, pair = blockIdx.x / a.tiles_q, s = pair / a.H, h = pair % a.H;
    const int q0 = qt * kPagedQueries, gt = min(kPagedQueries, g - q0);
    const int n = paged_rows(as_scalar(a.len)[s], cap);
    const long long qrow = (long long)s * a.Hq + h * g + q0;
    if (n == 0) {
        for (int i = tid; i < gt * D; i += 256) a.O[qrow * D + i] = 0.0f;
        if (tid < gt && a.lse != nullptr) a.lse[qrow + tid] = -__builtin_inff();
        return;
    }
    Sweep<BF16, D, WEIGHTS ? kToLds : kNowhere, ONCE> w(a, kept, kept_stride);
    w.begin(s, h, q0, n, 0, (n + TR - 1) / TR);
    w.run();
    w.leave(red, gt);
    __syncthreads();
    for (int i = tid; i < gt * D; i += 256) {
        const int q = i / D, e = i % D;
        float top, lsum, sum;
        red.query(q, e, top, lsum, sum);
        a.O[(qrow + q) * D + e] = sum / lsum;
        if (e == 0) {
            const float z = top + __builtin_amdgcn_logf(lsum);
            stat[q] = z;
            if (a.lse != nullptr) a.lse[qrow + q] = z * 0.693147180559945309f;
        }
    }
    if constexpr (WEIGHTS) {
        __syncthreads();
        for (int r = tid * 4; r < n; r += 1024) {
            f32x4_t w = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int q = 0; q < gt; ++q) {
                const f32x4_t z = *reinterpret_cast<const f32x4_t *>(kept + q * kept_stride + r);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] += __builtin_amdgcn_exp2f(z[i] - stat[q]);
            }
            account(a, (long long)pair * cap, r, n, w);
        }
    }
}

// What several workgroups left of one query head: their statistics, and where their parts lie.
struct Parts {
    int b0, b1, slot0, gs, ql;
    __device__ long long slot(int b) const { return (long long)(b == b0 ? slot0 : 2 * b) * gs + ql; }
};
template <int TR>
__device__ __forceinline__ Parts parts_of(const AttendArgs &a, int groups, int s, int h, int q, int n)
{
    Parts p;
    const int total = *a.total, ts = (n + TR - 1) / TR;
    const int pair0 = a.start[((long long)s * a.H + h) * a.tiles_q + q / kPagedQueries];
    p.b0 = share_owner(total, groups, pair0);
    p.b1 = share_owner(total, groups, pair0 + ts - 1);
    p.slot0 = 2 * p.b0 + (share_start(total, groups, p.b0) == pair0 ? 0 : 1);
    p.gs = min(kPagedQueries, a.Hq / a.H);
    p.ql = q % kPagedQueries;
    return p;
}

// One workgroup per query head of a sequence: its parts, if it has several, to their common maximum.
template <bool BF16, int D>
__device__ void join_row(const AttendArgs &a, int groups, int row)
{
    constexpr int TR = Shape<BF16, D>::TR;
    __shared__ float factor[kPagedGroups];
    __shared__ float red[4][D], red_l[4], red_m[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int g = a.Hq / a.H, s = row / a.Hq, qh = row % a.Hq, h = qh / g, q = qh % g;
    const int n = paged_rows(a.len[s], a.per_seq << a.page_shift);
    if (n == 0) {
        if (tid < D) a.O[(long long)row * D + tid] = 0.0f;
        if (tid == 0 && a.lse != nullptr) a.lse[row] = -__builtin_inff();
        return;
    }
    const Parts p = parts_of<TR>(a, groups, s, h, q, n);
    if (p.b0 == p.b1) return;                            // one workgroup had all of it and has written it
    // the first parts of each wave are on their way while the statistics are looked at
    constexpr int AHEAD = 8;
    float ahead[AHEAD][D / 64];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (p.b0 + wave + 4 * i <= p.b1)
#pragma unroll
            for (int e = 0; e < D / 64; ++e) ahead[i][e] = a.slots[p.slot(p.b0 + wave + 4 * i) * D + e * 64 + lane];
    float mine = -__builtin_inff(), l = 0.0f;            // of part b0 + tid
    if (p.b0 + tid <= p.b1) {
        mine = a.slot_stats[p.slot(p.b0 + tid) * 2];
        l = a.slot_stats[p.slot(p.b0 + tid) * 2 + 1];
    }
    float m = mine;
    for (int b = p.b0 + tid + 256; b <= p.b1; b += 256) m = fmaxf(m, a.slot_stats[p.slot(b) * 2]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    if (lane == 0) red_m[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red_m[0], red_m[1]), fmaxf(red_m[2], red_m[3]));
    factor[tid] = __builtin_amdgcn_exp2f(mine - m);
    l *= factor[tid];
    for (int b = p.b0 + tid + 256; b <= p.b1; b += 256) {
        const float f = __builtin_amdgcn_exp2f(a.slot_stats[p.slot(b) * 2] - m);
        factor[b - p.b0] = f;
        l = fmaf(a.slot_stats[p.slot(b) * 2 + 1], f, l);
    }
    l = lane_group_sum<64>(l);
    if (lane == 0) red_l[wave] = l;
    __syncthreads();
    l = red_l[0] + red_l[1] + red_l[2] + red_l[3];
    float acc[D / 64] = {};
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (p.b0 + wave + 4 * i <= p.b1)
#pragma unroll
            for (int e = 0; e < D / 64; ++e) acc[e] = fmaf(ahead[i][e], factor[wave + 4 * i], acc[e]);
#pragma unroll 4
    for (int b = p.b0 + wave + 4 * AHEAD; b <= p.b1; b += 4) {
        const float f = factor[b - p.b0];
#pragma unroll
        for (int e = 0; e < D / 64; ++e) acc[e] = fmaf(a.slots[p.slot(b) * D + e * 64 + lane], f, acc[e]);
    }
#pragma unroll
    for (int e = 0; e < D / 64; ++e) red[wave][e * 64 + lane] = acc[e];
    __syncthreads();
    if (tid < D) a.O[(long long)row * D + tid] = (red[0][tid] + red[1][tid] + red[2][tid] + red[3][tid]) / l;
    if (tid == 0 && a.lse != nullptr) a.lse[row] = (m + __builtin_amdgcn_logf(l)) * 0.693147180559945309f;
}

// 1024 rows of a (sequence, KV head): what the rows received is added to their accounts.
constexpr int kWeightRows = 1024;
template <bool BF16, int D>
__device__ __forceinline__ void add_weights(const AttendArgs &a, int groups, int s, int h, int n, int chunk, float *stat)
{
    constexpr int TR = Shape<BF16, D>::TR;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int cap = a.per_seq << a.page_shift, g = a.Hq / a.H, pair = s * a.H + h;
    const int r = chunk * kWeightRows + tid * 4;
    const float *z = a.logits + ((long long)pair * logit_rows(cap) + r / 16 * 16) * g + r % 16;
    f32x4_t w = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int q0 = 0; q0 < g; q0 += 256) {
        if (q0 > 0) __syncthreads();
        // the sum of all weights of query head q, log2: as written by the one workgroup that had it all, or from its parts
        for (int q = q0 + wave; q < min(g, q0 + 256); q += 4) {
            const Parts p = parts_of<TR>(a, groups, s, h, q, n);
            float all;
            if (p.b0 == p.b1) {
                all = a.stats[(long long)s * a.Hq + h * g + q];
            } else {
                float m = -__builtin_inff(), l = 0.0f;
                for (int b = p.b0 + lane; b <= p.b1; b += 64) m = fmaxf(m, a.slot_stats[p.slot(b) * 2]);
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
                for (int b = p.b0 + lane; b <= p.b1; b += 64)
                    l = fmaf(a.slot_stats[p.slot(b) * 2 + 1], __builtin_amdgcn_exp2f(a.slot_stats[p.slot(b) * 2] - m), l);
                all = m + __builtin_amdgcn_logf(lane_group_sum<64>(l));
            }
            if (lane == 0) stat[q - q0] = all;
        }
        __syncthreads();
        if (r < n)
#pragma unroll 4
            for (int q = q0; q < min(g, q0 + 256); ++q) {
                const f32x4_t x = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t *>(z + (long long)q * 16));
                const float all = stat[q - q0];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] += __builtin_amdgcn_exp2f(x[i] - all);
            }
    }
    if (r < n) account(a, (long long)pair * cap, r, n, w);
}

// The first S * Hq workgroups join, a query head of a sequence each; the others share out the rows whose weights are wanted.
template <bool BF16, int D>
__global__ void __launch_bounds__(256)
paged_finish(AttendArgs a, int groups)
{
    const int rows = a.S * a.Hq;
    if ((int)blockIdx.x < rows) {
        join_row<BF16, D>(a, groups, blockIdx.x);
        return;
    }
    __shared__ float stat[256];
    Run run;
    run.template find<kWeightRows>(a, a.H, gridDim.x - rows, blockIdx.x - rows);
    for (int u = run.from; u < run.to; ++u) {
        const int n = run.template skip<kWeightRows>(a, a.H, u), chunks = (n + kWeightRows - 1) / kWeightRows;
        const int h = (u - run.first) / chunks;
        add_weights<BF16, D>(a, groups, run.s, h, n, u - run.first - h * chunks, stat);
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_paged_attend(const ws_paged_cache &c, const void *Q, int Hq, float scale, float *O, float *lse, float decay,
                               const float *mass_in, float *mass_out, void *ws, hipStream_t st)
{
    const bool bf16 = c.dt == WS_BF16;
    const int cap = c.per_seq * c.page;
    const PagedAttendSpace sp = paged_attend_space(bf16, c.S, c.Hkv, Hq, cap, c.d, mass_out != nullptr);
    AttendArgs a = {};
    a.K = c.K, a.V = c.V, a.Q = Q, a.table = c.table, a.len = c.len;
    a.pages = c.pages, a.H = c.Hkv, a.page_shift = __builtin_ctz((unsigned)c.page), a.S = c.S, a.per_seq = c.per_seq, a.Hq = Hq;
    a.tiles_q = paged_query_tiles(Hq / c.Hkv);
    a.scale_log2 = scale * 1.4426950408889634f;
    char *base = reinterpret_cast<char *>(ws);
    a.total = reinterpret_cast<int32_t *>(base);
    a.start = reinterpret_cast<int32_t *>(base + sp.start);
    a.stats = reinterpret_cast<float *>(base + sp.stats);
    a.slot_stats = reinterpret_cast<float *>(base + sp.slot_stats);
    a.slots = reinterpret_cast<float *>(base + sp.slots);
    a.logits = mass_out ? reinterpret_cast<float *>(base + sp.logits) : nullptr;
    a.O = O, a.lse = lse, a.mass_in = mass_in, a.mass_out = mass_out, a.decay = decay;
    a.aligned = ((reinterpret_cast<uintptr_t>(mass_in) | reinterpret_cast<uintptr_t>(mass_out)) & 15) == 0;
    const int groups = paged_groups(bf16, c.S, c.Hkv, Hq, cap, c.d);
    const bool once = a.tiles_q == 1;
    auto go = [&](auto BF, auto DD) {
        constexpr bool B = decltype(BF)::value;
        constexpr int D = decltype(DD)::value;
        const dim3 grid((unsigned)groups), block(256);
        if (paged_whole_heads(c.S, c.Hkv, Hq, cap, mass_out != nullptr)) {
            const dim3 heads((unsigned)(c.S * c.Hkv * a.tiles_q));
            const int stride = mass_out ? logit_rows(cap) + 4 : 0;
            // (with accounts there are 16 query heads at most)
            if (mass_out) hipLaunchKernelGGL((paged_whole<B, D, true, true>), heads, block, stride * (Hq / c.Hkv) * sizeof(float), st, a, stride);
            else if (once) hipLaunchKernelGGL((paged_whole<B, D, false, true>), heads, block, 0, st, a, stride);
            else hipLaunchKernelGGL((paged_whole<B, D, false, false>), heads, block, 0, st, a, stride);
            return hipGetLastError();
        }
        if (mass_out && once) hipLaunchKernelGGL((paged_split<B, D, true, true>), grid, block, 0, st, a);
        else if (mass_out) hipLaunchKernelGGL((paged_split<B, D, true, false>), grid, block, 0, st, a);
        else if (once) hipLaunchKernelGGL((paged_split<B, D, false, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((paged_split<B, D, false, false>), grid, block, 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        // The lengths are on the device: of a long table most may be empty, and no launch is made of workgroups that find nothing to do.
        const long long chunks = mass_out ? (long long)c.S * c.Hkv * ((cap + kWeightRows - 1) / kWeightRows) : 0;
        const unsigned weighing = (unsigned)(chunks < 2048 ? chunks : 2048);
        hipLaunchKernelGGL((paged_finish<B, D>), dim3((unsigned)(c.S * Hq) + weighing), block, 0, st, a, groups);
        return hipGetLastError();
    };
    using std::integral_constant;
    if (bf16) return c.d == 64 ? go(std::true_type(), integral_constant<int, 64>()) : go(std::true_type(), integral_constant<int, 128>());
    return c.d == 64 ? go(std::false_type(), integral_constant<int, 64>()) : go(std::false_type(), integral_constant<int, 128>());
}

}  // namespace ws
