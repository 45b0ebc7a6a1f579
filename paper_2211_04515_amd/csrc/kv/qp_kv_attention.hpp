// Attention over the 4-bit key/value cache.
//
// Mathematics.  With key t = lo + c s (per token and head: codes c, grid lo, s) a score is a dot product with codes,
//     scale q.k_t = scale (s_t sum_d q_d (c_td - 8) + (lo_t + 8 s_t) sum_d q_d),
// and with p_t = exp(score_t - m) the answer's numerator is
//     sum_t p_t v_t = sum_t (p_t s_t) (c_t - 8) + sum_t p_t (lo_t + 8 s_t),
// the second term the same for all elements of a head.  So both products run on the codes themselves: c - 8 is an integer in
// [-8, 7], exact in fp16, and no value is ever dequantized.  (Centred codes, because the rounding of p_t s_t is multiplied by
// them: -8..7 costs about as much as the values' own spread would.)
//   q          is scaled by a power of two per column so that its largest element lies in [2^14, 2^15) and taken as fp16:
//              exact for bf16 (elements below 2^-30 of the largest aside, which round at 2^-39 of it); fp32 is split in two
//              halves, 22 bits of each element.
//   p_t s_t    is rounded to fp16 (fp32: split in two).  s_t is normalised by a power of two N so that the largest one seen lies
//              in [2^5, 2^7], and p_t <= 2^8, so that nothing overflows and what is lost at the lower end is 2^-32 of the largest.
//   Scores, the running maximum m, sum p_t, sum p_t (lo_t + 8 s_t) and the accumulators are fp32.
//
// Matrix shape.  v_mfma_f32_16x16x32_f16 with S^T = K q^T (16 tokens x 16 columns; a column is one token of the call and one of the
// query heads that share the key head) and O^T = V^T p^T.  With 32 tokens at a time, tile row m of the first product's two
// tiles j is token 8 (m div 4) + 4 j + m mod 4: then lane 16 g + n holds the scores of tokens 8 g .. 8 g + 7 of column n,
// which is just what the second product wants of it, so p never leaves the lane.  A word of value codes is eight tokens of one
// element for the same reason; elements are dealt out as d = m NB + block so that a lane's words are next to each other.
// A word w becomes eight halves as ((w >> 8 i) & 0x000f000f | 0x6400 6400) - 1032 and (.. & 0x00f000f0 | 0x5400 5400) - 72: codes
// 0, 4, 1, 5, 2, 6, 3, 7; queries and p are put in the same order.
// The maximum is lazy: a column's m moves only when a lane sees a score more than 8 (in log2) above it, so the loop has no exchange
// between lanes; what is rare (the maximum moves, N moves) is one branch of the whole wave.
//
// Who does what.  A block (four waves) takes one item: 64 NCT columns of one row and key head (each wave a quarter of the columns,
// all tokens), or, if it has at most 16 NCT columns, all waves the same columns and every fourth 32 tokens each, joined
// through LDS at the end.  Rows' lengths are known to the device only: every block adds up the whole call's work from them
// (a few hundred lengths: one load a lane) and finds which item, and which of S equal pieces of its tokens, is its own, so that
// about kvTarget pieces come out whatever the lengths.  Pieces leave (m, sum p, numerators) in the workspace, and a second
// kernel joins them in order.
#pragma once

#include "qp_kv.hpp"

namespace qp {

constexpr int kAtThreads = 256, kAtWaves = 4;
constexpr uint32_t kAtStep = 32;                 // tokens of a wave's step
constexpr uint32_t kAtTile = kAtStep * kAtWaves; // tokens that work is counted in
#ifndef QP_KV_TARGET
#define QP_KV_TARGET 1024
#endif
// pieces that a call is cut into: what the chip runs at the same time
template <int NCT> constexpr uint32_t kAtTarget = NCT == 1 ? QP_KV_TARGET : QP_KV_TARGET / 2;
// tiles that a piece has at least: joining costs a kernel and a pass over the pieces, more than it takes to go through these
#ifndef QP_KV_LEAST
#define QP_KV_LEAST 4
#endif
constexpr uint32_t kAtLeast = QP_KV_LEAST;
constexpr float kAtHeadroom = 8.0f;              // log2 that a score may lie above its column's m

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// The workspace: [0] columns that were split; a record for each; (m, sum) and numerators of the pieces, in units of 16 NCT columns.
struct AtWork {
    uint32_t *header;
    u32x4 *cols;
    float2 *sums;
    float *nums;
    uint32_t most_cols, most_units;
};
constexpr size_t kAtHeader = 256;
inline uint64_t at_items(uint32_t nct, const KvLayer &c, uint32_t group)      // a row has one for each 64 nct columns begun
{
    const uint64_t rows = c.rows < c.tokens ? c.rows : c.tokens;
    return c.kv_heads * ((uint64_t)c.tokens * group / (64u * nct) + rows);
}
// An item of n tiles is cut up if n exceeds a piece's share, and then into less than n / share + 1 <= 2 n / share pieces: twice
// the target at most for all of them, in target items at most.
template <int NCT> AtWork at_work(void *ws, const KvLayer &c, uint32_t dim, uint32_t group, size_t &bytes)
{
    const uint64_t tiles = (((uint64_t)c.pages_per_row << c.page_shift) + kAtTile - 1u) / kAtTile, items = at_items(NCT, c, group);
    const uint64_t columns = (uint64_t)c.tokens * c.kv_heads * group, target = kAtTarget<NCT>;
    // a piece's share is at least kAtLeast tiles, a quarter of them where the waves split columns
    const uint64_t least = (uint64_t)c.tokens * group > 16u * NCT ? (kAtLeast + 3u) / 4u : kAtLeast;
    uint64_t pieces = tiles <= least ? 0u : 2u * target, cols = tiles <= least ? 0u : target * 64u * NCT;
    if (items < 2u * target && items * tiles < pieces) pieces = items * tiles;   // (one tile each at the least)
    if (columns < cols) cols = columns;
    AtWork w{};
    w.most_units = (uint32_t)(pieces * ((uint64_t)c.tokens * group > 16u * NCT ? 4u : 1u));
    w.most_cols = (uint32_t)cols;
    const size_t sums = kAtHeader + (size_t)cols * sizeof(u32x4), nums = sums + (size_t)w.most_units * 16u * NCT * sizeof(float2);
    bytes = nums + (size_t)w.most_units * 16u * NCT * dim * sizeof(float);
    if (char *p = static_cast<char *>(ws)) {
        w.header = reinterpret_cast<uint32_t *>(p);
        w.cols = reinterpret_cast<u32x4 *>(p + kAtHeader);
        w.sums = reinterpret_cast<float2 *>(p + sums);
        w.nums = reinterpret_cast<float *>(p + nums);
    }
    return w;
}

// ---- which piece of which item a block has ---------------------------------------------------------------------------------
struct AtRow {               // a row's items: n4 with the columns split among the waves, n1 (0 or 1) with the tokens split
    uint32_t n4, n1, tiles, cols;
};
template <int NCT> __device__ __forceinline__ AtRow at_row(const KvLayer &c, const KvAttn &a, uint32_t r)
{
    const KvRow row = kv_row(c, r);
    AtRow o;
    o.cols = (uint32_t)row.count * a.group;
    const uint32_t full = o.cols / (64u * NCT), rest = o.cols % (64u * NCT);
    o.n1 = rest != 0u && rest <= 16u * NCT ? 1u : 0u;
    o.n4 = full + (rest > 16u * NCT ? 1u : 0u);
    const int64_t from = a.window ? (int64_t)row.length - row.count - a.window + 1 : 0;
    const uint32_t lo = from > 0 ? (uint32_t)from / kAtTile : 0u, hi = ((uint32_t)row.length + kAtTile - 1u) / kAtTile;
    o.tiles = hi > lo ? hi - lo : 1u;
    return o;
}
struct AtPiece {
    uint32_t row, head, ct, s, pieces;       // pieces: at most so many of the item's tokens
    uint32_t per;                            // tiles that a piece should have
    uint32_t unit, unit_step;                // where the item's partial results go (piece s at unit + s unit_step)
    uint32_t col;                            // ... and its columns' records
};
// Inclusive prefix sums of three numbers over the block; `part` holds each wave's totals.
__device__ __forceinline__ void at_scan(uint32_t (&x)[3], uint32_t (*part)[3], uint32_t (&total)[3])
{
    const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
    for (uint32_t d = 1; d < (uint32_t)kWave; d *= 2u)
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const uint32_t o = __shfl_up(x[i], d, kWave);
            if (lane >= d) x[i] += o;
        }
    if (lane == kWave - 1u)
#pragma unroll
        for (int i = 0; i < 3; ++i) part[wave][i] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        total[i] = 0u;
#pragma unroll
        for (uint32_t w = 0; w < (uint32_t)kAtWaves; ++w) {
            x[i] += w < wave ? part[w][i] : 0u;
            total[i] += part[w][i];
        }
    }
}
__device__ __forceinline__ uint64_t at_wave_sum(uint64_t v)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) v += ((uint64_t)__shfl_xor((uint32_t)(v >> 32), d, kWave) << 32) + __shfl_xor((uint32_t)v, d, kWave);
    return v;
}

// False: the call has fewer pieces than blocks.
template <int NCT>
__device__ __forceinline__ bool at_find(const KvLayer &c, const KvAttn &a, const AtWork &w, uint32_t block, AtPiece &mine)
{
    __shared__ uint32_t part[kAtWaves][3];
    __shared__ uint64_t work[kAtWaves];
    __shared__ AtPiece found;
    __shared__ uint32_t have, split;
    const uint32_t tid = threadIdx.x;
    const AtRow none{0u, 0u, 1u, 0u};
    const AtRow mine0 = tid < c.rows ? at_row<NCT>(c, a, tid) : none;      // (most calls have no more rows than that)
    uint64_t cost = (uint64_t)mine0.tiles * (mine0.n4 * 4u + mine0.n1);
    for (uint32_t r = tid + kAtThreads; r < c.rows; r += kAtThreads) {
        const AtRow o = at_row<NCT>(c, a, r);
        cost += (uint64_t)o.tiles * (o.n4 * 4u + o.n1);
    }
    cost = at_wave_sum(cost);
    if (tid % kWave == 0u) work[tid / kWave] = cost;
    if (tid == 0u) have = split = 0u;
    __syncthreads();
    const uint64_t all = (work[0] + work[1] + work[2] + work[3]) * c.kv_heads;
    const uint64_t share = max((all + kAtTarget<NCT> - 1u) / kAtTarget<NCT>, (uint64_t)kAtLeast);
    const uint32_t per1 = (uint32_t)min(share, (uint64_t)0x7fffffffu), per4 = (uint32_t)min((share + 3u) / 4u, (uint64_t)0x7fffffffu);
    uint32_t before[3] = {0u, 0u, 0u};                   // blocks, units, columns of the rows so far
    for (uint32_t r0 = 0; r0 < c.rows; r0 += kAtThreads) {
        const uint32_t r = r0 + tid;
        const AtRow o = r0 == 0u ? mine0 : r < c.rows ? at_row<NCT>(c, a, r) : none;
        const uint32_t s4 = (o.tiles + per4 - 1u) / per4, s1 = (o.tiles + per1 - 1u) / per1;
        const uint32_t last = o.n1 ? o.cols - o.n4 * 64u * NCT : 0u;          // columns of the item with split tokens
        const uint32_t b4 = c.kv_heads * o.n4 * s4, b1 = c.kv_heads * o.n1 * s1;
        const uint32_t u4 = s4 > 1u ? 4u * b4 : 0u, u1 = s1 > 1u ? b1 : 0u;
        const uint32_t k4 = s4 > 1u ? c.kv_heads * (o.cols - last) : 0u, k1 = s1 > 1u ? c.kv_heads * last : 0u;
        uint32_t x[3] = {b4 + b1, u4 + u1, k4 + k1}, total[3];
        at_scan(x, part, total);
        const uint32_t eb = before[0] + x[0], eu = before[1] + x[1], ek = before[2] + x[2];      // ends
        const uint32_t pb = eb - (b4 + b1), pu = eu - (u4 + u1), pk = ek - (k4 + k1);
        // (always so where the rows' tokens do not overlap: what the host sized the grid and the workspace for)
        const bool fits = pb <= gridDim.x && eb <= gridDim.x && pu <= w.most_units && eu <= w.most_units && pk <= w.most_cols && ek <= w.most_cols;
        if (fits && k4 + k1 != 0u) atomicMax(&split, ek);
        if (fits && block >= pb && block < eb) {
            uint32_t i = block - pb;
            AtPiece f;
            f.row = r;
            if (i < b4) {        // the last columns, which see the most tokens, first; heads side by side: an XCD per head
                f.head = i % c.kv_heads;
                i /= c.kv_heads;
                f.s = i % s4;
                f.ct = o.n4 - 1u - i / s4;
                f.pieces = s4;
                f.per = per4;
                f.unit = pu + (f.ct * c.kv_heads + f.head) * s4 * 4u;
                f.unit_step = 4u;
                f.col = pk + f.ct * 64u * NCT * c.kv_heads + f.head * min(64u * NCT, o.cols - f.ct * 64u * NCT);
            } else {
                i -= b4;
                f.head = i % c.kv_heads;
                f.s = i / c.kv_heads;
                f.ct = o.n4;
                f.pieces = s1;
                f.per = per1;
                f.unit = pu + u4 + f.head * s1;
                f.unit_step = 1u;
                f.col = pk + k4 + f.head * last;
            }
            found = f;
            have = 1u;
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) before[k] += total[k];
        __syncthreads();
        if (block < before[0] && block != 0u) break;     // (block 0 goes on: it says how many columns were split)
    }
    if (block == 0u && tid == 0u) w.header[0] = split;
    mine = found;
    return have != 0u;
}

// ---- a wave's work -----------------------------------------------------------------------------------------------------------
// The constants of at_codes in vector registers: (w & mask) | magic is one instruction then (it takes one scalar operand only),
// and two with the constants in it.
struct AtMagic {
    uint32_t big, small;
    __device__ __forceinline__ AtMagic() : big(0x64006400u), small(0x54005400u)
    {
#if defined(__AMDGCN__)
        asm volatile("" : "+v"(big), "+v"(small));
#endif
    }
};
__device__ __forceinline__ f16x8 at_codes(uint32_t w, const AtMagic &k)
{
    const f16x2 big = {(_Float16)-1032.0f, (_Float16)-1032.0f}, small = {(_Float16)-72.0f, (_Float16)-72.0f};
    const uint32_t x = w >> 8;
    const f16x2 a = __builtin_bit_cast(f16x2, (w & 0x000f000fu) | k.big) + big;
    const f16x2 b = __builtin_bit_cast(f16x2, (w & 0x00f000f0u) | k.small) + small;
    const f16x2 d = __builtin_bit_cast(f16x2, (x & 0x000f000fu) | k.big) + big;
    const f16x2 e = __builtin_bit_cast(f16x2, (x & 0x00f000f0u) | k.small) + small;
    return f16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}
__device__ __forceinline__ float at_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

template <int D, int NCT, int DT> struct AtWave {
    static constexpr int KS = (D + 31) / 32;         // words of a lane of a key, and steps of the first product
    static constexpr int NB = D / 16;                // words of a lane of eight tokens' values, and blocks of the answer
    static constexpr int PIECES = DT == QP_F32 ? 2 : 1;
    f16x8 q[NCT][PIECES][KS];
    f32x4 o[NCT][NB];
    float m[NCT], f[NCT], bq[NCT], l[NCT], lv[NCT];
    int32_t lo[NCT], hi[NCT];                        // the tokens that this lane's column sees
    float norm, sv_most;                             // N, and the largest value scale that it is good for
    int32_t norm_exp;

    struct Raw {
        uint32_t k[2][KS], v[NB];
        float2 grid;                                 // lanes 0..31: keys, 32..63: values
    };

    __device__ __forceinline__ void load_query(const KvLayer &c, const KvView &qv, const KvAttn &a, const KvRow &row, uint32_t head,
                                               uint32_t col0, uint32_t cols)
    {
        const uint32_t lane = threadIdx.x % kWave, g = lane / 16u, n = lane % 16u;
#pragma unroll
        for (int t = 0; t < NCT; ++t) {
            const uint32_t col = col0 + 16u * t + n;
            const bool is = col < cols;
            const uint32_t i = is ? col / a.group : 0u, h = head * a.group + (is ? col % a.group : 0u);
            const unsigned char *src = qv.data + ((uint64_t)row.begin + i) * qv.token_stride + (uint64_t)h * qv.head_stride;
            float x[KS][8];
            float top = 0.0f;
            bool bad = false;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const uint32_t unit = g * KS + s;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[s][e] = 0.0f;
                if (is && unit * 8u < (uint32_t)D) {
                    if constexpr (DT == QP_F32) {
                        const f32x4 u = reinterpret_cast<const f32x4 *>(src)[2u * unit], v = reinterpret_cast<const f32x4 *>(src)[2u * unit + 1u];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            x[s][e] = u[e];
                            x[s][4 + e] = v[e];
                        }
                    } else {
                        Vec16<DT>::load(src, unit, x[s]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    bad |= (__float_as_uint(x[s][e]) & 0x7f800000u) == 0x7f800000u;
                    top = fmaxf(top, fabsf(x[s][e]));
                }
            }
            top = fmaxf(top, kv_xor_f32(top, 16));
            top = fmaxf(top, kv_xor_f32(top, 32));
            uint32_t any = bad ? 1u : 0u;
            any |= __shfl_xor(any, 16, kWave);
            any |= __shfl_xor(any, 32, kWave);
            int32_t ex = 15;
            if (top > 0.0f && any == 0u) (void)frexpf(top, &ex);
            const int32_t up = min(15 - ex, 100);        // q 2^up: the largest element in [2^14, 2^15)
            float sum = 0.0f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                f16x8 high, low;
#pragma unroll
                for (int e = 0; e < 8; ++e) {            // code order 0, 4, 1, 5, 2, 6, 3, 7
                    const int src_e = e % 2 * 4 + e / 2;
                    const float y = any ? 0.0f : ldexpf(x[s][src_e], up);
                    sum += y;
                    high[e] = (_Float16)y;
                    low[e] = (_Float16)(y - (float)high[e]);
                }
                q[t][0][s] = high;
                if constexpr (PIECES == 2) q[t][1][s] = low;
            }
            sum += kv_xor_f32(sum, 16);
            sum += kv_xor_f32(sum, 32);
            bq[t] = any ? __uint_as_float(0x7fc00000u) : sum;
            // f > 0, and m f finite from the start: a masked score, -inf, gives p = 0 by itself
            f[t] = fmaxf(ldexpf(a.scale * 1.44269504088896341f, -up), 0x1p-126f);
            m[t] = -0x1p127f / fmaxf(f[t], 1.0f);
            l[t] = lv[t] = 0.0f;
#pragma unroll
            for (int b = 0; b < NB; ++b) o[t][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            const int64_t pos = (int64_t)row.length - row.count + i;
            hi[t] = !is ? 0x7fffffff : a.causal ? (int32_t)max((int64_t)0, min(pos + 1, (int64_t)row.length)) : row.length;
            lo[t] = is && a.window ? (int32_t)max((int64_t)0, pos - (int64_t)a.window + 1) : 0;
        }
        norm = 1.0f;
        norm_exp = 0;
        sv_most = 0.0f;
    }

    // 32 tokens from `t0` on, of the page that they all lie in
    __device__ __forceinline__ void load(Raw &x, const unsigned char *slab, uint32_t t0, uint32_t page_shift, int32_t length, bool there) const
    {
        const uint32_t lane = threadIdx.x % kWave, g = lane / 16u, n = lane % 16u;
        const uint32_t pt = 1u << page_shift, in = t0 & (pt - 1u);
        const uint32_t *kc = reinterpret_cast<const uint32_t *>(slab);
        const uint32_t *vc = kc + (size_t)pt * (D / kKvCodes);
        const float2 *grids = reinterpret_cast<const float2 *>(vc + (size_t)pt * (D / kKvCodes));
#pragma unroll
        for (int j = 0; j < 2; ++j)      // (the last words of a key that is no multiple of 32 long lie behind it, in the slab; their queries are 0)
            __builtin_memcpy(x.k[j], kc + (size_t)(in + 8u * (n / 4u) + 4u * j + n % 4u) * (D / kKvCodes) + g * KS, sizeof x.k[j]);
        __builtin_memcpy(x.v, vc + (size_t)(in / 8u + g) * D + n * NB, sizeof x.v);
        x.grid = grids[(lane < 32u ? 0u : pt) + in + lane % 32u];
        if (!there || (int32_t)(t0 + lane % 32u) >= length) x.grid = float2{0.0f, 0.0f};   // (never written: may be anything)
    }

    // the maximum or N moves
    __device__ __forceinline__ void rescale(const float (&top)[NCT], float sv_top)
    {
        sv_top = fmaxf(sv_top, kv_xor_f32(sv_top, 16));
        sv_top = fmaxf(sv_top, kv_xor_f32(sv_top, 32));
        float ratio = 1.0f;
        if (sv_top > sv_most) {          // (the same in all lanes)
            int32_t ex;
            (void)frexpf(sv_top, &ex);
            const int32_t now = 6 - ex;
            ratio = sv_most > 0.0f ? ldexpf(1.0f, now - norm_exp) : 1.0f;
            norm_exp = now;
            norm = ldexpf(1.0f, now);
            sv_most = ldexpf(1.0f, ex + 1);
        }
#pragma unroll
        for (int t = 0; t < NCT; ++t) {
            float x = fmaxf(top[t], kv_xor_f32(top[t], 16));
            x = fmaxf(x, kv_xor_f32(x, 32));
            const float next = fmaxf(m[t], x);
            const float alpha = at_exp2((m[t] - next) * f[t]);
            m[t] = next;
            l[t] *= alpha;
            lv[t] *= alpha;
            const float beta = alpha * ratio;
#pragma unroll
            for (int b = 0; b < NB; ++b) o[t][b] *= beta;
        }
    }

    // What a step makes of a grid; lanes 0..31: keys, 32..63: values.
    static __device__ __forceinline__ float2 centred(float2 grid) { return float2{grid.y, fmaf(8.0f, grid.y, grid.x)}; }

    // `key(j, k)`, `value(b)`: the fragments; `mem`: scales and lo + 8 scale of 32 keys, then of 32 values
    template <typename Key, typename Value>
    __device__ __forceinline__ void step(const Key &key, const Value &value, const float2 *mem, uint32_t t0, bool whole, bool there)
    {
        const uint32_t lane = threadIdx.x % kWave, g = lane / 16u;
        float sk[8], bk[8], sv[8], bv[8];                 // of tokens 8 g + i
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 gk = mem[8u * g + i], gv = mem[32u + 8u * g + i];
            sk[i] = gk.x;
            bk[i] = gk.y;
            sv[i] = gv.x;
            bv[i] = gv.y;
        }
        f32x4 s[NCT][2];
#pragma unroll
        for (int t = 0; t < NCT; ++t) s[t][0] = s[t][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const f16x8 a = key(j, k);
#pragma unroll
                for (int t = 0; t < NCT; ++t)
#pragma unroll
                    for (int z = PIECES - 1; z >= 0; --z) s[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, q[t][z][k], s[t][j], 0, 0, 0);
            }
        float y[NCT][8], top[NCT];
        float sv_top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sv_top = fmaxf(sv_top, sv[i]);
        bool moves = sv_top > sv_most;
#pragma unroll
        for (int t = 0; t < NCT; ++t) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[t][i] = fmaf(s[t][i / 4][i % 4], sk[i], bk[i] * bq[t]);
            if (!whole) {
                uint32_t from = t0 + 8u * g;
#if defined(__AMDGCN__)
                asm volatile("" : "+v"(from));   // (keeps this inside the branch: else 24 instructions of it are in every step)
#endif
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int32_t tok = (int32_t)from + i;
                    if (!there || tok < lo[t] || tok >= hi[t]) y[t][i] = -INFINITY;
                }
            }
            top[t] = y[t][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top[t] = fmaxf(top[t], y[t][i]);
            moves |= (top[t] - m[t]) * f[t] > kAtHeadroom;
        }
        if (__ballot(moves) != 0ull) rescale(top, sv_top);
        f16x8 p[NCT][PIECES];
#pragma unroll
        for (int i = 0; i < 8; ++i) sv[i] *= norm;
#pragma unroll
        for (int t = 0; t < NCT; ++t) {
            const float mf = -m[t] * f[t];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float e = at_exp2(fmaf(y[t][i], f[t], mf));
                l[t] += e;
                lv[t] = fmaf(e, bv[i], lv[t]);
                const float w = e * sv[i];
                const int at = i % 4 * 2 + i / 4;         // code order
                p[t][0][at] = (_Float16)w;
                if constexpr (PIECES == 2) p[t][1][at] = (_Float16)(w - (float)p[t][0][at]);
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const f16x8 a = value(b);
#pragma unroll
            for (int t = 0; t < NCT; ++t)
                if constexpr (PIECES == 1) {
                    o[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, p[t][0], o[t][b], 0, 0, 0);
                } else {
                    // added up outside the matrix unit: its sums of the whole row drift by a few 2^-18 (measured 3e-6 of the answer at
                    // 1000 tokens; so 7e-7, the plain fp32 form's error)
                    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
                    const f32x4 part = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, p[t][1], zero, 0, 0, 0);
                    o[t][b] += __builtin_amdgcn_mfma_f32_16x16x32_f16(a, p[t][0], part, 0, 0, 0);
                }
        }
    }

    // One wave for itself: 32 tokens that it has loaded.  `mem`: this wave's own.
    __device__ __forceinline__ void step_alone(const Raw &x, float2 *mem, const AtMagic &magic, uint32_t t0, bool whole, bool there)
    {
        mem[threadIdx.x % kWave] = centred(x.grid);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        step([&](int j, int k) { return at_codes(x.k[j][k], magic); }, [&](int b) { return at_codes(x.v[b], magic); }, mem, t0, whole, there);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }

    // The sums of all lanes of a column; o becomes the numerator, m the maximum in log2.
    __device__ __forceinline__ void finish()
    {
        const float back = ldexpf(1.0f, -norm_exp);
#pragma unroll
        for (int t = 0; t < NCT; ++t) {
            l[t] += kv_xor_f32(l[t], 16);
            l[t] += kv_xor_f32(l[t], 32);
            lv[t] += kv_xor_f32(lv[t], 16);
            lv[t] += kv_xor_f32(lv[t], 32);
            m[t] = l[t] == 0.0f ? -3.402823466e38f : m[t] * f[t];   // (a column that saw nothing: below any other)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[t][b][r] = fmaf(o[t][b][r], back, lv[t]);
        }
    }
};

#ifndef QP_W1
#define QP_W1 2
#endif
#ifndef QP_W2
#define QP_W2 2
#endif
template <int D, int NCT, int DT> constexpr int kAtResident = D > 128 ? 1 : NCT == 1 ? QP_W1 : DT == QP_F32 ? 1 : QP_W2;
__device__ __forceinline__ uint32_t at_bf16(float f)
{
    const uint32_t u = __float_as_uint(f);
    return (u & 0x7fffffffu) > 0x7f800000u ? (u >> 16) | 0x40u : (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

template <int D, int NCT, int DT>
__global__ __launch_bounds__(kAtThreads, (kAtResident<D, NCT, DT>)) void k_kv_attention(KvLayer c, KvView qv, KvView out, KvAttn a, AtWork w)
{
    using Wave = AtWave<D, NCT, DT>;
    constexpr int NB = Wave::NB;
    // either: two waves' numerators and (m, sum), when the four waves of an item with split tokens are joined, and their grids;
    // or: two steps' fragments, keys' and values', and grids, which the four waves of an item with split columns share
    constexpr int kFrags = 2 * Wave::KS + NB;
    struct Alone {
        float nums[2][16 * NCT][D + 4];
        float2 sums[2][16 * NCT];
        float2 grids[kAtWaves][64];
    };
    struct Shared {
        f16x8 frags[2][kFrags][kWave];
        float2 grids[2][64];
    };
    __shared__ __align__(16) unsigned char mem[sizeof(Alone) > sizeof(Shared) ? sizeof(Alone) : sizeof(Shared)];
    Alone &alone = *reinterpret_cast<Alone *>(mem);
    Shared &shared = *reinterpret_cast<Shared *>(mem);
    AtPiece me;
    if (!at_find<NCT>(c, a, w, blockIdx.x, me)) return;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, g = lane / 16u, n = lane % 16u;
    const uint32_t r = __builtin_amdgcn_readfirstlane(me.row), head = __builtin_amdgcn_readfirstlane(me.head);
    const KvRow row = kv_row(c, r);
    const uint32_t cols = (uint32_t)row.count * a.group, item0 = me.ct * 64u * NCT, item1 = min(cols, item0 + 64u * NCT);
    const bool split_tokens = me.unit_step == 1u;
    const uint32_t col0 = item0 + (split_tokens ? 0u : wave * 16u * NCT);
    // the tokens that any of the columns [from, to) sees
    const auto range = [&](uint32_t from, uint32_t to, uint32_t &t_lo, uint32_t &t_hi) {
        const int64_t first = (int64_t)row.length - row.count + from / a.group, last = (int64_t)row.length - row.count + (to - 1u) / a.group;
        t_lo = a.window ? (uint32_t)max((int64_t)0, first - (int64_t)a.window + 1) : 0u;
        t_hi = a.causal ? (uint32_t)max((int64_t)0, min(last + 1, (int64_t)row.length)) : (uint32_t)row.length;
        if (t_lo > t_hi) t_lo = t_hi;
    };
    uint32_t t_lo, t_hi;
    range(item0, item1, t_lo, t_hi);
    const uint32_t first = t_lo / kAtTile, tiles = t_hi > t_lo ? (t_hi + kAtTile - 1u) / kAtTile - first : 0u;
    const uint32_t pieces = max(1u, min(me.pieces, (tiles + me.per - 1u) / me.per));
    if (me.pieces > 1u && me.s == 0u)         // the columns' records for the kernel that joins them
        for (uint32_t k = threadIdx.x; k < item1 - item0; k += kAtThreads) {
            const uint32_t col = item0 + k, unit = me.unit + (split_tokens ? 0u : k / (16u * NCT));
            const uint32_t place = (uint32_t)(row.begin + (int32_t)(col / a.group)), h = head * a.group + col % a.group;
            w.cols[me.col + k] = u32x4{unit * (16u * NCT) + k % (16u * NCT), pieces > 1u ? pieces : 0u, me.unit_step * (16u * NCT), place * (c.kv_heads * a.group) + h};
        }
    if (me.s >= pieces) return;
    const uint32_t tile_a = first + (uint32_t)((uint64_t)tiles * me.s / pieces), tile_b = first + (uint32_t)((uint64_t)tiles * (me.s + 1u) / pieces);
    uint32_t a0 = tile_a * kAtTile, a1 = min(tile_b * kAtTile, t_hi);        // this piece's tokens
    const uint32_t col1 = min(item1, col0 + 16u * NCT);
    const uint32_t b0 = a0, b1 = a1;
    if (!split_tokens && col0 < col1) {       // ... and what this wave's columns see of them
        uint32_t w_lo, w_hi;
        range(col0, col1, w_lo, w_hi);
        a0 = max(a0, w_lo / kAtStep * kAtStep);
        a1 = min(a1, w_hi);
    }
    if (col0 >= col1) a1 = a0;
    Wave x;
    x.load_query(c, qv, a, row, head, col0, col1);
    int32_t sees_lo = 0, sees_hi = 0x7fffffff;                               // what all of the wave's columns see
#pragma unroll
    for (int t = 0; t < NCT; ++t) {
        sees_lo = max(sees_lo, x.lo[t]);
        sees_hi = min(sees_hi, x.hi[t]);
    }
#pragma unroll
    for (int d = 1; d < 16; d *= 2) {
        sees_lo = max(sees_lo, (int32_t)__shfl_xor((uint32_t)sees_lo, d, kWave));
        sees_hi = min(sees_hi, (int32_t)__shfl_xor((uint32_t)sees_hi, d, kWave));
    }
    const auto slab_at = [&](uint32_t t, bool &there) {
        const int32_t page = __builtin_amdgcn_readfirstlane(kv_page(c, r, t >> c.page_shift));
        there = page >= 0;
        return kv_slab(c, there ? page : 0, head);
    };
    const AtMagic magic;
    if (split_tokens) {
        uint32_t t0 = a0 + wave * kAtStep;
        typename Wave::Raw cur, nxt;
        bool there = false, there_next = false;
        if (t0 < a1) {
            const unsigned char *slab = slab_at(t0, there);
            x.load(cur, slab, t0, c.page_shift, row.length, there);
        }
        for (; t0 < a1; t0 += kAtTile) {
            if (t0 + kAtTile < a1) {
                const unsigned char *slab = slab_at(t0 + kAtTile, there_next);
                x.load(nxt, slab, t0 + kAtTile, c.page_shift, row.length, there_next);
            }
            const bool whole = there && (int32_t)t0 >= sees_lo && (int32_t)(t0 + kAtStep) <= sees_hi;
            x.step_alone(cur, alone.grids[wave], magic, t0, whole, there);
            cur = nxt;
            there = there_next;
        }
    } else {
        // every wave takes a quarter of a step's words apart for all of them; while a step runs the next one's fragments go to the
        // other half of LDS and the words of the one after it are on their way
        constexpr int kMine = (kFrags + kAtWaves - 1) / kAtWaves;
        uint32_t words[kMine];
        float2 grid{0.0f, 0.0f};
        bool there = false, there_next = false, there_far = false;
        const auto fetch = [&](uint32_t t, bool &is) {
            const unsigned char *slab = slab_at(t, is);
            const uint32_t pt = 1u << c.page_shift, in = t & (pt - 1u);
            const uint32_t *kc = reinterpret_cast<const uint32_t *>(slab), *vc = kc + (size_t)pt * (D / kKvCodes);
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const uint32_t fr = kAtWaves * i + wave;      // fragment: keys (j, k), then values (b)
                if (fr < 2u * Wave::KS)
                    words[i] = kc[(size_t)(in + 8u * (n / 4u) + 4u * (fr / Wave::KS) + n % 4u) * (D / kKvCodes) + g * Wave::KS + fr % Wave::KS];
                else if (fr < (uint32_t)kFrags)
                    words[i] = vc[(size_t)(in / 8u + g) * D + n * NB + (fr - 2u * Wave::KS)];
            }
            if (wave == 0u) {
                const float2 *grids = reinterpret_cast<const float2 *>(vc + (size_t)pt * (D / kKvCodes));
                grid = grids[(lane < 32u ? 0u : pt) + in + lane % 32u];
                if (!is || (int32_t)(t + lane % 32u) >= row.length) grid = float2{0.0f, 0.0f};
            }
        };
        const auto put = [&](uint32_t half) {
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const uint32_t fr = kAtWaves * i + wave;
                if (fr < (uint32_t)kFrags) shared.frags[half][fr][lane] = at_codes(words[i], magic);
            }
            if (wave == 0u) shared.grids[half][lane] = Wave::centred(grid);
        };
        uint32_t t = b0, half = 0u;
        if (t < b1) {
            fetch(t, there);
            put(0u);
            if (t + kAtStep < b1) fetch(t + kAtStep, there_next);
        }
        __syncthreads();
        for (; t < b1; t += kAtStep) {
            if (t + kAtStep < b1) {
                put(half ^ 1u);
                if (t + 2u * kAtStep < b1) fetch(t + 2u * kAtStep, there_far);
            }
            if (t >= a0 && t < a1) {
                const bool whole = there && (int32_t)t >= sees_lo && (int32_t)(t + kAtStep) <= sees_hi;
                x.step([&](int j, int k) { return shared.frags[half][j * Wave::KS + k][lane]; },
                       [&](int b) { return shared.frags[half][2 * Wave::KS + b][lane]; }, shared.grids[half], t, whole, there);
            }
            __syncthreads();
            half ^= 1u;
            there = there_next;
            there_next = there_far;
        }
    }
    x.finish();
    if (split_tokens) {                       // waves 2, 3 into 0, 1, then 1 into 0
#pragma unroll
        for (uint32_t half = 2; half >= 1; half /= 2) {
            if (wave >= half && wave < 2u * half) {
#pragma unroll
                for (int t = 0; t < NCT; ++t) {
                    float *dst = &alone.nums[wave - half][16 * t + n][4u * NB * g];
#pragma unroll
                    for (int r4 = 0; r4 < 4; ++r4)
#pragma unroll
                        for (int b = 0; b < NB; ++b) dst[r4 * NB + b] = x.o[t][b][r4];
                    if (g == 0u) alone.sums[wave - half][16 * t + n] = float2{x.m[t], x.l[t]};
                }
            }
            __syncthreads();
            if (wave < half) {
#pragma unroll
                for (int t = 0; t < NCT; ++t) {
                    const float *src = &alone.nums[wave][16 * t + n][4u * NB * g];
                    const float2 other = alone.sums[wave][16 * t + n];
                    const float top = fmaxf(x.m[t], other.x), ea = at_exp2(x.m[t] - top), eb = at_exp2(other.x - top);
                    x.m[t] = top;
                    x.l[t] = fmaf(x.l[t], ea, other.y * eb);
#pragma unroll
                    for (int r4 = 0; r4 < 4; ++r4)
#pragma unroll
                        for (int b = 0; b < NB; ++b) x.o[t][b][r4] = fmaf(x.o[t][b][r4], ea, src[r4 * NB + b] * eb);
                }
            }
            __syncthreads();
        }
        if (wave != 0u) return;
    }
#pragma unroll
    for (int t = 0; t < NCT; ++t) {
        const uint32_t col = col0 + 16u * t + n;
        if (col >= col1) continue;
        float v[4 * NB];
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
#pragma unroll
            for (int b = 0; b < NB; ++b) v[r4 * NB + b] = x.o[t][b][r4];
        if (pieces > 1u) {
            const size_t at = (size_t)(me.unit + me.s * me.unit_step + (split_tokens ? 0u : wave)) * (16u * NCT) + 16u * t + n;
            if (g == 0u) w.sums[at] = float2{x.m[t], x.l[t]};
            f32x4 *dst = reinterpret_cast<f32x4 *>(w.nums + at * D + 4u * NB * g);
#pragma unroll
            for (int b = 0; b < NB; ++b) dst[b] = f32x4{v[4 * b], v[4 * b + 1], v[4 * b + 2], v[4 * b + 3]};
            continue;
        }
        const float inv = x.l[t] == 0.0f ? 0.0f : 1.0f / x.l[t];
        unsigned char *dst = out.data + ((uint64_t)row.begin + col / a.group) * out.token_stride + (uint64_t)(head * a.group + col % a.group) * out.head_stride;
        if constexpr (DT == QP_F32) {
            f32x4 *d4 = reinterpret_cast<f32x4 *>(dst) + NB * g;
#pragma unroll
            for (int b = 0; b < NB; ++b) d4[b] = f32x4{v[4 * b] * inv, v[4 * b + 1] * inv, v[4 * b + 2] * inv, v[4 * b + 3] * inv};
        } else {
            u32x2 *d2 = reinterpret_cast<u32x2 *>(dst) + NB * g;
#pragma unroll
            for (int b = 0; b < NB; ++b)
                d2[b] = u32x2{at_bf16(v[4 * b] * inv) | (at_bf16(v[4 * b + 1] * inv) << 16),
                              at_bf16(v[4 * b + 2] * inv) | (at_bf16(v[4 * b + 3] * inv) << 16)};
        }
    }
}

// ---- the pieces of a column, joined: a block a column, every fourth piece a wave ----------------------------------------------
template <int D, int NCT, int DT> __global__ __launch_bounds__(kAtThreads) void k_kv_join(KvView out, uint32_t q_heads, AtWork w)
{
    constexpr int PER = (D + kWave - 1) / kWave;
    __shared__ float weight[2 * kAtTarget<NCT>];
    __shared__ float part[kAtWaves][D], top_of[kAtWaves], sum_of[kAtWaves];
    const uint32_t tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
    const uint32_t count = w.header[0];
    for (uint32_t k = blockIdx.x; k < count; k += gridDim.x) {
        const u32x4 rec = w.cols[k];
        const uint32_t pieces = rec[1];
        if (pieces == 0u) continue;           // its item came out in one piece after all
        float top = -3.402823466e38f;
        for (uint32_t i = tid; i < pieces; i += kAtThreads) top = fmaxf(top, w.sums[rec[0] + (size_t)i * rec[2]].x);
        top = wave_max(top);
        if (lane == 0u) top_of[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(top_of[0], top_of[1]), fmaxf(top_of[2], top_of[3]));
        float sum = 0.0f;
        for (uint32_t i = tid; i < pieces; i += kAtThreads) {
            const float2 ml = w.sums[rec[0] + (size_t)i * rec[2]];
            const float e = at_exp2(ml.x - top);
            weight[i] = e;
            sum += e * ml.y;
        }
        sum += dpp_f32<kDppQuadSwap1>(sum);
        sum += dpp_f32<kDppQuadSwap2>(sum);
        sum += dpp_f32<kDppHalfMirror>(sum);
        sum += dpp_f32<kDppRowMirror>(sum);
        sum += kv_xor_f32(sum, 16);
        sum += kv_xor_f32(sum, 32);
        if (lane == 0u) sum_of[wave] = sum;
        __syncthreads();
        float acc[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) acc[e] = 0.0f;
#pragma unroll 4
        for (uint32_t i = wave; i < pieces; i += kAtWaves) {
            const float *src = w.nums + (rec[0] + (size_t)i * rec[2]) * D;
            const float e = weight[i];
#pragma unroll
            for (int z = 0; z < PER; ++z)
                if (lane + kWave * z < (uint32_t)D) acc[z] = fmaf(e, src[lane + kWave * z], acc[z]);
        }
#pragma unroll
        for (int z = 0; z < PER; ++z)
            if (lane + kWave * z < (uint32_t)D) part[wave][lane + kWave * z] = acc[z];
        __syncthreads();
        const float l = (sum_of[0] + sum_of[1]) + (sum_of[2] + sum_of[3]);
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        unsigned char *dst = out.data + (uint64_t)(rec[3] / q_heads) * out.token_stride + (uint64_t)(rec[3] % q_heads) * out.head_stride;
        for (uint32_t d = tid; d < (uint32_t)D; d += kAtThreads) {
            const float v = ((part[0][d] + part[1][d]) + (part[2][d] + part[3][d])) * inv;
            if constexpr (DT == QP_F32) reinterpret_cast<float *>(dst)[d] = v;
            else reinterpret_cast<uint16_t *>(dst)[d] = (uint16_t)at_bf16(v);
        }
        __syncthreads();                      // (the shared arrays are used again)
    }
}

template <int D, int NCT, int DT>
static hipError_t at_launch(const KvLayer &c, const KvView &q, const KvView &out, const KvAttn &a, void *ws, hipStream_t s)
{
    size_t bytes;
    const AtWork w = at_work<NCT>(ws, c, D, a.group, bytes);
    // kAtTarget pieces and one more for each item at most
    const unsigned blocks = (unsigned)(kAtTarget<NCT> + at_items(NCT, c, a.group));
    hipLaunchKernelGGL((k_kv_attention<D, NCT, DT>), dim3(blocks), dim3(kAtThreads), 0, s, c, q, out, a, w);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || w.most_cols == 0u) return e;      // (no row is longer than a piece)
    hipLaunchKernelGGL((k_kv_join<D, NCT, DT>), dim3(w.most_cols < 2048u ? w.most_cols : 2048u), dim3(kAtThreads), 0, s, out, c.kv_heads * a.group, w);
    return hipGetLastError();
}

// Columns that a wave takes, 16 NCT: 16 where rows bring no more than that on average (single tokens), else 32: a word of codes, once
// taken apart, serves twice as many.
inline bool at_narrow(uint32_t group, uint32_t rows, uint64_t tokens) { return tokens * group <= 16ull * rows; }

template <int D> hipError_t at_dim(const KvLayer &c, int dtype, const KvView &q, const KvView &out, const KvAttn &a, void *ws, hipStream_t s)
{
    if (at_narrow(a.group, c.rows, c.tokens))
        return dtype == QP_F32 ? at_launch<D, 1, QP_F32>(c, q, out, a, ws, s) : at_launch<D, 1, QP_BF16>(c, q, out, a, ws, s);
    return dtype == QP_F32 ? at_launch<D, 2, QP_F32>(c, q, out, a, ws, s) : at_launch<D, 2, QP_BF16>(c, q, out, a, ws, s);
}
#define QP_KV_ATTENTION_DIM(D) \
    template hipError_t at_dim<D>(const KvLayer &, int, const KvView &, const KvView &, const KvAttn &, void *, hipStream_t)

}  // namespace qp
