// Rows of the 4-bit key/value cache: quantize into pages, and back.
//
// A wave takes the eight tokens whose value codes share words (tokens 8 g .. 8 g + 7 of a row, or those of them that the call
// brings) of one head: lane 8 j + p has token j, elements 8 (p + 8 i) .. + 7 for i = 0, 1, ..., so eight lanes read 128
// (bf16) or 256 (fp32) consecutive bytes of a token.  A lane's eight codes are one word of the key codes as they are;
// for the values an 8 x 8 transpose of nibbles across the eight lanes with the same p (three exchanges) turns "eight
// elements of token j" into "element j of eight tokens".  Words that hold other tokens too are read and merged; no other
// wave of the call writes them, because all of the call's tokens of a word are this wave's.
// Bound by HBM: (2 or 4) bytes in and 1/2 + 8/head_dim out for each element, or the reverse.  Measured: 4 rows of up to 32768 tokens read
// back to bf16 (8 heads of 128) in 111 us, 4.6 TB/s, a large copy's rate; 5 prompts of 1777 tokens in fp32 (12 heads of 64) written in
// 17.2 us and read in 13.7; one token for each of 64 rows 5.9 us either way, which is the launch and a chain of dependent
// loads: two rounds of the search for the row (of 65 entries), its range and length, its page, then the token's elements and the word that
// they are merged into; reading back, the grid and codes.
#include "qp_kv.hpp"

namespace qp {

constexpr int kKvThreads = 256;

// ---- which row a token belongs to: the last r with begin[r] <= t, found 64 entries at a time -----------------------------
__device__ __forceinline__ int32_t kv_find_row(const KvLayer &c, int32_t t)
{
    const uint32_t lane = threadIdx.x % kWave;
    uint32_t lo = 0, n = c.rows + 1u;
    while (true) {
        const uint32_t step = (n + kWave - 1u) / kWave;
        const uint32_t at = lane * step;
        const bool under = at < n && c.begin[lo + at] <= t;
        const uint32_t below = (uint32_t)__popcll(__ballot(under));   // (entries ascend, so these are the first ones)
        if (below == 0u) return -1;
        lo += (below - 1u) * step;
        n = min(step, c.rows + 1u - lo);
        if (step == 1u) break;
    }
    return lo < c.rows ? (int32_t)lo : -1;
}

// nibble i of lane j's word <-> nibble j of lane i's, among the lanes with the same lane % 8
__device__ __forceinline__ uint32_t kv_transpose(uint32_t w, uint32_t j)
{
    uint32_t o = __shfl_xor(w, 32, kWave);
    w = j & 4u ? (w & 0xffff0000u) | (o >> 16) : (w & 0x0000ffffu) | (o << 16);
    o = __shfl_xor(w, 16, kWave);
    w = j & 2u ? (w & 0xff00ff00u) | ((o >> 8) & 0x00ff00ffu) : (w & 0x00ff00ffu) | ((o << 8) & 0xff00ff00u);
    o = __shfl_xor(w, 8, kWave);
    w = j & 1u ? (w & 0xf0f0f0f0u) | ((o >> 4) & 0x0f0f0f0fu) : (w & 0x0f0f0f0fu) | ((o << 4) & 0xf0f0f0f0u);
    return w;
}

template <int DT> __device__ __forceinline__ void kv_load8(const unsigned char *p, uint32_t unit, float (&f)[8])
{
    if constexpr (DT == QP_F32) {
        float a[4], b[4];
        load16_stream<DT>(p, 2u * unit, a);
        load16_stream<DT>(p, 2u * unit + 1u, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = a[i];
            f[4 + i] = b[i];
        }
    } else {
        load16_stream<DT>(p, unit, f);
    }
}

// fp32 to bf16, half to even; NaN stays NaN
__device__ __forceinline__ uint32_t kv_bf16(float f)
{
    const uint32_t u = __float_as_uint(f);
    return (u & 0x7fffffffu) > 0x7f800000u ? (u >> 16) | 0x40u : (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

template <int DT> __device__ __forceinline__ void kv_store8(unsigned char *p, uint32_t unit, const float (&f)[8])
{
    if constexpr (DT == QP_F32) {
        const f32x4 a = {f[0], f[1], f[2], f[3]}, b = {f[4], f[5], f[6], f[7]};
        __builtin_nontemporal_store(a, reinterpret_cast<f32x4 *>(p) + 2u * unit);
        __builtin_nontemporal_store(b, reinterpret_cast<f32x4 *>(p) + 2u * unit + 1u);
    } else {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = kv_bf16(f[2 * i]) | (kv_bf16(f[2 * i + 1]) << 16);
        __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(p) + unit);
    }
}

// The tokens of a call that one step of a wave takes: token t of the call is the first of them.
struct KvOctet {
    uint32_t slot;           // of the first token's page
    uint32_t tg;             // the page's group of eight
    uint32_t j0, count;      // tokens j0 .. j0 + count - 1 of the group
    int32_t next;            // the call's token behind them
    bool starts;             // the first of the call's tokens in that group
};
// A walk over the call's tokens [t, end): the row that the last one was in is kept, and so is the page.
struct KvWalk {
    KvRow row;
    int32_t r, at;           // the row, or -1; the position of its first token
    uint32_t slot;
    int32_t page;
    __device__ __forceinline__ KvWalk() : row{0, 0, 0}, r(-1), at(0), slot(0xffffffffu), page(-1) {}
    // From token t on: the tokens of t's row that share its group.  `first(r, row)`: the position of a row's first token.  False: token t has
    // no place (r < 0: it is no row's).
    template <typename First> __device__ __forceinline__ bool octet(const KvLayer &c, int32_t t, const First &first, KvOctet &o)
    {
        o.next = t + 1;
        if (r < 0 || t < row.begin || t >= row.begin + row.count) {
            r = __builtin_amdgcn_readfirstlane(kv_find_row(c, t));
            slot = 0xffffffffu;
            if (r < 0) return false;
            row = kv_row(c, (uint32_t)r);
            at = first((uint32_t)r, row);
            if (t < row.begin || t >= row.begin + row.count) {       // token_begin does not ascend
                r = -1;
                return false;
            }
        }
        const int64_t pos = (int64_t)at + (t - row.begin);
        if (pos < 0 || pos >= (int64_t)(c.pages_per_row << c.page_shift)) return false;
        o.j0 = (uint32_t)pos & 7u;
        o.count = min(8u - o.j0, (uint32_t)(row.begin + row.count - t));
        o.next = t + (int32_t)o.count;
        o.slot = (uint32_t)pos >> c.page_shift;
        o.tg = ((uint32_t)pos & ((1u << c.page_shift) - 1u)) >> 3;
        o.starts = o.j0 == 0u || t == row.begin;         // (a token ahead of the row's start has no place, and the next one is the group's first)
        return true;
    }
    __device__ __forceinline__ int32_t page_of(const KvLayer &c, const KvOctet &o)
    {
        if (o.slot != slot) {
            slot = o.slot;
            page = kv_page(c, (uint32_t)r, slot);
        }
        return page;
    }
};

// ---- quantize ----------------------------------------------------------------------------------------------------------
struct KvGrid {
    float lo, scale, inv;
};
template <int UNITS> __device__ __forceinline__ KvGrid kv_grid(const float (&x)[UNITS][8], const bool (&has)[UNITS])
{
    float mn = INFINITY, mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool fine = has[u] && (__float_as_uint(x[u][e]) & 0x7f800000u) != 0x7f800000u;
            mn = fminf(mn, fine ? x[u][e] : INFINITY);
            mx = fmaxf(mx, fine ? x[u][e] : -INFINITY);
        }
    // the eight lanes of a token are neighbours
    mn = fminf(mn, dpp_f32<kDppQuadSwap1>(mn));
    mx = fmaxf(mx, dpp_f32<kDppQuadSwap1>(mx));
    mn = fminf(mn, dpp_f32<kDppQuadSwap2>(mn));
    mx = fmaxf(mx, dpp_f32<kDppQuadSwap2>(mx));
    mn = fminf(mn, dpp_f32<kDppHalfMirror>(mn));
    mx = fmaxf(mx, dpp_f32<kDppHalfMirror>(mx));
    KvGrid g;
    const bool none = mn > mx;
    g.lo = none ? 0.0f : fminf(fmaxf(mn, -0x1p126f), 0x1p126f);
    const float hi = none ? 0.0f : fminf(fmaxf(mx, -0x1p126f), 0x1p126f);
    g.scale = (hi - g.lo) / 15.0f;
    if (!(g.scale >= 0x1p-120f)) g.scale = 0.0f;
    g.inv = g.scale > 0.0f ? 1.0f / g.scale : 0.0f;
    return g;
}
__device__ __forceinline__ uint32_t kv_codes(const float (&x)[8], const KvGrid &g)
{
    uint32_t w = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float c = fminf(fmaxf(rintf((x[e] - g.lo) * g.inv), 0.0f), 15.0f);   // (fmaxf first: NaN -> 0)
        w |= (uint32_t)c << (4 * e);
    }
    return w;
}

// `span`: tokens of the call that a wave looks through for octets that begin there
template <int D, int DT>
__global__ __launch_bounds__(kKvThreads) void k_kv_append(KvLayer c, KvView k, KvView v, uint32_t span, uint32_t block0)
{
    constexpr int W = D / kKvCodes;              // words of a token
    constexpr int UNITS = (W + 7) / 8;           // words of a lane
    const uint32_t lane = threadIdx.x % kWave, j = lane / 8u, p = lane % 8u;
    const uint64_t wave = ((uint64_t)block0 + blockIdx.x) * (kKvThreads / kWave) + threadIdx.x / kWave;
    const uint32_t head = (uint32_t)(wave % c.kv_heads);
    const uint64_t t0 = wave / c.kv_heads * span;
    if (t0 >= c.tokens) return;
    const int32_t end = (int32_t)min(t0 + span, (uint64_t)c.tokens);
    const auto first = [](uint32_t, const KvRow &row) { return row.length - row.count; };
    KvWalk walk;
    for (int32_t t = (int32_t)t0; t < end;) {
        KvOctet o;
        const bool good = walk.octet(c, t, first, o);
        const int32_t here = t;
        t = o.next;
        if (!good || !o.starts) continue;        // an octet is taken where it begins
        const int32_t page = walk.page_of(c, o);
        if (page < 0) continue;
        unsigned char *slab = kv_slab(c, page, head);
        const uint32_t pt = 1u << c.page_shift;
        uint32_t *kcodes = reinterpret_cast<uint32_t *>(slab), *vcodes = kcodes + (size_t)pt * W;
        float *grids = reinterpret_cast<float *>(vcodes + (size_t)pt * W);
        const bool mine = j >= o.j0 && j < o.j0 + o.count;
        const uint64_t tok = mine ? (uint64_t)here + (j - o.j0) : (uint64_t)here;
        const unsigned char *kp = k.data + tok * k.token_stride + head * k.head_stride;
        const unsigned char *vp = v.data + tok * v.token_stride + head * v.head_stride;
        float x[UNITS][8], y[UNITS][8];
        bool has[UNITS];
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            has[u] = mine && p + 8u * u < (uint32_t)W;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] = y[u][e] = 0.0f;
            if (has[u]) {
                kv_load8<DT>(kp, p + 8u * u, x[u]);
                kv_load8<DT>(vp, p + 8u * u, y[u]);
            }
        }
        const KvGrid gk = kv_grid(x, has), gv = kv_grid(y, has);
        const uint32_t slot = o.tg * 8u + j;
        const uint32_t all = o.count == 8u ? 0xffffffffu : ((1u << (4u * o.count)) - 1u) << (4u * o.j0);   // the tokens' nibbles
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if (has[u]) kcodes[(size_t)slot * W + p + 8u * u] = kv_codes(x[u], gk);
            const uint32_t word = kv_transpose(has[u] ? kv_codes(y[u], gv) : 0u, j);
            if (p + 8u * u < (uint32_t)W) {
                uint32_t *dst = vcodes + (size_t)o.tg * D + 8u * (p + 8u * u) + j;
                *dst = all == 0xffffffffu ? word : (*dst & ~all) | (word & all);
            }
        }
        if (mine && p == 0u) {
            reinterpret_cast<float2 *>(grids)[slot] = make_float2(gk.lo, gk.scale);
            reinterpret_cast<float2 *>(grids)[pt + slot] = make_float2(gv.lo, gv.scale);
        }
    }
}

// ---- and back ------------------------------------------------------------------------------------------------------------
template <int D, int DT>
__global__ __launch_bounds__(kKvThreads) void k_kv_read(KvLayer c, const int32_t *__restrict__ firsts, KvView k, KvView v, uint32_t span, uint32_t block0)
{
    constexpr int W = D / kKvCodes;
    constexpr int UNITS = (W + 7) / 8;
    const uint32_t lane = threadIdx.x % kWave, j = lane / 8u, p = lane % 8u;
    const uint64_t wave = ((uint64_t)block0 + blockIdx.x) * (kKvThreads / kWave) + threadIdx.x / kWave;
    const uint32_t head = (uint32_t)(wave % c.kv_heads);
    const uint64_t t0 = wave / c.kv_heads * span;
    if (t0 >= c.tokens) return;
    const int32_t end = (int32_t)min(t0 + span, (uint64_t)c.tokens);
    const auto first = [firsts](uint32_t r, const KvRow &) { return firsts ? firsts[r] : 0; };
    KvWalk walk;
    for (int32_t t = (int32_t)t0; t < end;) {
        KvOctet o;
        const bool good = walk.octet(c, t, first, o);
        const int32_t here = t;
        t = o.next;
        if (!good) {
            if (walk.r < 0) continue;        // the token is no row's
            o.j0 = 0u;                       // a place outside the table: this token alone, zeros
            o.count = 1u;
        } else if (!o.starts) {
            continue;
        }
        const int32_t page = good ? walk.page_of(c, o) : -1;
        const bool mine = j >= o.j0 && j < o.j0 + o.count;
        const uint64_t tok = mine ? (uint64_t)here + (j - o.j0) : (uint64_t)here;
        unsigned char *kp = k.data + tok * k.token_stride + head * k.head_stride;
        unsigned char *vp = v.data + tok * v.token_stride + head * v.head_stride;
        const float zero[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        const int64_t pos = (int64_t)walk.at + ((int64_t)here - walk.row.begin) + ((int64_t)j - o.j0);
        const bool there = page >= 0 && mine && pos < (int64_t)walk.row.length;
        if (page < 0) {
#pragma unroll
            for (int u = 0; u < UNITS; ++u)
                if (mine && p + 8u * u < (uint32_t)W) {
                    kv_store8<DT>(kp, p + 8u * u, zero);
                    kv_store8<DT>(vp, p + 8u * u, zero);
                }
            continue;
        }
        const unsigned char *slab = kv_slab(c, page, head);
        const uint32_t pt = 1u << c.page_shift;
        const uint32_t *kcodes = reinterpret_cast<const uint32_t *>(slab), *vcodes = kcodes + (size_t)pt * W;
        const float2 *grids = reinterpret_cast<const float2 *>(vcodes + (size_t)pt * W);
        const uint32_t slot = o.tg * 8u + j;
        const float2 gk = grids[slot], gv = grids[pt + slot];
        uint32_t a[UNITS], b[UNITS];
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            a[u] = b[u] = 0u;
            if (p + 8u * u < (uint32_t)W) {
                a[u] = kcodes[(size_t)slot * W + p + 8u * u];
                b[u] = vcodes[(size_t)o.tg * D + 8u * (p + 8u * u) + j];
            }
        }
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const uint32_t wv = kv_transpose(b[u], j);
            if (!(mine && p + 8u * u < (uint32_t)W)) continue;
            float x[8], y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = there ? fmaf((float)((a[u] >> (4 * e)) & 15u), gk.y, gk.x) : 0.0f;
                y[e] = there ? fmaf((float)((wv >> (4 * e)) & 15u), gv.y, gv.x) : 0.0f;
            }
            kv_store8<DT>(kp, p + 8u * u, x);
            kv_store8<DT>(vp, p + 8u * u, y);
        }
    }
}

// A wave looks through one token where rows bring fewer than eight on average: with single tokens every octet is a token of its own, and
// eight of them one after the other would take eight times the latency.  Else through eight, an octet's worth, as long as that fills the
// chip, and through 32 where that still does: the row is found once for four octets.
#ifndef QP_KV_SPAN_FILL
#define QP_KV_SPAN_FILL (256u * 32u)
#endif
static uint32_t kv_span(const KvLayer &c)
{
    if (c.tokens < 8u * (uint64_t)c.rows) return 1u;
    return (uint64_t)c.tokens * c.kv_heads >= 32ull * QP_KV_SPAN_FILL ? 32u : 8u;
}
static uint64_t kv_rows_blocks(const KvLayer &c, uint32_t span)
{
    const uint64_t waves = ((uint64_t)c.tokens + span - 1u) / span * c.kv_heads;
    return (waves + kKvThreads / kWave - 1u) / (kKvThreads / kWave);
}

template <int D, int DT> static hipError_t append_as(const KvLayer &c, const KvView &k, const KvView &v, hipStream_t s)
{
    const uint32_t span = kv_span(c);
    return kv_launches(kv_rows_blocks(c, span), [&](dim3 grid, uint32_t block0) {
        hipLaunchKernelGGL((k_kv_append<D, DT>), grid, dim3(kKvThreads), 0, s, c, k, v, span, block0);
    });
}
template <int D> static hipError_t append_dim(const KvLayer &c, int dtype, const KvView &k, const KvView &v, hipStream_t s)
{
    return dtype == QP_F32 ? append_as<D, QP_F32>(c, k, v, s) : append_as<D, QP_BF16>(c, k, v, s);
}
template <int D, int DT> static hipError_t read_as(const KvLayer &c, const int32_t *first, const KvView &k, const KvView &v, hipStream_t s)
{
    const uint32_t span = kv_span(c);
    return kv_launches(kv_rows_blocks(c, span), [&](dim3 grid, uint32_t block0) {
        hipLaunchKernelGGL((k_kv_read<D, DT>), grid, dim3(kKvThreads), 0, s, c, first, k, v, span, block0);
    });
}
template <int D>
static hipError_t read_dim(const KvLayer &c, int dtype, const int32_t *first, const KvView &k, const KvView &v, hipStream_t s)
{
    return dtype == QP_F32 ? read_as<D, QP_F32>(c, first, k, v, s) : read_as<D, QP_BF16>(c, first, k, v, s);
}

hipError_t launch_kv_append(const KvLayer &c, uint32_t dim, int dtype, const KvView &k, const KvView &v, hipStream_t s)
{
    switch (dim) {
        case 64: return append_dim<64>(c, dtype, k, v, s);
        case 80: return append_dim<80>(c, dtype, k, v, s);
        case 96: return append_dim<96>(c, dtype, k, v, s);
        case 128: return append_dim<128>(c, dtype, k, v, s);
        case 256: return append_dim<256>(c, dtype, k, v, s);
        default: return hipErrorInvalidValue;
    }
}

hipError_t launch_kv_read(const KvLayer &c, uint32_t dim, int dtype, const int32_t *first, const KvView &k, const KvView &v, hipStream_t s)
{
    switch (dim) {
        case 64: return read_dim<64>(c, dtype, first, k, v, s);
        case 80: return read_dim<80>(c, dtype, first, k, v, s);
        case 96: return read_dim<96>(c, dtype, first, k, v, s);
        case 128: return read_dim<128>(c, dtype, first, k, v, s);
        case 256: return read_dim<256>(c, dtype, first, k, v, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace qp
