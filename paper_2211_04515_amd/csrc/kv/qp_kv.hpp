// What the kernels of the 4-bit key/value cache share: the layout of a page, the rows of a call, launch declarations.
// The layout itself is described in quantpipe.h.
#pragma once

#include "../qp_common.hpp"

namespace qp {

constexpr uint32_t kKvMaxPages = 1u << 24;
constexpr uint32_t kKvMaxRows = 65536;
constexpr int kKvCodes = 8;                     // codes in a word

// One layer of a cache and the rows that live in it, as the kernels take them.
struct KvLayer {
    unsigned char *pages;                       // of the layer
    const int32_t *table, *lengths, *begin;     // begin: token_begin_dev
    uint64_t page_bytes;
    uint32_t slab_bytes;                        // of one head of a page
    uint32_t n_pages, rows, pages_per_row;
    uint32_t kv_heads, tokens;
    uint32_t page_shift;                        // log2(page_tokens)
};

struct KvView {
    unsigned char *data;
    uint64_t token_stride, head_stride;         // in bytes
};

// A row of a call: which of the call's tokens are its own, and how long it is.
struct KvRow {
    int32_t begin, count, length;
};
__device__ __forceinline__ KvRow kv_row(const KvLayer &c, uint32_t r)
{
    const int32_t most = (int32_t)c.tokens;
    const int32_t b = min(max(c.begin[r], 0), most), e = min(max(c.begin[r + 1], 0), most);
    const int32_t cap = (int32_t)(c.pages_per_row << c.page_shift);
    return KvRow{b, max(e - b, 0), min(max(c.lengths[r], 0), cap)};
}

// The page of slot `slot` of row r, or -1.
__device__ __forceinline__ int32_t kv_page(const KvLayer &c, uint32_t r, uint32_t slot)
{
    if (slot >= c.pages_per_row) return -1;
    const int32_t p = c.table[(uint64_t)r * c.pages_per_row + slot];
    return (uint32_t)p < c.n_pages ? p : -1;
}
__device__ __forceinline__ unsigned char *kv_slab(const KvLayer &c, int32_t page, uint32_t head)
{
    return c.pages + (uint64_t)(uint32_t)page * c.page_bytes + (uint64_t)head * c.slab_bytes;
}

__device__ __forceinline__ float kv_xor_f32(float v, int mask) { return __uint_as_float(__shfl_xor(__float_as_uint(v), mask, kWave)); }

// The pool record's parts.
struct KvPool {
    int32_t *header, *refs, *count, *last, *list, *pairs;   // [16], then [n_pages] each, pairs [n_pages][2]
};
__host__ __device__ inline KvPool kv_pool(void *pool, uint32_t n_pages)
{
    int32_t *p = static_cast<int32_t *>(pool);
    int32_t *r = p + QP_KV_POOL_HEADER;
    return KvPool{p, r, r + n_pages, r + 2 * (size_t)n_pages, r + 3 * (size_t)n_pages, r + 4 * (size_t)n_pages};
}
enum : uint32_t { kKvShort = 0, kKvOutgrown = 1, kKvRefused = 2, kKvLive = 3, kKvMoves = 4 };   // words of the header

// Inclusive prefix sums over a wave's lanes: within rows of 16 by shifts that bring in zeros, then what the rows before come to.
__device__ __forceinline__ uint32_t kv_wave_scan(uint32_t v)
{
    int x = (int)v;
    x += dpp_i32<0x111>(x);                     // row_shr:1, 2, 4, 8
    x += dpp_i32<0x112>(x);
    x += dpp_i32<0x114>(x);
    x += dpp_i32<0x118>(x);
    const uint32_t row = threadIdx.x % kWave / 16u;
    const int a = __builtin_amdgcn_readlane(x, 15), b = a + __builtin_amdgcn_readlane(x, 31), c = b + __builtin_amdgcn_readlane(x, 47);
    return (uint32_t)(x + (row == 0u ? 0 : row == 1u ? a : row == 2u ? b : c));
}

// A launch has fewer than 2^32 threads; what has more blocks (65536 rows of 1024 heads each) goes in several, and a block's number is blockIdx.x and
// what its launch is told to add.
#ifndef QP_KV_GRID
#define QP_KV_GRID (1u << 23)
#endif
template <typename Launch> hipError_t kv_launches(uint64_t blocks, const Launch &launch)
{
    hipError_t e = hipSuccess;
    for (uint64_t b = 0; b < blocks && e == hipSuccess; b += QP_KV_GRID) {
        launch(dim3((unsigned)(blocks - b < QP_KV_GRID ? blocks - b : QP_KV_GRID)), (uint32_t)b);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_kv_append(const KvLayer &c, uint32_t dim, int dtype, const KvView &k, const KvView &v, hipStream_t s);
hipError_t launch_kv_read(const KvLayer &c, uint32_t dim, int dtype, const int32_t *first, const KvView &k, const KvView &v,
                          hipStream_t s);

struct KvPages {                                // all layers of a cache, for calls that move pages
    unsigned char *pages;
    uint64_t page_bytes, layer_bytes;
    uint32_t layers, n_pages, page_shift;
};
hipError_t launch_kv_pool_init(uint32_t n_pages, void *pool, hipStream_t s);
hipError_t launch_kv_reserve(const KvPages &c, const qp_kv_rows_t &rows, const int32_t *want, void *pool, hipStream_t s);
hipError_t launch_kv_fork(const KvPages &c, const qp_kv_rows_t &rows, const int32_t *parent, void *pool, hipStream_t s);
hipError_t launch_kv_free(const KvPages &c, const qp_kv_rows_t &rows, const int32_t *keep, void *pool, hipStream_t s);
hipError_t launch_kv_compact(const KvPages &c, const qp_kv_rows_t &rows, void *pool, hipStream_t s);

struct KvAttn {
    float scale;
    uint32_t group;                             // query heads of a key head
    uint32_t causal, window;
};

}  // namespace qp
