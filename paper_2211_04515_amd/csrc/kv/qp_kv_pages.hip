// Pages of the 4-bit key/value cache: handed out, shared, given up, moved together.
//
// The books are int32 arrays (page tables, lengths, reference counts), small next to the pages: a serving step's worth is
// tens of kilobytes.  What they cost is latency, so each call is one kernel over them and, where pages move, one over the pages
// that takes its list from the first: nothing is decided on the host.  Handing out pages and compacting need an order over the whole
// pool (the lowest free page first), which one block of 1024 lanes keeps with prefix sums: it reads 32 KB of reference counts at a
// time.  Sharing and giving up only add to counts, whose order does not matter.
// The copy kernel is bound by HBM: 16-byte loads and stores, all layers' pages of a list spread over the whole chip.  Measured: 117 us where
// 16 layers' pages of 48 requests move together (266 of 1.2 MB on average), 126 with the books before it, 5.4 TB/s read and written (a plain copy of
// 4 GiB: 4.7).
// A beam step (8 requests of 5 beams: free, fork, reserve, 32 pages of 16 layers copied) is 29 us: 16.4 of copying (4.6 TB/s), 7.8 to reserve,
// 3.5 to fork, 2.8 to free.
#include "qp_kv.hpp"

namespace qp {

constexpr int kKvPlan = 1024;                 // lanes of the one block that plans
constexpr int kKvScan = 8;                    // reference counts that a lane takes at a time
constexpr uint32_t kKvCopyThreads = 256, kKvCopyUnroll = 4;
constexpr uint32_t kKvCopyTile = kKvCopyThreads * kKvCopyUnroll * 16u;   // bytes of a block's step
#ifndef QP_KV_COPY_BLOCKS
#define QP_KV_COPY_BLOCKS 2048
#endif

// tokens -> pages begun
__device__ __forceinline__ uint32_t kv_pages_of(int64_t tokens, uint32_t shift) { return (uint32_t)((tokens + (1 << shift) - 1) >> shift); }
__device__ __forceinline__ int64_t kv_length(const qp_kv_rows_t &rows, uint32_t r, uint32_t shift)
{
    const int64_t cap = (int64_t)rows.pages_per_row << shift;
    return min(max((int64_t)rows.lengths_dev[r], (int64_t)0), cap);
}

// Inclusive prefix sums of N numbers over the block's 1024 lanes, and their totals.  `part` holds each wave's.
template <int N> __device__ __forceinline__ void wave_scan(uint32_t (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = kv_wave_scan(x[i]);
}
template <int N> __device__ __forceinline__ void block_scan(uint32_t (&x)[N], uint32_t (*part)[kKvPlan / kWave], uint32_t (&total)[N])
{
    const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    wave_scan(x);
    __syncthreads();                          // (the sums of an earlier scan have been read)
    if (lane == kWave - 1u)
#pragma unroll
        for (int i = 0; i < N; ++i) part[i][wave] = x[i];
    __syncthreads();
    uint32_t sums[N];                         // (every wave adds the 16 up for itself)
#pragma unroll
    for (int i = 0; i < N; ++i) sums[i] = lane < (uint32_t)(kKvPlan / kWave) ? part[i][lane] : 0u;
    wave_scan(sums);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        total[i] = (uint32_t)__builtin_amdgcn_readlane((int)sums[i], kKvPlan / kWave - 1);
        const uint32_t before = (uint32_t)__builtin_amdgcn_readlane((int)sums[i], (int)(wave ? wave - 1u : 0u));
        x[i] += wave ? before : 0u;
    }
}
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t (*part)[kKvPlan / kWave], uint32_t &total)
{
    uint32_t x[1] = {v}, t[1];
    block_scan(x, part, t);
    total = t[0];
    return x[0];
}

__global__ __launch_bounds__(256) void k_kv_pool_init(int32_t *pool, uint32_t words)
{
    for (uint32_t i = blockIdx.x * 256u + threadIdx.x; i < words; i += gridDim.x * 256u) pool[i] = 0;
}

// ---- pages that move: pairs {from, to}, in every layer ---------------------------------------------------------------------
// (`went`: what a compaction has noted at the pages that move, cleared here for the next call; zero already after a reservation.)
__global__ __launch_bounds__(kKvCopyThreads) void k_kv_move(KvPages c, const int32_t *__restrict__ header, const int32_t *__restrict__ pairs, int32_t *went)
{
    const uint32_t count = (uint32_t)header[kKvMoves];
    for (uint32_t i = blockIdx.x * kKvCopyThreads + threadIdx.x; i < count; i += gridDim.x * kKvCopyThreads) went[pairs[2u * i]] = 0;
    const uint32_t tiles = (uint32_t)((c.page_bytes + kKvCopyTile - 1u) / kKvCopyTile);      // of a page
    const uint64_t work = (uint64_t)count * c.layers * tiles;
    for (uint64_t i = blockIdx.x; i < work; i += gridDim.x) {
        const uint32_t tile = (uint32_t)(i % tiles);
        const uint64_t rest = i / tiles;
        const uint32_t pair = (uint32_t)(rest % count), layer = (uint32_t)(rest / count);
        const unsigned char *from = c.pages + layer * c.layer_bytes + (uint64_t)(uint32_t)pairs[2u * pair] * c.page_bytes;
        unsigned char *to = c.pages + layer * c.layer_bytes + (uint64_t)(uint32_t)pairs[2u * pair + 1u] * c.page_bytes;
        const uint64_t at = (uint64_t)tile * kKvCopyTile + threadIdx.x * 16u;
        u32x4 w[kKvCopyUnroll];
#pragma unroll
        for (uint32_t u = 0; u < kKvCopyUnroll; ++u) {
            const uint64_t o = at + u * kKvCopyThreads * 16u;
            if (o < c.page_bytes) w[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + o));
        }
#pragma unroll
        for (uint32_t u = 0; u < kKvCopyUnroll; ++u) {
            const uint64_t o = at + u * kKvCopyThreads * 16u;
            if (o < c.page_bytes) __builtin_nontemporal_store(w[u], reinterpret_cast<u32x4 *>(to + o));
        }
    }
}

// ---- reserve -----------------------------------------------------------------------------------------------------------
// A row of the call: its length, what it wants, and the page that it writes next if others hold that too (else -1).
struct KvWish {
    int64_t length;
    int32_t want, shared;
};
__device__ __forceinline__ KvWish kv_wish(const qp_kv_rows_t &rows, const KvPages &c, const KvPool &p, const int32_t *want, uint32_t r)
{
    KvWish o{kv_length(rows, r, c.page_shift), want[r], -1};
    if (o.want <= 0 || (o.length & ((1 << c.page_shift) - 1)) == 0) return o;
    const int32_t page = rows.table_dev[(uint64_t)r * rows.pages_per_row + (uint64_t)(o.length >> c.page_shift)];
    if ((uint32_t)page < c.n_pages && p.refs[page] > 1) o.shared = page;
    return o;
}
// What it asks for: `fresh` pages for the slots from `slot` on, the first of them in the place of the shared page if `copy`.
struct KvAsk {
    uint32_t slot, fresh;
    bool copy;
};
__device__ __forceinline__ KvAsk kv_ask(const KvPages &c, const KvPool &p, uint32_t r, const KvWish &w)
{
    KvAsk a;
    // If every holder of the page asks, the last row among them keeps it: what serving them in turn comes to.
    // (count and last are this kernel's atomics: read where those are, not through a cache line fetched before them)
    a.copy = w.shared >= 0 && !(ld_dev(reinterpret_cast<uint32_t *>(p.count + w.shared)) == (uint32_t)p.refs[w.shared] &&
                                ld_dev(reinterpret_cast<uint32_t *>(p.last + w.shared)) == r + 1u);
    a.fresh = w.want > 0 ? kv_pages_of(w.length + w.want, c.page_shift) - kv_pages_of(w.length, c.page_shift) + (a.copy ? 1u : 0u) : 0u;
    a.slot = a.copy ? (uint32_t)(w.length >> c.page_shift) : kv_pages_of(w.length, c.page_shift);
    return a;
}

// Latency is all that it costs: a lane keeps its first row's wish and ask in registers (most calls have no more rows than lanes), so
// that what it reads is read once: 15.5 -> 9.8 us for 40 rows; the list of new pages in LDS 9.1, sums by lane shifts instead of LDS 7.8.
__global__ __launch_bounds__(kKvPlan) void k_kv_reserve(KvPages c, qp_kv_rows_t rows, const int32_t *__restrict__ want, void *pool)
{
    __shared__ uint32_t part[3][kKvPlan / kWave];
    __shared__ uint32_t ask_fresh[kKvPlan], ask_slot[kKvPlan], ask_base[kKvPlan];
    __shared__ int32_t near_list[kKvPlan];    // the first of the new pages; what does not fit goes to the pool's room
    const uint32_t tid = threadIdx.x;
    const KvPool p = kv_pool(pool, c.n_pages);
    const KvWish nothing{0, 0, -1};
    const KvWish first = tid < rows.rows ? kv_wish(rows, c, p, want, tid) : nothing;
    const auto wish = [&](uint32_t r) { return r == tid ? first : kv_wish(rows, c, p, want, r); };
    // the free pages among the first, on their way while the rows are looked at
    uint32_t bits0 = 0;
#pragma unroll
    for (uint32_t i = 0; i < (uint32_t)kKvScan; ++i) bits0 |= (tid * kKvScan + i < c.n_pages && p.refs[tid * kKvScan + i] == 0 ? 1u : 0u) << i;
    // how many of a shared page's holders write into it next, and the last of them
    for (uint32_t r = tid; r < rows.rows; r += kKvPlan) {
        const int32_t page = wish(r).shared;
        if (page >= 0) {
            atomicAdd(reinterpret_cast<uint32_t *>(p.count + page), 1u);
            atomicMax(reinterpret_cast<uint32_t *>(p.last + page), r + 1u);
        }
    }
    __syncthreads();
    const KvAsk none{0u, 0u, false};
    const KvAsk first_ask = tid < rows.rows ? kv_ask(c, p, tid, first) : none;
    const auto ask = [&](uint32_t r) { return r == tid ? first_ask : kv_ask(c, p, r, wish(r)); };
    const int64_t cap = (int64_t)rows.pages_per_row << c.page_shift;
    uint64_t need = 0;
    uint32_t over = 0;
    for (uint32_t r = tid; r < rows.rows; r += kKvPlan) {
        const KvWish w = wish(r);
        if (w.want > 0 && w.length + w.want > cap) ++over;
        else need += ask(r).fresh;
    }
    uint32_t counts[3] = {over, (uint32_t)need & 0xffffu, (uint32_t)(need >> 16)}, sums[3];
    block_scan(counts, part, sums);
    const uint32_t rows_over = sums[0], total = (uint32_t)min(((uint64_t)sums[2] << 16) + sums[1], (uint64_t)0x7fffffffu);
    // the free pages with the lowest indices, as many as are needed
    uint32_t found = 0;
    for (uint32_t p0 = 0; p0 < c.n_pages && found < total && rows_over == 0u; p0 += kKvPlan * kKvScan) {
        const uint32_t at = p0 + tid * kKvScan;
        uint32_t bits = bits0;
        if (p0 != 0u) {
            bits = 0;
#pragma unroll
            for (uint32_t i = 0; i < (uint32_t)kKvScan; ++i) bits |= (at + i < c.n_pages && p.refs[at + i] == 0 ? 1u : 0u) << i;
        }
        const uint32_t mine = (uint32_t)__popcll(bits);
        uint32_t sum = 0;
        uint32_t place = found + block_scan(mine, part, sum) - mine;
        for (uint32_t i = 0; i < (uint32_t)kKvScan; ++i)
            if ((bits >> i) & 1u) {
                if (place < min(total, (uint32_t)kKvPlan)) near_list[place] = (int32_t)(at + i);
                else if (place < total) p.list[place] = (int32_t)(at + i);
                ++place;
            }
        found += sum;
    }
    const bool done = rows_over == 0u && found >= total;
    const auto page_at = [&](uint32_t k) { return k < (uint32_t)kKvPlan ? near_list[k] : p.list[k]; };
    __syncthreads();                          // the list is whole
    uint32_t base = 0, moves = 0, first_moves = 0;
    for (uint32_t r0 = 0; r0 < rows.rows && done; r0 += kKvPlan) {
        const uint32_t r = r0 + tid;
        const bool is = r < rows.rows;
        const KvWish w = is ? wish(r) : nothing;
        const KvAsk a = is ? ask(r) : none;
        uint32_t at[2] = {a.fresh, a.copy ? 1u : 0u}, all[2];
        block_scan(at, part, all);
        const uint32_t mine = base + at[0] - a.fresh, move = moves + at[1] - (a.copy ? 1u : 0u);
        ask_fresh[tid] = a.fresh;
        ask_slot[tid] = a.slot;
        ask_base[tid] = mine;
        if (a.copy) {
            p.pairs[2u * move] = w.shared;
            p.pairs[2u * move + 1u] = page_at(mine);
        }
        __syncthreads();                      // every row of these has looked at the counts and the table
        if (is && w.want > 0) rows.lengths_dev[r] = (int32_t)(w.length + w.want);
        for (uint32_t k = tid / kWave; k < min((uint32_t)kKvPlan, rows.rows - r0); k += kKvPlan / kWave)   // a wave a row: its pages
            for (uint32_t i = tid % kWave; i < ask_fresh[k]; i += kWave)
                rows.table_dev[(uint64_t)(r0 + k) * rows.pages_per_row + ask_slot[k] + i] = page_at(ask_base[k] + i);
        base += all[0];
        moves += all[1];
        if (r0 == 0u) first_moves = moves;
        __syncthreads();
    }
    // the counts change once no row looks at them any more; the shared pages' books are cleared for the next call
    if (done) {
        for (uint32_t i = tid; i < total; i += kKvPlan) p.refs[page_at(i)] = 1;
        if (first_ask.copy) atomicAdd(reinterpret_cast<uint32_t *>(p.refs + first.shared), 0xffffffffu);
        for (uint32_t i = first_moves + tid; i < moves; i += kKvPlan) {          // (of rows behind the first 1024)
            const int32_t page = p.pairs[2u * i];
            atomicAdd(reinterpret_cast<uint32_t *>(p.refs + page), 0xffffffffu);
            p.count[page] = p.last[page] = 0;
        }
    }
    if (tid < rows.rows && first.shared >= 0) p.count[first.shared] = p.last[first.shared] = 0;
    for (uint32_t r = tid + kKvPlan; r < rows.rows; r += kKvPlan) {   // (a counted page that was not copied is still its row's next one)
        const int64_t len = kv_length(rows, r, c.page_shift) - (done && want[r] > 0 ? want[r] : 0);
        if (want[r] <= 0 || (len & ((1 << c.page_shift) - 1)) == 0) continue;
        const int32_t page = rows.table_dev[(uint64_t)r * rows.pages_per_row + (uint64_t)(len >> c.page_shift)];
        if ((uint32_t)page < c.n_pages) p.count[page] = p.last[page] = 0;
    }
    if (tid == 0u) {
        p.header[kKvShort] = (int32_t)(done || rows_over ? 0u : total - found);
        p.header[kKvOutgrown] = (int32_t)rows_over;
        p.header[kKvMoves] = (int32_t)moves;
    }
}

// ---- fork, free: a block for each row --------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_kv_fork(KvPages c, qp_kv_rows_t rows, const int32_t *__restrict__ parent, void *pool)
{
    const KvPool p = kv_pool(pool, c.n_pages);
    const uint32_t r = blockIdx.x;
    const int32_t from = parent[r];
    if (from < 0) return;
    const bool good = (uint32_t)from < rows.rows && (uint32_t)from != r && parent[(uint32_t)from < rows.rows ? from : 0] < 0 &&
                      rows.lengths_dev[r] <= 0;
    __syncthreads();                          // (every lane has seen the row's own length)
    if (!good) {
        if (threadIdx.x == 0u) atomicAdd(reinterpret_cast<uint32_t *>(p.header + kKvRefused), 1u);
        return;
    }
    const int64_t len = kv_length(rows, (uint32_t)from, c.page_shift);
    const uint32_t held = kv_pages_of(len, c.page_shift);
    for (uint32_t i = threadIdx.x; i < held; i += 256u) {
        const int32_t page = rows.table_dev[(uint64_t)from * rows.pages_per_row + i];
        rows.table_dev[(uint64_t)r * rows.pages_per_row + i] = page;
        if ((uint32_t)page < c.n_pages) atomicAdd(reinterpret_cast<uint32_t *>(p.refs + page), 1u);
    }
    if (threadIdx.x == 0u) rows.lengths_dev[r] = (int32_t)len;
}

__global__ __launch_bounds__(256) void k_kv_free(KvPages c, qp_kv_rows_t rows, const int32_t *__restrict__ keep, void *pool)
{
    const KvPool p = kv_pool(pool, c.n_pages);
    const uint32_t r = blockIdx.x;
    const int64_t len = kv_length(rows, r, c.page_shift);
    const int32_t k = keep[r];
    __syncthreads();                          // (every lane has seen the length)
    if (k < 0 || k >= len) return;
    const uint32_t from = kv_pages_of(k, c.page_shift), to = kv_pages_of(len, c.page_shift);
    for (uint32_t i = from + threadIdx.x; i < to; i += 256u) {
        int32_t *entry = rows.table_dev + (uint64_t)r * rows.pages_per_row + i;
        if ((uint32_t)*entry < c.n_pages) atomicAdd(reinterpret_cast<uint32_t *>(p.refs + *entry), 0xffffffffu);
        *entry = -1;
    }
    if (threadIdx.x == 0u) rows.lengths_dev[r] = k;
}

// ---- compact -----------------------------------------------------------------------------------------------------------
// Lists the moves: with L pages in use, the i-th free place below L takes the i-th page in use at or above L.  There are as many
// of the one as of the other.  `count` (all zero between calls) says where a moved page went, + 1.
__global__ __launch_bounds__(kKvPlan) void k_kv_compact(KvPages c, void *pool)
{
    __shared__ uint32_t part[3][kKvPlan / kWave];
    const uint32_t tid = threadIdx.x;
    const KvPool p = kv_pool(pool, c.n_pages);
    uint32_t live = 0, mine = 0;
    for (uint32_t p0 = 0; p0 < c.n_pages; p0 += kKvPlan * kKvScan) {
        const uint32_t at = p0 + tid * kKvScan;
#pragma unroll
        for (uint32_t i = 0; i < (uint32_t)kKvScan; ++i) mine += at + i < c.n_pages && p.refs[at + i] > 0 ? 1u : 0u;
    }
    block_scan(mine, part, live);
    uint32_t holes = 0, movers = 0;
    for (uint32_t p0 = 0; p0 < c.n_pages; p0 += kKvPlan * kKvScan) {
        const uint32_t at = p0 + tid * kKvScan;
        uint32_t bits = 0, below = 0, above = 0;
#pragma unroll
        for (uint32_t i = 0; i < (uint32_t)kKvScan; ++i) {
            if (at + i >= c.n_pages) break;
            const bool used = p.refs[at + i] > 0;
            const bool is = at + i < live ? !used : used;
            bits |= (is ? 1u : 0u) << i;
            below += is && at + i < live ? 1u : 0u;
            above += is && at + i >= live ? 1u : 0u;
        }
        uint32_t at2[2] = {below, above}, all[2];
        block_scan(at2, part, all);
        uint32_t hole = holes + at2[0] - below, mover = movers + at2[1] - above;
        for (uint32_t i = 0; i < (uint32_t)kKvScan; ++i)
            if ((bits >> i) & 1u) {
                if (at + i < live) p.pairs[2u * hole++ + 1u] = (int32_t)(at + i);
                else p.pairs[2u * mover++] = (int32_t)(at + i);
            }
        holes += all[0];
        movers += all[1];
    }
    __syncthreads();                          // the pairs are whole
    for (uint32_t i = tid; i < holes; i += kKvPlan) {
        const int32_t from = p.pairs[2u * i], to = p.pairs[2u * i + 1u];
        p.refs[to] = p.refs[from];
        p.refs[from] = 0;
        p.count[from] = to + 1;
    }
    if (tid == 0u) {
        p.header[kKvMoves] = (int32_t)holes;
        p.header[kKvLive] = (int32_t)live;
    }
}
__global__ __launch_bounds__(256) void k_kv_renumber(KvPages c, qp_kv_rows_t rows, void *pool)
{
    const KvPool p = kv_pool(pool, c.n_pages);
    const uint32_t r = blockIdx.x;
    const uint32_t held = kv_pages_of(kv_length(rows, r, c.page_shift), c.page_shift);
    for (uint32_t i = threadIdx.x; i < held; i += 256u) {
        int32_t *entry = rows.table_dev + (uint64_t)r * rows.pages_per_row + i;
        if ((uint32_t)*entry < c.n_pages && p.count[*entry] > 0) *entry = p.count[*entry] - 1;
    }
}
static dim3 blocks_for(uint64_t items, uint32_t per, uint32_t most)
{
    const uint64_t b = (items + per - 1u) / per;
    return dim3((unsigned)(b < 1u ? 1u : b < most ? b : most));
}
static dim3 move_blocks(const KvPages &c, uint64_t most_pairs)
{
    return blocks_for(most_pairs * c.layers * ((c.page_bytes + kKvCopyTile - 1u) / kKvCopyTile), 1u, QP_KV_COPY_BLOCKS);
}

hipError_t launch_kv_pool_init(uint32_t n_pages, void *pool, hipStream_t s)
{
    const uint32_t words = QP_KV_POOL_HEADER + 6u * n_pages;
    hipLaunchKernelGGL(k_kv_pool_init, blocks_for(words, 256u, 1024u), dim3(256), 0, s, static_cast<int32_t *>(pool), words);
    return hipGetLastError();
}

hipError_t launch_kv_reserve(const KvPages &c, const qp_kv_rows_t &rows, const int32_t *want, void *pool, hipStream_t s)
{
    const KvPool p = kv_pool(pool, c.n_pages);
    hipLaunchKernelGGL(k_kv_reserve, dim3(1), dim3(kKvPlan), 0, s, c, rows, want, pool);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_kv_move, move_blocks(c, rows.rows), dim3(kKvCopyThreads), 0, s, c, p.header, p.pairs, p.count);
    return hipGetLastError();
}

hipError_t launch_kv_fork(const KvPages &c, const qp_kv_rows_t &rows, const int32_t *parent, void *pool, hipStream_t s)
{
    hipLaunchKernelGGL(k_kv_fork, dim3(rows.rows), dim3(256), 0, s, c, rows, parent, pool);
    return hipGetLastError();
}

hipError_t launch_kv_free(const KvPages &c, const qp_kv_rows_t &rows, const int32_t *keep, void *pool, hipStream_t s)
{
    hipLaunchKernelGGL(k_kv_free, dim3(rows.rows), dim3(256), 0, s, c, rows, keep, pool);
    return hipGetLastError();
}

hipError_t launch_kv_compact(const KvPages &c, const qp_kv_rows_t &rows, void *pool, hipStream_t s)
{
    const KvPool p = kv_pool(pool, c.n_pages);
    hipLaunchKernelGGL(k_kv_compact, dim3(1), dim3(kKvPlan), 0, s, c, pool);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_kv_renumber, dim3(rows.rows), dim3(256), 0, s, c, rows, pool);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(k_kv_move, move_blocks(c, c.n_pages), dim3(kKvCopyThreads), 0, s, c, p.header, p.pairs, p.count);
    return hipGetLastError();
}

}  // namespace qp
