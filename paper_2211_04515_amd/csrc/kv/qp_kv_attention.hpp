// Attention over the 4-bit key/value cache.
//
// Mathematics.  With key t = lo + c s (per token and head: codes c, grid lo, s) a score is a dot product with codes,
//     scale q.k_t = scale (s_t sum_d q_d (c_td - 8) + (lo_t + 8 s_t) sum_d q_d),
// and with p_t = 2^(score_t - m), scores in log2, the answer's numerator is
//     sum_t p_t v_t = sum_t (p_t s_t) (c_t - 8) + sum_t p_t (lo_t + 8 s_t),
// the second term the same for all elements of a head.  So both products run on the codes themselves: c - 8 is an integer in
// [-8, 7], exact in fp16, and no value is ever dequantized.  (Centred codes, because the rounding of p_t s_t is multiplied by
// them: -8..7 costs about as much as the values' own spread would.)
//   q          is taken as 16 q in fp16: exact for bf16 (what is below 2^-14 rounds at 2^-29); fp32 is split in two halves, 22 bits
//              of each element.  A column whose largest element lies outside [2^-4, 2^11) gets a power of two of its own.
//   p_t s_t    is rounded to fp16 (fp32: split in two).  One half does for bf16 answers, whose own rounding is 1.66e-3 of them in the 2-norm: with
//              the weights' it is 1.68e-3, and one answer in ten rounds to the other neighbour.  Two would double the second product.
//              m is no maximum of the scores but the column's own reference, such that the largest p_t s_t that it has seen lies between 2^6, when m
//              was last moved, and 2^15.6: nothing overflows, and what is lost at the lower end is 2^-31 of the largest.  Of the tokens that the column sees, with the weight that it gives them: one reference for all columns of a wave, or one
//              from the scales alone, lets a token with a vast value take the bits of columns that do not see or weigh it.  p_t itself stays
//              below 2^96, which sums in fp32 hold, so where the largest p_t s_t is less than 2^-83 of the largest p_t, what is lost is 2^-114 of that.
//   Scores, sum p_t, sum p_t (lo_t + 8 s_t) and the accumulators are fp32.  m is a whole number, so that moving it rounds nothing.
//
// Matrix shape.  v_mfma_f32_16x16x32_f16 with S^T = K q^T (16 tokens x 16 columns; a column is one token of the call and one of the
// query heads that share the key head) and O^T = V^T p^T.  With 32 tokens at a time, tile row m of the first product's two
// tiles j is token 8 (m div 4) + 4 j + m mod 4: then lane 16 g + n holds the scores of tokens 8 g .. 8 g + 7 of column n,
// which is just what the second product wants of it, so p never leaves the lane.  A word of value codes is eight tokens of one
// element for the same reason; elements are dealt out as d = m NB + block so that a lane's words are next to each other.
// A word w becomes eight halves as ((w >> 8 i) & 0x000f000f | 0x6400 6400) - 1032 and (.. & 0x00f000f0 | 0x5400 5400) - 72: codes
// 0, 4, 1, 5, 2, 6, 3, 7; queries and p are put in the same order.
// The reference is lazy: m moves only when p s would pass fp16, so the loop has no exchange between lanes; what is rare is one branch of the whole
// wave, entered if a lane's largest score and its tokens' largest scale could do that together, and there each column decides for itself.  Scores are
// made relative to m in the step that applies the grid, with scale log2(e) / 16 in the grid already: two instructions for a score, and the
// exponential's argument is there.
//
// Who does what.  An item is some columns of one row and key head, a block (four waves) takes an item or a piece of its tokens:
//   few    16 columns; every wave all of them and every fourth 32 tokens, joined through LDS at the end.  What a single token of a
//          row, or a few of them, need: bound by HBM, (head_dim + 16) bytes for each token and key head.
//   many   128 columns, 32 a wave; all waves the same tokens, whose words each wave takes apart a quarter of and shares through
//          LDS.  Prompts: 12 vector instructions for each score (3 for taking codes apart) beside two matrix ones for 16.
// A call whose rows bring 16 columns or fewer on average goes to `few` alone; else rows are cut into 128 columns for `many`, and
// a rest of 16 or fewer goes to `few`, in the same launch (single tokens in a batch with prompts).  Rows' lengths are known to the device only: every
// wave adds up the whole call's work from them (a row a lane; of more than 64 rows a small kernel ahead does it once) and finds which
// item, and which of S equal pieces of its tokens, is its block's, so that about as many pieces come out as the chip runs at a time,
// whatever the lengths.  Pieces leave (m, sum p, numerators) in the workspace, sum p brought to [1/2, 1), and a last kernel joins them in order.
//
// Measured (bf16, heads of 128): one token each for 4 rows of up to 131072 (8 key heads, 64 of queries) 114 us, 4.9 TB/s, where a loop that only
// reads reaches 5.9 to 6.7; for 32 rows of up to 4096 33 us, 3.1 TB/s, of which joining and finding work are 6; a prompt of 8192 tokens (4 key
// heads, 16 of queries) 358 us, 768 TFLOP/s, where a large library product in fp16 runs at 1220.  Of the SIMDs' clocks there 59 % are vector
// instructions' and 30 % the matrix unit's: neither is full.  A wave spends half of its time in instructions, 27 % waiting for its turn to issue one
// and 23 % for data and barriers, which two waves a SIMD do not cover for each other.
#pragma once

#include "qp_kv.hpp"

namespace qp {

constexpr int kAtThreads = 256, kAtWaves = 4;
constexpr uint32_t kAtStep = 32;                 // tokens of a wave's step
constexpr uint32_t kAtTile = kAtStep * kAtWaves; // tokens that work is counted in
constexpr uint32_t kAtUnit = 16;                 // columns that partial results are counted in
template <bool MANY> constexpr uint32_t kAtCols = MANY ? 128u : kAtUnit;     // columns of an item
// The pieces that a call is cut into, no more if it can be.  Set for the blocks that run at the same time with bf16 heads of 128 (two waves a SIMD for
// many columns, three for few); at_launch takes fewer where it says so.  What registers and LDS leave room for at other sizes, waves a SIMD, which is
// blocks a CU: few columns 4 (64, and 80 in bf16), 3 (80 in fp32, 96, 128 in bf16), 2 (128 in fp32), 1 (256); many columns 2 in bf16 up to 128, else 1,
// and the few columns' items in the same launch run at that too.  So fp32 prompts of heads up to 96 are cut for twice the blocks that run, and few
// columns of 256 for 512, of heads of 64 for 768 of 1024.
#ifndef QP_KV_FEW
#define QP_KV_FEW 768
#endif
#ifndef QP_KV_MANY
#define QP_KV_MANY 512
#endif
template <bool MANY> constexpr uint32_t kAtSlots = MANY ? QP_KV_MANY : QP_KV_FEW;
// Tiles that a piece has at least: joining costs a kernel and a pass over the pieces, more than it takes to go through these.
#ifndef QP_KV_LEAST
#define QP_KV_LEAST 4
#endif
constexpr uint32_t kAtLeast = QP_KV_LEAST;
// A column's reference, in log2: p = 2^(score - m) may be up to 2^kAtMost, so that sums stay in fp32, and p times the token's value scale up to
// 2^kAtFull, so that it fits fp16; where one would pass, m rises to where the one is 2^kAtFar at most and the other 2^kAtRoom.
constexpr float kAtMost = 96.0f, kAtFar = 89.0f, kAtFull = 15.5f, kAtRoom = 8.0f;

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// A part of the workspace, for one kind of items: the header ([0] columns that were split, [1] tiles of a piece); with more rows than a
// wave has lanes where the parts of each end; a record for each column that was split; (m, sum) and numerators of the pieces, in units of
// 16 columns.
struct AtWork {
    uint32_t *header;
    u32x4 *ends;
    u32x4 *cols;
    float2 *sums;
    float *nums;
    uint32_t most_cols, most_units;
    uint32_t wide;                               // rows are cut into 128 columns first
    uint32_t slots;                              // pieces that the call is to be cut into
    uint32_t blocks;                             // of the launch
};
constexpr size_t kAtHeader = 256;
// Columns that a wave of `few` shall not take one by one: see above.
inline bool at_wide(uint32_t group, uint32_t rows, uint64_t tokens) { return tokens * group > (uint64_t)kAtUnit * rows; }
template <bool MANY> uint64_t at_items(const KvLayer &c, uint32_t group)     // at most; a row has one for each kAtCols begun
{
    const uint64_t rows = c.rows < c.tokens ? c.rows : c.tokens;
    if (!MANY && at_wide(group, c.rows, c.tokens)) return c.kv_heads * rows;
    return c.kv_heads * ((uint64_t)c.tokens * group / kAtCols<MANY> + rows);
}
// The items that are cut up have 2 kAtSlots pieces together at most, see at_share, so there are kAtSlots of them at most.
template <bool MANY> AtWork at_work(char *ws, const KvLayer &c, uint32_t dim, uint32_t group, size_t &bytes)
{
    const uint64_t tiles = (((uint64_t)c.pages_per_row << c.page_shift) + kAtTile - 1u) / kAtTile, items = at_items<MANY>(c, group);
    const uint64_t columns = (uint64_t)c.tokens * c.kv_heads * group, slots = kAtSlots<MANY>;
    uint64_t pieces = tiles <= kAtLeast ? 0u : 2u * slots, cols = tiles <= kAtLeast ? 0u : slots * kAtCols<MANY>;
    if (items < 2u * slots && items * tiles < pieces) pieces = items * tiles;
    if (columns < cols) cols = columns;
    AtWork w{};
    w.wide = at_wide(group, c.rows, c.tokens) ? 1u : 0u;
    w.slots = kAtSlots<MANY>;
    w.most_units = (uint32_t)(pieces * (kAtCols<MANY> / kAtUnit));
    w.most_cols = (uint32_t)cols;
    w.blocks = (uint32_t)(2u * slots + items);   // (pieces: see at_share; an item that is not cut up is one)
    const size_t records = kAtHeader + (c.rows > (uint32_t)kWave ? (size_t)c.rows * sizeof(u32x4) : 0u);
    const size_t sums = records + (size_t)cols * sizeof(u32x4), nums = sums + (size_t)w.most_units * kAtUnit * sizeof(float2);
    bytes = nums + (size_t)w.most_units * kAtUnit * dim * sizeof(float);
    if (ws) {
        w.header = reinterpret_cast<uint32_t *>(ws);
        w.ends = reinterpret_cast<u32x4 *>(ws + kAtHeader);
        w.cols = reinterpret_cast<u32x4 *>(ws + records);
        w.sums = reinterpret_cast<float2 *>(ws + sums);
        w.nums = reinterpret_cast<float *>(ws + nums);
    }
    return w;
}
// The whole workspace of a call.
inline size_t at_bytes(const KvLayer &c, uint32_t dim, uint32_t group, size_t &few)
{
    size_t many = 0;
    (void)at_work<false>(nullptr, c, dim, group, few);
    if (at_wide(group, c.rows, c.tokens)) (void)at_work<true>(nullptr, c, dim, group, many);
    few = (few + 255u) / 256u * 256u;
    return few + many;
}

// ---- which piece of which item a block has ---------------------------------------------------------------------------------
struct AtRow {
    KvRow row;
    uint32_t items, first, cols, tiles;          // items from column `first` on; `cols`: where the last one ends
};
template <bool MANY> __device__ __forceinline__ AtRow at_row(const KvLayer &c, const KvAttn &a, bool wide, uint32_t r)
{
    AtRow o;
    const KvRow row = o.row = kv_row(c, r);
    const uint32_t cols = (uint32_t)row.count * a.group, rest = cols % kAtCols<true>;
    const bool small = rest <= kAtUnit;          // the rest is for `few`
    o.first = !MANY && wide ? (small ? cols - rest : cols) : 0u;
    o.cols = MANY && small ? cols - rest : cols;
    o.items = (o.cols - o.first + kAtCols<MANY> - 1u) / kAtCols<MANY>;
    const int64_t from = a.window ? (int64_t)row.length - row.count - a.window + 1 : 0;
    const uint32_t lo = from > 0 ? (uint32_t)from / kAtTile : 0u, hi = ((uint32_t)row.length + kAtTile - 1u) / kAtTile;
    o.tiles = hi > lo ? hi - lo : 1u;
    return o;
}
struct AtPiece {
    KvRow at;
    uint32_t row, head, col0, col1, s, pieces;   // columns; pieces: at most so many of the item's tokens
    uint32_t per;                                // tiles that a piece should have
    uint32_t unit, rec;                          // where the item's partial results and its columns' records go
};
// Prefix sums that stay at kAtCap, which is more than any launch has, instead of passing 32 bits (rows that overlap can come to that).
constexpr uint32_t kAtCap = 0x7fffffffu;
__device__ __forceinline__ uint32_t at_plus(uint32_t x, uint32_t y) { return min(x + y, kAtCap); }
__device__ __forceinline__ uint32_t at_wave_scan(uint32_t v)
{
    const uint64_t sum = ((uint64_t)kv_wave_scan(v >> 16) << 16) + kv_wave_scan(v & 0xffffu);
    return (uint32_t)min(sum, (uint64_t)kAtCap);
}

// What a row adds to the call: blocks, units of partial results, columns with records.
template <bool MANY> struct AtParts {
    uint32_t pieces, blocks, units, cols;
    __device__ __forceinline__ AtParts(const KvLayer &c, const AtRow &o, uint32_t per)
    {
        pieces = (o.tiles + per - 1u) / per;
        blocks = c.kv_heads * o.items * pieces;
        units = pieces > 1u ? blocks * (kAtCols<MANY> / kAtUnit) : 0u;
        cols = pieces > 1u ? c.kv_heads * (o.cols - o.first) : 0u;
    }
    // `e`: where its parts end among all rows'.  True where the rows' tokens do not overlap: what the host sized the grid and the workspace for.
    __device__ __forceinline__ bool fits(const AtWork &w, const uint32_t (&e)[3]) const
    {
        return e[0] - blocks <= w.blocks && e[0] <= w.blocks && e[1] - units <= w.most_units && e[1] <= w.most_units && e[2] - cols <= w.most_cols &&
               e[2] <= w.most_cols;
    }
    // the row's block i
    __device__ __forceinline__ AtPiece piece(const KvLayer &c, const AtRow &o, uint32_t r, uint32_t per, const uint32_t (&e)[3], uint32_t i) const
    {
        AtPiece f;
        f.at = o.row;
        f.row = r;
        f.head = i % c.kv_heads;                 // heads side by side: an XCD per head, whose tokens its L2 then holds
        i /= c.kv_heads;
        f.s = i % pieces;
        const uint32_t item = o.items - 1u - i / pieces;          // the last columns, which see the most tokens, first
        f.col0 = o.first + item * kAtCols<MANY>;
        f.col1 = min(f.col0 + kAtCols<MANY>, o.cols);
        f.pieces = pieces;
        f.per = per;
        f.unit = e[1] - units + (item * c.kv_heads + f.head) * pieces * (kAtCols<MANY> / kAtUnit);
        f.rec = e[2] - cols + (f.col0 - o.first) * c.kv_heads + f.head * (f.col1 - f.col0);
        return f;
    }
};
// Tiles that a piece should have.  The pieces of a call are to run in one round, so there should be `slots` of them but no more (a piece
// too many makes a second round: 32 rows of up to 4096 tokens 33.6 us with 768 pieces, 39.8 with 800), in two rounds where the items alone are more;
// with yet more items only what is longer than a slot's share is cut.  `count(per)`: the pieces that come of a share.
// Either count(per) <= 2 slots, or per > 2 cost / slots (the steps below more than double per, and from then on an item of n tiles
// in more than one piece has less than 2 n / per): 2 slots pieces at most come of items that are cut.
template <typename Count> __device__ __forceinline__ uint32_t at_share(uint64_t cost, uint64_t items, uint32_t slots, const Count &count)
{
    const uint64_t goal = items <= slots ? slots : items <= 2u * slots ? 2u * slots : slots;
    const uint64_t share = cost + goal - 1u <= 0xffffffffull ? (uint32_t)(cost + goal - 1u) / (uint32_t)goal : (cost + goal - 1u) / goal;
    uint32_t per = (uint32_t)min(max(share, (uint64_t)kAtLeast), (uint64_t)0x3fffffffu);
    if (items <= 2u * slots)
        for (int i = 0; i < 20 && count(per) > goal; ++i) per += max(1u, per / 16u);
    return per;
}

// False: the call has fewer pieces than blocks.
template <bool MANY> __device__ __forceinline__ bool at_find(const KvLayer &c, const KvAttn &a, const AtWork &w, uint32_t block, AtPiece &mine)
{
    const uint32_t tid = threadIdx.x, lane = tid % kWave;
    AtRow none{};
    none.tiles = 1u;
    if (c.rows <= (uint32_t)kWave) {             // every wave for itself, a row a lane: nothing to wait for but the lengths
        const AtRow o = lane < c.rows ? at_row<MANY>(c, a, w.wide, lane) : none;
        const uint64_t steps = (uint64_t)o.tiles * o.items;
        const uint64_t cost = (((uint64_t)wave_sum_u32((uint32_t)(steps >> 20)) << 20) + wave_sum_u32((uint32_t)steps & 0xfffffu)) * c.kv_heads;
        const uint64_t items = (uint64_t)wave_sum_u32(o.items) * c.kv_heads;
        const uint32_t per = at_share(cost, items, w.slots, [&](uint32_t p) { return (uint64_t)wave_sum_u32(o.items * ((o.tiles + p - 1u) / p)) * c.kv_heads; });
        const AtParts<MANY> parts(c, o, per);
        const uint32_t e[3] = {at_wave_scan(parts.blocks), at_wave_scan(parts.units), at_wave_scan(parts.cols)};
        const bool fits = parts.fits(w, e);
        if (block == 0u && tid < (uint32_t)kWave) {
            const uint32_t split = wave_max_u32(fits && parts.cols != 0u ? e[2] : 0u);
            if (tid == 0u) w.header[0] = split;
        }
        const uint64_t owner = __ballot(fits && block >= e[0] - parts.blocks && block < e[0]);
        if (owner == 0ull) return false;
        const int from = __builtin_ctzll(owner);
        const auto get = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, from); };
        AtRow row{KvRow{(int32_t)get((uint32_t)o.row.begin), (int32_t)get((uint32_t)o.row.count), (int32_t)get((uint32_t)o.row.length)},
                  get(o.items), get(o.first), get(o.cols), get(o.tiles)};
        const uint32_t end[3] = {get(e[0]), get(e[1]), get(e[2])};
        const AtParts<MANY> its(c, row, per);
        mine = its.piece(c, row, (uint32_t)from, per, end, block - (end[0] - its.blocks));
        return true;
    }
    // k_kv_plan has been here: the first row that ends behind the block, 64 of them at a time
    uint32_t r = 0, n = c.rows;
    while (true) {
        const uint32_t step = (n + kWave - 1u) / kWave, at = lane * step;
        const uint32_t under = (uint32_t)__popcll(__ballot(at < n && w.ends[r + min(at, n - 1u)][0] <= block));
        if (under == 0u) break;
        r += (under - 1u) * step;
        n = min(step, c.rows - r);
        if (step == 1u) {
            ++r;
            break;
        }
    }
    if (r >= c.rows) return false;
    const u32x4 ends = w.ends[r];
    const uint32_t end[3] = {ends[0], ends[1], ends[2]}, per = w.header[1];
    const AtRow row = at_row<MANY>(c, a, w.wide, r);
    const AtParts<MANY> its(c, row, per);
    if (!its.fits(w, end) || block < end[0] - its.blocks || block >= end[0]) return false;
    mine = its.piece(c, row, r, per, end, block - (end[0] - its.blocks));
    return true;
}

__device__ __forceinline__ uint64_t at_wave_sum(uint64_t v)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) v += ((uint64_t)__shfl_xor((uint32_t)(v >> 32), d, kWave) << 32) + __shfl_xor((uint32_t)v, d, kWave);
    return v;
}

// With more rows than a wave has lanes, one block for each kind of items adds the rows up ahead of them: else every block would, and 4096 rows
// of up to 500 tokens took 1356 us, so 580; 20000 of 200 17.6 ms, so 2.0; 1024 of 1000 302, so 251.  (Where it begins is the wave's size, no
// measured crossing: 96 rows of 1000 took 30 us, so 34, which is the launch.)
constexpr uint32_t kAtPlan = 1024;
template <bool MANY> __device__ __forceinline__ void at_plan(const KvLayer &c, const KvAttn &a, const AtWork &w)
{
    __shared__ uint64_t work[kAtPlan / kWave];
    __shared__ uint32_t part[kAtPlan / kWave][3];
    __shared__ uint32_t split;
    const uint32_t tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    uint64_t cost = 0;
    for (uint32_t r = tid; r < c.rows; r += kAtPlan) {
        const AtRow o = at_row<MANY>(c, a, w.wide, r);
        cost += (uint64_t)o.tiles * o.items;
    }
    cost = at_wave_sum(cost);
    if (lane == 0u) work[wave] = cost;
    if (tid == 0u) split = 0u;
    __syncthreads();
    cost = 0;
    for (uint32_t i = 0; i < kAtPlan / kWave; ++i) cost += work[i];
    // (many rows: their mean piece is taken for what is lost at their ends)
    const uint32_t per = at_share(cost * c.kv_heads * 5u / 4u, 4u * (uint64_t)w.slots, w.slots, [](uint32_t) { return 0ull; });
    uint32_t before[3] = {0u, 0u, 0u};           // blocks, units, columns of the rows so far
    for (uint32_t r0 = 0; r0 < c.rows; r0 += kAtPlan) {
        const uint32_t r = r0 + tid;
        AtRow o{};
        o.tiles = 1u;
        if (r < c.rows) o = at_row<MANY>(c, a, w.wide, r);
        const AtParts<MANY> parts(c, o, per);
        uint32_t e[3] = {at_wave_scan(parts.blocks), at_wave_scan(parts.units), at_wave_scan(parts.cols)};
        if (lane == kWave - 1u)
            for (int k = 0; k < 3; ++k) part[wave][k] = e[k];
        __syncthreads();
        for (int k = 0; k < 3; ++k) {
            uint32_t all = before[k];
            for (uint32_t i = 0; i < kAtPlan / kWave; ++i) {
                if (i == wave) e[k] = at_plus(e[k], all);
                all = at_plus(all, part[i][k]);
            }
            before[k] = all;
        }
        if (r < c.rows) w.ends[r] = u32x4{e[0], e[1], e[2], 0u};
        if (parts.cols != 0u && parts.fits(w, e)) atomicMax(&split, e[2]);
        __syncthreads();                         // (the sums are used again)
    }
    if (tid == 0u) {
        w.header[0] = split;
        w.header[1] = per;
    }
}
template <int D> __global__ __launch_bounds__(kAtPlan) void k_kv_plan(KvLayer c, KvAttn a, AtWork few, AtWork many)
{
    if (blockIdx.x == 0u) at_plan<false>(c, a, few);
    else at_plan<true>(c, a, many);
}

// The pages of a row, 64 at a time: lane i has slot base + i's.  (A load for each would be waited for in each step: 600 cycles.)
struct AtPages {
    int32_t page;
    uint32_t base;
    __device__ __forceinline__ void load(const KvLayer &c, uint32_t row, uint32_t slot)
    {
        base = slot;
        page = kv_page(c, row, slot + threadIdx.x % kWave);
    }
    // the page of slot `slot`, which is the same in all lanes and never below an earlier call's
    __device__ __forceinline__ int32_t at(const KvLayer &c, uint32_t row, uint32_t slot)
    {
        if (slot - base >= (uint32_t)kWave) load(c, row, slot);
        return __builtin_amdgcn_readlane(page, (int)(slot - base));
    }
};

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
// A word that was loaded steps ago, looked at only now.  (Left to itself the compiler moves the first instructions of at_codes up to the
// load and waits for it there: a prompt of 8192 tokens 367 -> 387 us.)
__device__ __forceinline__ uint32_t at_now(uint32_t w)
{
#if defined(__AMDGCN__)
    asm volatile("" : "+v"(w));
#endif
    return w;
}
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
// 2^x for whole numbers x up to 127; 0 below -126.
__device__ __forceinline__ float at_power(float x) { return x < -126.0f ? 0.0f : __uint_as_float((uint32_t)((int32_t)x + 127) << 23); }
// log2 of x >= 0, between whole numbers on a straight line, which is 0.09 too low at most and never falls as x grows (0: -127); and its sum with y.
__device__ __forceinline__ float at_log2_plus(float x, float y) { return fmaf((float)__float_as_uint(x), 0x1p-23f, y - 127.0f); }

template <int D, int NCT, int DT> struct AtWave {
    static constexpr int KS = (D + 31) / 32;         // words of a lane of a key, and steps of the first product
    static constexpr int NB = D / 16;                // words of a lane of eight tokens' values, and blocks of the answer
    static constexpr int PIECES = DT == QP_F32 ? 2 : 1;
    f16x8 q[NCT][PIECES][KS];
    f32x4 o[NCT][NB];
    float m[NCT], bq[NCT], l[NCT], lv[NCT];          // m: the column's reference, a whole number
    float over[NCT];                                 // what a score relative to m may be: kAtMost, or -inf while nothing was seen
    float own[NCT];                                  // the column's own power of two
    bool owns;                                       // any column of the wave has one
    int32_t lo[NCT], hi[NCT];                        // the tokens that this lane's column sees

    struct Raw {
        uint32_t k[2][KS], v[NB];
        float2 grid;                                 // lanes 0..31: keys, 32..63: values
        bool written;                                // else the grid may be anything (looked at when it is used: not to wait for it before)
    };

    // A lane's elements of a column tile's queries as they lie in memory: 8 KS of a column's, from 8 g KS on.
    struct Query {
        u32x4 w[KS][DT == QP_F32 ? 2 : 1];
    };
    __device__ __forceinline__ void load_query(Query &x, const KvView &qv, const KvAttn &a, const KvRow &row, uint32_t head, int t, uint32_t col0, uint32_t cols) const
    {
        const uint32_t lane = threadIdx.x % kWave, g = lane / 16u, n = lane % 16u, col = col0 + 16u * t + n;
        const bool is = col < cols;
        const uint32_t i = is ? col / a.group : 0u, h = head * a.group + (is ? col % a.group : 0u);
        const unsigned char *src = qv.data + ((uint64_t)row.begin + i) * qv.token_stride + (uint64_t)h * qv.head_stride;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const uint32_t unit = g * KS + s;
#pragma unroll
            for (int z = 0; z < (DT == QP_F32 ? 2 : 1); ++z) {
                x.w[s][z] = u32x4{0u, 0u, 0u, 0u};
                if (is && unit * 8u < (uint32_t)D) x.w[s][z] = reinterpret_cast<const u32x4 *>(src)[unit * (DT == QP_F32 ? 2u : 1u) + z];
            }
        }
    }
    // Column tile t's fragments, and its columns' state.
    __device__ __forceinline__ void make_query(const Query &w, const KvAttn &a, const KvRow &row, int t, uint32_t col0, uint32_t cols)
    {
        const uint32_t col = col0 + 16u * t + threadIdx.x % 16u;
        const bool is = col < cols;
        const uint32_t i = is ? col / a.group : 0u;
        float x[KS][8];
        float top = 0.0f;
        bool bad = false;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (DT == QP_F32) x[s][e] = __uint_as_float(w.w[s][e / 4][e % 4]);
                else x[s][e] = __uint_as_float(e % 2 ? w.w[s][0][e / 2] & 0xffff0000u : w.w[s][0][e / 2] << 16);
                bad |= (__float_as_uint(x[s][e]) & 0x7f800000u) == 0x7f800000u;
                top = fmaxf(top, fabsf(x[s][e]));
            }
        }
        top = fmaxf(top, kv_xor_f32(top, 16));
        top = fmaxf(top, kv_xor_f32(top, 32));
        uint32_t any = bad ? 1u : 0u;
        any |= __shfl_xor(any, 16, kWave);
        any |= __shfl_xor(any, 32, kWave);
        int32_t up = 4;
        if (top != 0.0f && any == 0u && !(top >= 0x1p-4f && top < 0x1p11f)) {
            int32_t ex;
            (void)frexpf(top, &ex);
            up = min(15 - ex, 100);                  // q 2^up: the largest element in [2^14, 2^15)
        }
        own[t] = ldexpf(1.0f, 4 - up);
        owns = (t != 0 && owns) || __ballot(up != 4) != 0ull;
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
        bq[t] = any ? __uint_as_float(0x7fc00000u) : sum * own[t];
        m[t] = 0.0f;
        over[t] = -INFINITY;
        l[t] = lv[t] = 0.0f;
#pragma unroll
        for (int b = 0; b < NB; ++b) o[t][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        const int64_t pos = (int64_t)row.length - row.count + i;
        hi[t] = !is ? 0x7fffffff : a.causal ? (int32_t)max((int64_t)0, min(pos + 1, (int64_t)row.length)) : row.length;
        lo[t] = is && a.window ? (int32_t)max((int64_t)0, pos - (int64_t)a.window + 1) : 0;
    }

    // Where a lane's words and grid of 32 tokens lie, in bytes from the head's slab + (first token's slot) * D / 2 (the grid: + 8 of the
    // slot): codes of a token are D / 2 bytes and so is an eighth of eight tokens' values.
    uint32_t key_at, value_at, grid_at;
    __device__ __forceinline__ void place(uint32_t page_shift)
    {
        const uint32_t lane = threadIdx.x % kWave, g = lane / 16u, n = lane % 16u, pt = 1u << page_shift;
        key_at = (8u * (n / 4u) + n % 4u) * (D / 2) + g * KS * 4u;
        value_at = pt * (D / 2) + (g * D + n * NB) * 4u;
        grid_at = pt * D + (lane < 32u ? 0u : pt * 8u) + lane % 32u * 8u;
    }
    // 32 tokens from `t0` on, of the page that they all lie in
    __device__ __forceinline__ void load(Raw &x, const unsigned char *slab, uint32_t t0, uint32_t page_shift, int32_t length, bool there) const
    {
        const uint32_t in = t0 & ((1u << page_shift) - 1u);
        const unsigned char *codes = slab + (size_t)in * (D / 2);
#pragma unroll
        for (int j = 0; j < 2; ++j)      // (the last words of a key that is no multiple of 32 long lie behind it, in the slab; their queries are 0)
            __builtin_memcpy(x.k[j], codes + key_at + 4u * j * (D / 2), sizeof x.k[j]);
        __builtin_memcpy(x.v, codes + value_at, sizeof x.v);
        x.grid = *reinterpret_cast<const float2 *>(slab + (size_t)in * 8u + grid_at);
        x.written = there && (int32_t)(t0 + threadIdx.x % 32u) < length;
    }

    // The references of the columns that have to be raised.  Each column's own scores and the scales of the tokens that it sees decide (the others'
    // scores are -inf here), so that an answer is the same to the bit whatever the wave's other columns do.
    // `s`: scores relative to m, which follow; `top`: this lane's largest ones; `mem`: as in weigh
    template <int SUB, typename Mem> __device__ __forceinline__ void raise(f32x4 (&s)[SUB][NCT][2], const float (&top)[NCT], const Mem &mem)
    {
        uint32_t lane = threadIdx.x % kWave;
#if defined(__AMDGCN__)
        asm volatile("" : "+v"(lane));       // (else what follows from it is kept in registers for this branch)
#endif
        const uint32_t g = lane / 16u, n = lane % 16u;
#pragma unroll
        for (int t = 0; t < NCT; ++t) {
            // log2 of the largest p s, and of the largest p times what counts as a token's size: |lo + 8 s| too, far down, for lv's sake
            const float x = top[t];
            float weight = -INFINITY, size = -INFINITY;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 gv = mem(u)[32u + 8u * g + i];
                    const float at = s[u][t][i / 4][i % 4];
                    weight = fmaxf(weight, at_log2_plus(gv.x, at));
                    size = fmaxf(size, at_log2_plus(fmaxf(gv.x, fabsf(gv.y) * 0x1p-20f), at));
                }
            // a column's lanes are n, n + 16, n + 32, n + 48
            const bool first = over[t] < 0.0f, moves = (__ballot(x > over[t] || weight > kAtFull) >> n & 0x0001000100010001ull) != 0ull;
            float by = fmaxf(x - kAtFar, size - kAtRoom);
            by = fmaxf(by, kv_xor_f32(by, 16));
            by = fmaxf(by, kv_xor_f32(by, 32));
            // (whole numbers: what was summed is scaled by powers of two, without a rounding)
            const float up = moves ? ceilf(by) : 0.0f;
            over[t] = moves ? kAtMost : over[t];
            m[t] += up;
            float down = first ? 1.0f : at_power(-up);                // (first: there is nothing to scale)
#if defined(__AMDGCN__)
            asm volatile("" : "+v"(down));   // (else lanes that do not move branch past the products, which copies o: 28 registers, a block less a CU)
#endif
            l[t] *= down;
            lv[t] *= down;
#pragma unroll
            for (int b = 0; b < NB; ++b) o[t][b] *= down;
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                s[u][t][0] -= up;
                s[u][t][1] -= up;
            }
        }
    }

    // What a step makes of a grid: {scale, lo + 8 scale}; those of keys (lanes 0..31, values 32..63) with the scores' factor.
    static __device__ __forceinline__ float2 centred(float2 grid, bool written, float key_factor)
    {
        const float f = threadIdx.x % kWave < 32u ? key_factor : 1.0f;
        return written ? float2{grid.y * f, fmaf(8.0f, grid.y, grid.x) * f} : float2{0.0f, 0.0f};
    }

    // Scores of 32 SUB tokens, before the grids: the first product.  `key(u, j, k)`: the fragments.
    template <int SUB> struct Scores {
        f32x4 s[SUB][NCT][2];
    };
    template <int SUB, typename Key> __device__ __forceinline__ void products(Scores<SUB> &x, const Key &key) const
    {
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
#pragma unroll
            for (int t = 0; t < NCT; ++t) x.s[u][t][0] = x.s[u][t][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const f16x8 a = key(u, j, k);
#pragma unroll
                    for (int t = 0; t < NCT; ++t)
#pragma unroll
                        for (int z = PIECES - 1; z >= 0; --z) x.s[u][t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, q[t][z][k], x.s[u][t][j], 0, 0, 0);
                }
        }
    }
    // The rest of a step: softmax and the second product.  `value(u, b)`: the fragments; `mem(u)`: scales and lo + 8 scale of 32 keys, then of
    // 32 values; `there(u)`: the page is.
    template <int SUB, typename Value, typename Mem, typename There>
    __device__ __forceinline__ void weigh(Scores<SUB> &x, const Value &value, const Mem &mem, uint32_t t0, bool whole, const There &there)
    {
        const uint32_t lane = threadIdx.x % kWave, g = lane / 16u;
        float top[NCT], sv_top = 0.0f;
        if (owns) {
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int t = 0; t < NCT; ++t) {
                    x.s[u][t][0] *= own[t];
                    x.s[u][t][1] *= own[t];
                }
        }
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            float sk[8], bk[8];                           // of tokens 8 g + i
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 gk = mem(u)[8u * g + i];
                sk[i] = gk.x;
                bk[i] = gk.y;
                sv_top = fmaxf(sv_top, mem(u)[32u + 8u * g + i].x);
            }
#pragma unroll
            for (int t = 0; t < NCT; ++t)
#pragma unroll
                for (int i = 0; i < 8; ++i) x.s[u][t][i / 4][i % 4] = fmaf(x.s[u][t][i / 4][i % 4], sk[i], fmaf(bk[i], bq[t], -m[t]));
        }
        if (!whole) {
            uint32_t from = t0 + 8u * g;
#if defined(__AMDGCN__)
            asm volatile("" : "+v"(from));   // (keeps this inside the branch: else it is in every step)
#endif
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int t = 0; t < NCT; ++t)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int32_t tok = (int32_t)from + 32 * u + i;
                        if (!there(u) || tok < lo[t] || tok >= hi[t]) x.s[u][t][i / 4][i % 4] = -INFINITY;
                    }
        }
        // No column moves if its largest score in this lane would not with the largest scale of the lane's tokens, seen or not.  (2^-6 less than what it may
        // be, for the roundings on both sides: whether a column moves depends on nothing but the column)
        const float room = kAtFull - 0x1p-6f - at_log2_plus(sv_top, 0.0f);
        bool moves = false;
#pragma unroll
        for (int t = 0; t < NCT; ++t) {
            top[t] = x.s[0][t][0][0];
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = u ? 0 : 1; i < 8; ++i) top[t] = fmaxf(top[t], x.s[u][t][i / 4][i % 4]);
            moves |= top[t] > fminf(over[t], room);
        }
        if (__ballot(moves) != 0ull) raise<SUB>(x.s, top, mem);
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            f16x8 p[NCT][PIECES];
            float sv[8], bv[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 gv = mem(u)[32u + 8u * g + i];
                sv[i] = gv.x;
                bv[i] = gv.y;
            }
#pragma unroll
            for (int t = 0; t < NCT; ++t) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float e = at_exp2(x.s[u][t][i / 4][i % 4]);
                    l[t] += e;
                    lv[t] = fmaf(e, bv[i], lv[t]);
                    float w = e * sv[i];
#if defined(__AMDGCN__)
                    // (else one half's product is rounded to fp32 first and the other's is not, and where that makes a difference, once in
                    // 2^13 weights, the halves do not add up: answers off by 1e-4)
                    if constexpr (PIECES == 2) asm volatile("" : "+v"(w));
#endif
                    const int at = i % 4 * 2 + i / 4;     // code order
                    p[t][0][at] = (_Float16)w;
                    if constexpr (PIECES == 2) p[t][1][at] = (_Float16)(w - (float)p[t][0][at]);
                }
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const f16x8 a = value(u, b);
#pragma unroll
                for (int t = 0; t < NCT; ++t)
#pragma unroll
                    for (int z = PIECES - 1; z >= 0; --z) o[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, p[t][z], o[t][b], 0, 0, 0);
            }
        }
    }

    // One wave for itself: 32 tokens that it has loaded.  `mem`: this wave's own.
    __device__ __forceinline__ void step_alone(const Raw &x, float2 *mem, const AtMagic &magic, float key_factor, uint32_t t0, bool whole, bool there)
    {
        mem[threadIdx.x % kWave] = centred(x.grid, x.written, key_factor);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        Scores<1> s;
        products<1>(s, [&](int, int j, int k) { return at_codes(at_now(x.k[j][k]), magic); });
        weigh<1>(s, [&](int, int b) { return at_codes(at_now(x.v[b]), magic); }, [&](int) { return mem; }, t0, whole, [&](int) { return there; });
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }

    // The sums of all lanes of a column; o becomes the numerator.  l is brought to [1/2, 1), so that m of different waves and pieces compare.
    __device__ __forceinline__ void finish()
    {
#pragma unroll
        for (int t = 0; t < NCT; ++t) {
            l[t] += kv_xor_f32(l[t], 16);
            l[t] += kv_xor_f32(l[t], 32);
            lv[t] += kv_xor_f32(lv[t], 16);
            lv[t] += kv_xor_f32(lv[t], 32);
            int32_t ex;
            const bool none = l[t] == 0.0f;
            l[t] = frexpf(l[t], &ex);
            m[t] = none ? -3.402823466e38f : m[t] + (float)ex;   // (a column that saw nothing: below any other)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[t][b][r] = ldexpf(o[t][b][r] + lv[t], -ex);
        }
    }
};

__device__ __forceinline__ uint32_t at_bf16(float f)
{
    const uint32_t u = __float_as_uint(f);
    return (u & 0x7fffffffu) > 0x7f800000u ? (u >> 16) | 0x40u : (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

// What a block of either kind knows of its piece.
struct AtBlock {
    KvRow row;
    AtPiece p;
    uint32_t pieces;             // of the item, as many as it has tiles for
    uint32_t t0, t1;             // the piece's tokens; t0 a multiple of kAtTile
};
// the tokens that any of the row's columns [from, to) sees
__device__ __forceinline__ void at_range(const KvRow &row, const KvAttn &a, uint32_t from, uint32_t to, uint32_t &lo, uint32_t &hi)
{
    const int64_t start = (int64_t)row.length - row.count;
    const int64_t first = start + from / a.group, last = start + (to - 1u) / a.group;
    lo = a.window ? (uint32_t)max((int64_t)0, first - (int64_t)a.window + 1) : 0u;
    hi = a.causal ? (uint32_t)max((int64_t)0, min(last + 1, (int64_t)row.length)) : (uint32_t)row.length;
    if (lo > hi) lo = hi;
}
template <bool MANY> __device__ __forceinline__ bool at_begin(const KvLayer &c, const KvAttn &a, const AtWork &w, uint32_t block, AtBlock &b)
{
    if (!at_find<MANY>(c, a, w, block, b.p)) return false;
    AtPiece &p = b.p;
    p.row = __builtin_amdgcn_readfirstlane(p.row);
    p.head = __builtin_amdgcn_readfirstlane(p.head);
    p.col0 = __builtin_amdgcn_readfirstlane(p.col0);
    p.col1 = __builtin_amdgcn_readfirstlane(p.col1);
    p.s = __builtin_amdgcn_readfirstlane(p.s);
    p.pieces = __builtin_amdgcn_readfirstlane(p.pieces);
    p.per = __builtin_amdgcn_readfirstlane(p.per);
    b.row = KvRow{__builtin_amdgcn_readfirstlane(p.at.begin), __builtin_amdgcn_readfirstlane(p.at.count), __builtin_amdgcn_readfirstlane(p.at.length)};
    uint32_t lo, hi;
    at_range(b.row, a, p.col0, p.col1, lo, hi);
    const uint32_t first = lo / kAtTile, tiles = hi > lo ? (hi + kAtTile - 1u) / kAtTile - first : 0u;
    b.pieces = max(1u, min(p.pieces, (tiles + p.per - 1u) / p.per));
    if (p.pieces > 1u && p.s == 0u)           // the columns' records for the kernel that joins them
        for (uint32_t k = threadIdx.x; k < p.col1 - p.col0; k += kAtThreads) {
            const uint32_t col = p.col0 + k, place = (uint32_t)b.row.begin + col / a.group, h = p.head * a.group + col % a.group;
            w.cols[p.rec + k] = u32x4{p.unit * kAtUnit + k, b.pieces > 1u ? b.pieces : 0u, kAtCols<MANY>, place * (c.kv_heads * a.group) + h};
        }
    if (p.s >= b.pieces) return false;
    const uint32_t each = tiles / b.pieces, more = tiles % b.pieces;          // (the first `more` pieces have one more)
    const uint32_t from = first + p.s * each + min(p.s, more);
    b.t0 = from * kAtTile;
    b.t1 = min((from + each + (p.s < more ? 1u : 0u)) * kAtTile, hi);
    return true;
}
// The tokens that all of a wave's columns see.
template <typename Wave, int NCT> __device__ __forceinline__ void at_sees(const Wave &x, int32_t &lo, int32_t &hi)
{
    lo = 0;
    hi = 0x7fffffff;
#pragma unroll
    for (int t = 0; t < NCT; ++t) {
        lo = max(lo, x.lo[t]);
        hi = min(hi, x.hi[t]);
    }
#pragma unroll
    for (int d = 1; d < 16; d *= 2) {
        lo = max(lo, (int32_t)__shfl_xor((uint32_t)lo, d, kWave));
        hi = min(hi, (int32_t)__shfl_xor((uint32_t)hi, d, kWave));
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
}
// A wave's columns [col0, col1): the answer, or the piece's part of it (`k0`: the first one's place in the item).
template <int D, int NCT, int DT>
__device__ __forceinline__ void at_store(const AtWave<D, NCT, DT> &x, const AtBlock &b, const KvAttn &a, const AtWork &w, const KvView &out, uint32_t item_cols,
                                         uint32_t col0, uint32_t col1)
{
    constexpr int NB = AtWave<D, NCT, DT>::NB;
    const uint32_t lane = threadIdx.x % kWave, g = lane / 16u, n = lane % 16u;
#pragma unroll
    for (int t = 0; t < NCT; ++t) {
        const uint32_t col = col0 + 16u * t + n;
        if (col >= col1) continue;
        float v[4 * NB];
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
#pragma unroll
            for (int i = 0; i < NB; ++i) v[r4 * NB + i] = x.o[t][i][r4];
        if (b.pieces > 1u) {
            const size_t at = (size_t)b.p.unit * kAtUnit + (size_t)b.p.s * item_cols + (col - b.p.col0);
            if (g == 0u) w.sums[at] = float2{x.m[t], x.l[t]};
            f32x4 *dst = reinterpret_cast<f32x4 *>(w.nums + at * D + 4u * NB * g);
#pragma unroll
            for (int i = 0; i < NB; ++i) dst[i] = f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
            continue;
        }
        const float inv = x.l[t] == 0.0f ? 0.0f : 1.0f / x.l[t];
        unsigned char *dst = out.data + ((uint64_t)b.row.begin + col / a.group) * out.token_stride + (uint64_t)(b.p.head * a.group + col % a.group) * out.head_stride;
        if constexpr (DT == QP_F32) {
            f32x4 *d4 = reinterpret_cast<f32x4 *>(dst) + NB * g;
#pragma unroll
            for (int i = 0; i < NB; ++i) d4[i] = f32x4{v[4 * i] * inv, v[4 * i + 1] * inv, v[4 * i + 2] * inv, v[4 * i + 3] * inv};
        } else {
            u32x2 *d2 = reinterpret_cast<u32x2 *>(dst) + NB * g;
#pragma unroll
            for (int i = 0; i < NB; ++i)
                d2[i] = u32x2{at_bf16(v[4 * i] * inv) | (at_bf16(v[4 * i + 1] * inv) << 16),
                              at_bf16(v[4 * i + 2] * inv) | (at_bf16(v[4 * i + 3] * inv) << 16)};
        }
    }
}

// LDS of a block with few columns: two waves' numerators and (m, sum) when the four are joined; the grids of each wave's step.
template <int D> struct AtFewLds {
    float nums[2][16][D + 4];
    float2 grids[kAtWaves][64];
    float2 sums[2][16];
};
template <int D, int DT>
__device__ __forceinline__ void at_few(const KvLayer &c, const KvView &qv, const KvView &out, const KvAttn &a, const AtWork &w, uint32_t block, AtFewLds<D> &lds)
{
    using Wave = AtWave<D, 1, DT>;
    constexpr int NB = Wave::NB;
    float (&nums)[2][16][D + 4] = lds.nums;
    float2 (&sums)[2][16] = lds.sums;
    float2 (&grids)[kAtWaves][64] = lds.grids;
    AtBlock b;
    if (!at_begin<false>(c, a, w, block, b)) return;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, g = lane / 16u, n = lane % 16u;
    AtPages pages;
    const auto slab_at = [&](uint32_t t, bool &there) {
        const int32_t page = pages.at(c, b.p.row, t >> c.page_shift);
        there = page >= 0;
        return kv_slab(c, there ? page : 0, b.p.head);
    };
    // Two steps' words are on their way: a step's registers are filled again, for the step after the next, as soon as it is done
    // with them.  (Three or four fit no longer three blocks on a CU.)
    constexpr int kAhead = 2;
    Wave x;
    typename Wave::Query query;
    typename Wave::Raw raw[kAhead];
    bool there[kAhead];
    uint32_t t0 = b.t0 + wave * kAtStep;
    x.place(c.page_shift);
    x.load_query(query, qv, a, b.row, b.p.head, 0, b.p.col0, b.p.col1);       // (all of it on its way at once)
    pages.load(c, b.p.row, t0 >> c.page_shift);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        there[i] = false;
        if (t0 + i * kAtTile < b.t1) {
            const unsigned char *slab = slab_at(t0 + i * kAtTile, there[i]);
            x.load(raw[i], slab, t0 + i * kAtTile, c.page_shift, b.row.length, there[i]);
        }
    }
    x.make_query(query, a, b.row, 0, b.p.col0, b.p.col1);
    int32_t sees_lo, sees_hi;
    at_sees<Wave, 1>(x, sees_lo, sees_hi);
    const AtMagic magic;
    const float key_factor = a.scale * (1.44269504088896341f / 16.0f);
    while (t0 < b.t1) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (t0 >= b.t1) break;
            const bool whole = there[i] && (int32_t)t0 >= sees_lo && (int32_t)(t0 + kAtStep) <= sees_hi;
            x.step_alone(raw[i], grids[wave], magic, key_factor, t0, whole, there[i]);
            if (t0 + kAhead * kAtTile < b.t1) {
                const unsigned char *slab = slab_at(t0 + kAhead * kAtTile, there[i]);
                x.load(raw[i], slab, t0 + kAhead * kAtTile, c.page_shift, b.row.length, there[i]);
            }
            t0 += kAtTile;
        }
    }
    x.finish();
#pragma unroll
    for (uint32_t half = 2; half >= 1; half /= 2) {      // waves 2, 3 into 0, 1, then 1 into 0
        if (wave >= half && wave < 2u * half) {
            float *dst = &nums[wave - half][n][4u * NB * g];
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
#pragma unroll
                for (int i = 0; i < NB; ++i) dst[r4 * NB + i] = x.o[0][i][r4];
            if (g == 0u) sums[wave - half][n] = float2{x.m[0], x.l[0]};
        }
        __syncthreads();
        if (wave < half) {
            const float *src = &nums[wave][n][4u * NB * g];
            const float2 other = sums[wave][n];
            const float top = fmaxf(x.m[0], other.x), ea = at_exp2(x.m[0] - top), eb = at_exp2(other.x - top);
            x.m[0] = top;
            x.l[0] = fmaf(x.l[0], ea, other.y * eb);
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
#pragma unroll
                for (int i = 0; i < NB; ++i) x.o[0][i][r4] = fmaf(x.o[0][i][r4], ea, src[r4 * NB + i] * eb);
        }
        __syncthreads();
    }
    if (wave == 0u) at_store<D, 1, DT>(x, b, a, w, out, kAtCols<false>, b.p.col0, b.p.col1);
}

template <int D, int DT>
__global__ __launch_bounds__(kAtThreads, D <= 128 ? 2 : 1) void k_kv_attention_few(KvLayer c, KvView qv, KvView out, KvAttn a, AtWork w, uint32_t block0)
{
    __shared__ __align__(16) AtFewLds<D> lds;
    at_few<D, DT>(c, qv, out, a, w, block0 + blockIdx.x, lds);
}

// Of 32 tokens: the fragments of keys (j, k), then of values, and the grids.
template <int D> struct AtStage {
    f16x8 frags[2 * ((D + 31) / 32) + D / 16][kWave];
    float2 grids[64];
};
template <int D> constexpr uint32_t kAtSub = D <= 128 ? 2 : 1;      // of them between two barriers
template <int D, int DT>
__device__ __forceinline__ void at_many(const KvLayer &c, const KvView &qv, const KvView &out, const KvAttn &a, const AtWork &w, uint32_t block,
                                        AtStage<D> (&stages)[2][kAtSub<D>])
{
    constexpr int NCT = 2;
    using Wave = AtWave<D, NCT, DT>;
    using Stage = AtStage<D>;
    constexpr int NB = Wave::NB, KS = Wave::KS;
    constexpr uint32_t kSub = kAtSub<D>, kStage = kSub * kAtStep;
    AtBlock b;
    if (!at_begin<true>(c, a, w, block, b)) return;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, g = lane / 16u, n = lane % 16u;
    const uint32_t col0 = min(b.p.col0 + wave * 16u * NCT, b.p.col1), col1 = min(col0 + 16u * NCT, b.p.col1);
    const AtMagic magic;
    const float key_factor = a.scale * (1.44269504088896341f / 16.0f);
    // Every wave takes a quarter of a stage's words apart for all of them: while the waves go through a stage, the next one's
    // fragments go to the other half of LDS and the words of the one after it are on their way.  A wave has one of the two tiles of
    // keys and half of the values of 32 tokens, each one load (of heads of 256 either a tile of keys or half of the values: the stage
    // is 32 tokens then): with a load for each fragment, a prompt of 8192 tokens took 402 us, so 381.
    constexpr int kHalf = (NB + 1) / 2;
    const uint32_t mine = kSub == 2u ? wave / 2u : 0u, side = wave % 2u;
    const bool keys = kSub == 2u || wave < 2u, values = kSub == 2u || wave >= 2u;
    uint32_t wk[KS], wv[kHalf];
    float2 grid{0.0f, 0.0f};
    bool written = false;
    bool there[3][kSub];                                            // of this stage, the next, the one after
    // where this lane's words of 32 tokens lie, as in AtWave::place
    const uint32_t key_at = (8u * (n / 4u) + 4u * side + n % 4u) * (D / 2) + g * KS * 4u;
    const uint32_t value_at = (D / 2 << c.page_shift) + (g * D + n * NB + side * kHalf) * 4u;
    const uint32_t grid_at = (D << c.page_shift) + (lane < 32u ? 0u : 8u << c.page_shift) + lane % 32u * 8u;
    AtPages pages;
    pages.load(c, b.p.row, b.t0 >> c.page_shift);
    const auto fetch = [&](uint32_t t, bool (&is)[kSub]) {
        int32_t page = -1;
#pragma unroll
        for (uint32_t u = 0; u < kSub; ++u) {
            const uint32_t at = t + u * kAtStep;
            const int32_t p = at < b.t1 ? pages.at(c, b.p.row, at >> c.page_shift) : -1;
            is[u] = p >= 0;
            if (u == mine) page = p;
        }
        const uint32_t at = t + mine * kAtStep, in = at & ((1u << c.page_shift) - 1u);
        const unsigned char *slab = kv_slab(c, page < 0 ? 0 : page, b.p.head), *codes = slab + (size_t)in * (D / 2);
        if (keys) __builtin_memcpy(wk, codes + key_at, sizeof wk);
        if (values) __builtin_memcpy(wv, codes + value_at, sizeof wv);   // (an odd number of blocks: the last word is not this head's, and not used)
        if (keys) grid = *reinterpret_cast<const float2 *>(slab + (size_t)in * 8u + grid_at);
        written = page >= 0 && (int32_t)(at + lane % 32u) < b.row.length;
    };
    const auto put = [&](uint32_t half) {
        Stage &st = stages[half][mine];
        if (keys) {
#pragma unroll
            for (uint32_t k = 0; k < (uint32_t)KS; ++k) st.frags[side * KS + k][lane] = at_codes(at_now(wk[k]), magic);
        }
        if (values) {
#pragma unroll
            for (uint32_t i = 0; i < (uint32_t)kHalf; ++i)
                if (NB % 2 == 0 || side * kHalf + i < (uint32_t)NB) st.frags[2 * KS + side * kHalf + i][lane] = at_codes(at_now(wv[i]), magic);
        }
        if (keys) st.grids[lane] = Wave::centred(grid, written, key_factor);      // (both sides the same: no branch)
    };
    uint32_t half = 0u;
    fetch(b.t0, there[0]);                                          // (on its way while the queries are made ready; past the end: page 0, unused)
    Wave x;
    typename Wave::Query query;
#pragma unroll
    for (int i = 0; i < NCT; ++i) {
        x.load_query(query, qv, a, b.row, b.p.head, i, col0, col1);
        x.make_query(query, a, b.row, i, col0, col1);
    }
    int32_t sees_lo, sees_hi;
    at_sees<Wave, NCT>(x, sees_lo, sees_hi);
    uint32_t w_lo = 0u, w_hi = 0u;                                  // what any of this wave's columns sees
    if (col0 < col1) at_range(b.row, a, col0, col1, w_lo, w_hi);
    put(0u);
    fetch(b.t0 + kStage, there[1]);
    __syncthreads();
    for (uint32_t t = b.t0; t < b.t1; t += kStage) {
        if (t + kStage > w_lo && t < w_hi) {
            const Stage(&st)[kSub] = stages[half];
            bool all = true;
#pragma unroll
            for (uint32_t u = 0; u < kSub; ++u) all = all && there[0][u];
            const bool whole = all && (int32_t)t >= sees_lo && (int32_t)(t + kStage) <= sees_hi;
            typename Wave::template Scores<kSub> s;
            x.template products<kSub>(s, [&](int u, int j, int k) { return st[u].frags[j * KS + k][lane]; });
            put(half ^ 1u);                   // (between the products, as far as the compiler mixes them: the one is the matrix unit's)
            fetch(t + 2u * kStage, there[2]);
            x.template weigh<kSub>(s, [&](int u, int i) { return st[u].frags[2 * KS + i][lane]; }, [&](int u) { return st[u].grids; }, t, whole,
                                   [&](int u) { return there[0][u]; });
        } else {
            put(half ^ 1u);
            fetch(t + 2u * kStage, there[2]);
        }
        __syncthreads();
        half ^= 1u;
#pragma unroll
        for (uint32_t u = 0; u < kSub; ++u) {
            there[0][u] = there[1][u];
            there[1][u] = there[2][u];
        }
    }
    x.finish();
    at_store<D, NCT, DT>(x, b, a, w, out, kAtCols<true>, col0, col1);
}

// Both kinds at once: the rests that are for `few` come behind the others, beside their last work (a launch of their own: 4 rows
// of 130 new tokens and 1000 in all 58 us, so 47; a prompt of 2048 among 63 single tokens 155, so 148).
template <int D, int DT>
__global__ __launch_bounds__(kAtThreads, D <= 128 && DT == QP_BF16 ? 2 : 1) void k_kv_attention_many(KvLayer c, KvView qv, KvView out, KvAttn a, AtWork few, AtWork many,
                                                                                                     uint32_t block0)
{
    union Lds {
        AtFewLds<D> few;
        AtStage<D> many[2][kAtSub<D>];
    };
    __shared__ __align__(16) unsigned char lds[sizeof(Lds)];
    const uint32_t block = block0 + blockIdx.x;
    if (block < many.blocks) at_many<D, DT>(c, qv, out, a, many, block, *reinterpret_cast<AtStage<D>(*)[2][kAtSub<D>]>(lds));
    else at_few<D, DT>(c, qv, out, a, few, block - many.blocks, *reinterpret_cast<AtFewLds<D> *>(lds));
}

// ---- the pieces of a column, joined ----------------------------------------------------------------------------------------
// Few columns (single tokens, perhaps of very long rows): a block a column, every fourth piece a wave.  Many: a wave a column.
constexpr uint32_t kAtJoinBlocks = 2048, kAtJoinFew = 2048;
template <int D, int DT> __device__ __forceinline__ void at_answer(const KvView &out, uint32_t q_heads, uint32_t place, uint32_t d, float v)
{
    unsigned char *dst = out.data + (uint64_t)(place / q_heads) * out.token_stride + (uint64_t)(place % q_heads) * out.head_stride;
    if constexpr (DT == QP_F32) reinterpret_cast<float *>(dst)[d] = v;
    else reinterpret_cast<uint16_t *>(dst)[d] = (uint16_t)at_bf16(v);
}
__device__ __forceinline__ float at_wave_sum(float v)
{
    v += dpp_f32<kDppQuadSwap1>(v);
    v += dpp_f32<kDppQuadSwap2>(v);
    v += dpp_f32<kDppHalfMirror>(v);
    v += dpp_f32<kDppRowMirror>(v);
    v += kv_xor_f32(v, 16);
    return v + kv_xor_f32(v, 32);
}
template <int D, int DT> __global__ __launch_bounds__(kAtThreads) void k_kv_join(KvView out, uint32_t q_heads, AtWork few, AtWork many)
{
    constexpr int PER = (D + kWave - 1) / kWave;
    constexpr uint32_t kMost = 2u * (kAtSlots<false> > kAtSlots<true> ? kAtSlots<false> : kAtSlots<true>);
    __shared__ float weight[kMost];
    __shared__ float part[kAtWaves][D], top_of[kAtWaves], sum_of[kAtWaves];
    const uint32_t tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
    const uint32_t first = few.most_cols ? few.header[0] : 0u, count = first + (many.most_cols ? many.header[0] : 0u);
    if (count > kAtJoinFew) {
        for (uint32_t k = blockIdx.x * kAtWaves + wave; k < count; k += gridDim.x * kAtWaves) {
            const AtWork &w = k < first ? few : many;
            const u32x4 rec = w.cols[k < first ? k : k - first];
            const uint32_t pieces = rec[1];
            if (pieces == 0u) continue;       // its item came out in one piece after all
            float top = -3.402823466e38f, sum = 0.0f, acc[PER];
            for (uint32_t i = lane; i < pieces; i += kWave) top = fmaxf(top, w.sums[rec[0] + (size_t)i * rec[2]].x);
            top = wave_max(top);
#pragma unroll
            for (int z = 0; z < PER; ++z) acc[z] = 0.0f;
            for (uint32_t i0 = 0; i0 < pieces; i0 += kWave) {
                float e = 0.0f;
                if (i0 + lane < pieces) {
                    const float2 ml = w.sums[rec[0] + (size_t)(i0 + lane) * rec[2]];
                    e = at_exp2(ml.x - top);
                    sum = fmaf(e, ml.y, sum);
                }
                const uint32_t n = min((uint32_t)kWave, pieces - i0);
                for (uint32_t i = 0; i < n; ++i) {
                    const float *src = w.nums + (rec[0] + (size_t)(i0 + i) * rec[2]) * D;
                    const float f = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(e), i));
#pragma unroll
                    for (int z = 0; z < PER; ++z)
                        if (lane + kWave * z < (uint32_t)D) acc[z] = fmaf(f, src[lane + kWave * z], acc[z]);
                }
            }
            sum = at_wave_sum(sum);
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
            for (int z = 0; z < PER; ++z)
                if (lane + kWave * z < (uint32_t)D) at_answer<D, DT>(out, q_heads, rec[3], lane + kWave * z, acc[z] * inv);
        }
        return;
    }
    for (uint32_t k = blockIdx.x; k < count; k += gridDim.x) {
        const AtWork &w = k < first ? few : many;
        const u32x4 rec = w.cols[k < first ? k : k - first];
        const uint32_t pieces = rec[1];
        if (pieces == 0u) continue;
        // (a lane's first piece, and each wave's first row of numerators, on their way before the sums are known)
        const float2 ml0 = tid < pieces ? w.sums[rec[0] + (size_t)tid * rec[2]] : float2{-3.402823466e38f, 0.0f};
        float first_row[PER];
#pragma unroll
        for (int z = 0; z < PER; ++z) first_row[z] = wave < pieces && lane + kWave * z < (uint32_t)D ? w.nums[(rec[0] + (size_t)wave * rec[2]) * D + lane + kWave * z] : 0.0f;
        float top = ml0.x;
        for (uint32_t i = tid + kAtThreads; i < pieces; i += kAtThreads) top = fmaxf(top, w.sums[rec[0] + (size_t)i * rec[2]].x);
        top = wave_max(top);
        if (lane == 0u) top_of[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(top_of[0], top_of[1]), fmaxf(top_of[2], top_of[3]));
        float sum = 0.0f;
        for (uint32_t i = tid; i < pieces; i += kAtThreads) {
            const float2 ml = i == tid ? ml0 : w.sums[rec[0] + (size_t)i * rec[2]];
            const float e = at_exp2(ml.x - top);
            weight[i] = e;
            sum = fmaf(e, ml.y, sum);
        }
        sum = at_wave_sum(sum);
        if (lane == 0u) sum_of[wave] = sum;
        __syncthreads();
        float acc[PER];
#pragma unroll
        for (int z = 0; z < PER; ++z) acc[z] = wave < pieces ? weight[wave] * first_row[z] : 0.0f;
#pragma unroll 4
        for (uint32_t i = wave + kAtWaves; i < pieces; i += kAtWaves) {
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
        for (uint32_t d = tid; d < (uint32_t)D; d += kAtThreads)
            at_answer<D, DT>(out, q_heads, rec[3], d, ((part[0][d] + part[1][d]) + (part[2][d] + part[3][d])) * inv);
        __syncthreads();                      // (the shared arrays are used again)
    }
}

template <int D, int DT>
static hipError_t at_launch(const KvLayer &c, const KvView &q, const KvView &out, const KvAttn &a, char *ws, hipStream_t s)
{
    const bool wide = at_wide(a.group, c.rows, c.tokens);
    size_t few_bytes, bytes;
    (void)at_bytes(c, D, a.group, few_bytes);
    AtWork few = at_work<false>(ws, c, D, a.group, bytes);
    AtWork many = wide ? at_work<true>(ws + few_bytes, c, D, a.group, bytes) : AtWork{};
    if (D == 256 || (D == 128 && DT == QP_F32)) {      // (one block a CU with many columns; with few two of 128 in fp32, one of 256)
        few.slots = kAtSlots<false> * 2u / 3u;
        many.slots = kAtSlots<true> / 2u;
    }
    hipError_t e;
    if (c.rows > (uint32_t)kWave) {
        hipLaunchKernelGGL(k_kv_plan<D>, dim3(wide ? 2u : 1u), dim3(kAtPlan), 0, s, c, a, few, many);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    e = kv_launches((uint64_t)many.blocks + few.blocks, [&](dim3 grid, uint32_t block0) {
        if (wide) hipLaunchKernelGGL((k_kv_attention_many<D, DT>), grid, dim3(kAtThreads), 0, s, c, q, out, a, few, many, block0);
        else hipLaunchKernelGGL((k_kv_attention_few<D, DT>), grid, dim3(kAtThreads), 0, s, c, q, out, a, few, block0);
    });
    if (e != hipSuccess) return e;
    const uint32_t cols = few.most_cols + many.most_cols;
    if (cols == 0u) return hipSuccess;        // no row is longer than a piece
    hipLaunchKernelGGL((k_kv_join<D, DT>), dim3(cols < kAtJoinBlocks ? cols : kAtJoinBlocks), dim3(kAtThreads), 0, s, out, c.kv_heads * a.group, few, many);
    return hipGetLastError();
}

template <int D> hipError_t at_dim(const KvLayer &c, int dtype, const KvView &q, const KvView &out, const KvAttn &a, void *ws, hipStream_t s)
{
    char *p = static_cast<char *>(ws);
    return dtype == QP_F32 ? at_launch<D, QP_F32>(c, q, out, a, p, s) : at_launch<D, QP_BF16>(c, q, out, a, p, s);
}
#define QP_KV_ATTENTION_DIM(D) \
    template hipError_t at_dim<D>(const KvLayer &, int, const KvView &, const KvView &, const KvAttn &, void *, hipStream_t)

}  // namespace qp
