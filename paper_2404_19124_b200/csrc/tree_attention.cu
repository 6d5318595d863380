// Attention of a tree of drafted tokens over a paged cache and the tree itself: softmax(scale Q K^T + mask) V with the scores
// and the sums on the tensor cores (tcgen05), fp32 in TMEM.
//
// Work.  A unit is a sequence, a key head and up to 256 of the query rows that share it (row = node * group + head within the
// group); its keys, the cache's and then the tree's, are cut into tiles of 128.  All tiles of all units in a row are dealt to
// the CTAs, one per SM, in runs of equal cost (see Deal), so that ragged batches and few long sequences fill the GPU alike.  A unit
// that a CTA has to itself is written straight to `out`; of the others every CTA leaves its rows, normalised, with their
// log-sum-exp in the workspace, and tree_combine_kernel joins them.  Lengths are read on the device: a captured launch
// serves any.
//
// Roles of a CTA (20 warps):
//   warps 0-3, 4-7  softmax of stream 0 and 1, a thread per row: scores from TMEM, running maximum and sum, probabilities back to
//                   TMEM in place of the scores, results
//   warps 8, 9      one lane issues the MMAs of stream 0 and of stream 1:  S = Q K^T [128 x 64], O += P V, P read from TMEM; a
//                   lane for both spent as long on waits and commits as the tensor cores on the products.  Warp 8 allocates TMEM
//   warps 10, 11    nothing (registers are given away by groups of four warps)
//   warps 12-15     bring the tiles of K and V that lie in the cache, as TMA boxes: a page (or 128 tokens of one) by 64 columns
//   warps 16-19     bring the others row by row with 16-byte asynchronous copies (rows that do not exist read as zeros): Q, the tile
//                   in which the cache ends and the tree begins, the tree, and caches whose pages do not tile 128 keys
// Tiles are 128-byte-swizzled either way.
//
// Two streams of softmax, 64 keys at a step, each with two score buffers, so that the scores of the next step are there when one
// is done and the products of the last step run meanwhile.  (With one buffer of 128 keys per stream neither the tensor cores, 43 %
// busy, nor the exponentials, 39 %, were the limit, but the way round.)  Units of more than 128 rows have a stream per 128
// rows, which take both halves of every tile of keys; in smaller ones each stream takes a half, and the two results are joined.
//
// What bounds it.  Up to 128 rows per key head, the keys' way from HBM: 131072 tokens of one sequence 110 to 120 us, 4.6 TB/s of
// 6.5; 16 sequences with 40 key heads and trees of 31 to 61 nodes 110 to 120 us, 3.6 TB/s (units of 10 tiles, whose ends nothing hides).
// With more rows the chain scores - softmax - products of a step and the power cap: 64 sequences, trees of 65 to 129 nodes,
// four query heads per key head 368 us from a cool start, 390 to 460 on and on (1.6 GHz), 0.55 of 1.63 PFLOP/s.  Few tiles:
// latency, 20 us for single tokens of 4 sequences, of which the second kernel is 4.
#include <limits.h>
#include <math.h>

#include <cuda_fp16.h>

#include "spec_common.cuh"
#include "tc_gemm.cuh"

namespace spec {

namespace {

using tc::ex2_approx;
using tc::mbar_arrive;
using tc::mbar_init;
using tc::smem_u32;
using tc::tc_fence_after;
using tc::tc_fence_before;
using tc::umma_commit;

constexpr int kTileKeys = 128;
constexpr int kTileRows = 128;
constexpr int kStepKeys = 64;
constexpr int kHalfBytes = kTileKeys * 128;     // 64 columns of a tile of 128 rows
constexpr int kSoftmaxThreads = 256;
constexpr int kMmaWarp = kSoftmaxThreads / 32, kBoxWarp = kMmaWarp + 4;        // the first of each
constexpr int kBoxWarps = 4;
constexpr int kLoadThreads = 128;
constexpr int kFirstLoader = 32 * (kBoxWarp + kBoxWarps);
constexpr int kThreads = kFirstLoader + kLoadThreads;
// A tile of K or V is complete after kBoxWarps arrivals of kLoadThreads each (TMA) or kLoadThreads of kBoxWarps each (copies).
constexpr int kTileArrivals = kBoxWarps * kLoadThreads;
// Registers of a thread after the roles have parted; 128 * (2 * 160 + 48 + 48 + 64) is what the launch has (640 threads of 96).  (All
// that the roles call is inlined: around a call the compiler does not go beyond the launch's 96.)  Spills cost more than warps
// bring: with 168 for the softmax and 48 for the rest the 13B trees took 132 us instead of 113.
constexpr int kSoftmaxRegs = 160, kMmaRegs = 48, kBoxRegs = 48, kRowRegs = 64;
static_assert(2 * kSoftmaxRegs + kMmaRegs + kBoxRegs + kRowRegs <= 5 * 96, "registers of the launch");
constexpr int kTmemCols = 512;                  // 128 columns each: the two buffers of S0, of S1, then O0, O1
constexpr int kUnitFlags = 8;
constexpr uint64_t kWaitMaxNs = 1000000000;     // after which a wait gives up
constexpr uint32_t kWaitHintNs = 20000;
constexpr float kRescaleAbove = 8.f;            // see softmax_step
// Probabilities are 2^kLift times what the maximum gives them.  In fp16, whose least number is 2^-24, those of less than 2^-25 of the
// maximum would become zero in the products but not in their sum (131071 keys 17.4 below one: 0.36 % of the result's weight lost);
// this way the border is 2^-32, and the greatest, 2^(kRescaleAbove + 7), is below 65504.
template <int kDtype>
constexpr float kLift = kDtype == SPEC_F16 ? 7.f : 0.f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

// Columns come in halves of 64: D <= 64 takes one, and twice the slots.
template <int kHalves>
struct Ring {
    static constexpr int kBytes = kHalves * kHalfBytes;
    static constexpr int kK = kHalves == 2 ? 3 : 6, kV = kHalves == 2 ? 2 : 5, kQ = 2;
};
constexpr int kMaxK = 6, kMaxV = 5;

// The cost of the whole call is dealt to `ctas` CTAs: CTA c has the tiles that begin in [start(c), start(c + 1)).  A unit costs
// unit_cost beside its tiles, behind its first one: what its end takes (a masked tile, results, a pipeline that empties) is time that
// no tile explains.  CTAs are as few as it takes for each to have a tile in every unit that its run meets.
// Costs of 0, 2, 3 and 4, us: 13B trees 135, 115, 110, 109; trees of 65 to 129 nodes, grouped heads, 447, 432, 393, 405; 32 short
// sequences of 40 heads 180, 130, 129, 127; 64 chains of 4 tokens, grouped heads, 133, 123, 125, 127; 256 single tokens 304, 274,
// 270, 270; one long context 112, 111, 111, 111.  With fewer than kManyTiles tiles a CTA it makes no difference (single
// tokens of 4 sequences 20.8 either way, 8 trees of 33 nodes 35.8 and 35.7).
constexpr int kUnitCost = 3;           // where CTAs have at least kManyTiles of cost each, else 0
constexpr int kManyTiles = 16;
struct Deal {
    long long cost;
    int ctas, unit_cost;
    __device__ long long start(int c) const {
        return (unsigned long long)cost < 0x1000000ull ? (unsigned)cost * (unsigned)c / (unsigned)ctas
                                                       : (unsigned long long)cost * (unsigned)c / (unsigned)ctas;
    }
    // whose is the tile that begins at `pos`
    __device__ int owner(long long pos) const {
        return (int)(((unsigned long long)(pos + 1) * (unsigned)ctas - 1) / (unsigned long long)cost);
    }
};

struct Shared {
    uint64_t q_full[2], q_empty[2], k_full[kMaxK], k_empty[kMaxK], v_full[kMaxV], v_empty[kMaxV];
    uint64_t s_full[2][2], p_full[2][2], pv_done[2][2], meet, drained, boxes_asked, rows_asked;
    uint32_t tmem_base;
    volatile int abort_flag;
    int ended[kBoxWarps];                       // what box_role returned
    volatile int not_finite[kUnitFlags];        // the unit's tree has values that are not finite (see finite_values)
    int start_b;
    long long start_off, left;
    Deal deal;
    float stat[2][kTileRows][2];                // running maximum and sum of the two streams
};
template <int kHalves>
constexpr int smem_bytes() {
    return (Ring<kHalves>::kK + Ring<kHalves>::kV + Ring<kHalves>::kQ) * Ring<kHalves>::kBytes + (int)sizeof(Shared);
}
static_assert(smem_bytes<2>() <= 232448 && smem_bytes<1>() <= 232448, "shared memory of an SM");

struct Join;
struct AttnArgs {
    spec_tree_attention_t a;
    int group;                // query heads per key head
    float scale_log2;         // |scale| log2(e)
    uint32_t desc_qk, desc_pv;
    float *part_out;          // [2 * CTAs][part_rows][D]
    float *part_lse;          // [2 * CTAs][part_rows]
    int part_rows;
    Join *joins;              // [CTAs]
    int max_len;              // of a sequence's cache
    int box_tokens;           // tokens of a TMA box, 0: the cache is not read by TMA (see cache_map)
    int box_pieces;           // kTileKeys / box_tokens
    CUtensorMap k_map, v_map; // the caches as (column, token, head, page)
};

// Waits are bounded by time.  A try sleeps in hardware until the phase ends or the hint has passed: warps that poll take the issue
// slots that the softmax needs.
__device__ __forceinline__ bool try_wait(uint64_t *bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity), "r"(kWaitHintNs) : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity, Shared *sh, int32_t *err) {
    if (try_wait(bar, parity)) return true;
    const uint64_t start = now_ns();
    while (!try_wait(bar, parity)) {
        if (sh->abort_flag) return false;
        if (now_ns() - start > kWaitMaxNs) {
            sh->abort_flag = 1;
            report_error(err, SPEC_ERR_TIMEOUT);
            return false;
        }
    }
    return true;
}
// The whole warp waits, leaves converged and with one verdict.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, Shared *sh, int32_t *err) {
    return __all_sync(0xffffffffu, wait(bar, parity, sh, err));
}

// ---- work ------------------------------------------------------------------------------------------------------------
struct Seq {
    int len, nodes, row_tiles, tiles;  // row_tiles: of 128 rows, per key head; tiles: of 128 keys
    __device__ long long head_cost(int unit_cost) const { return (long long)row_tiles * tiles + (row_tiles + 1) / 2 * unit_cost; }
};

__device__ __forceinline__ Seq seq_of(const AttnArgs &g, int b, bool report) {
    const spec_tree_attention_t &a = g.a;
    const int len = a.seq_len[b], nodes = a.n_nodes != nullptr ? a.n_nodes[b] : a.T;
    Seq s;
    s.len = min(max(len, 0), g.max_len);
    s.nodes = min(max(nodes, 0), a.T);
    if (report && (s.len != len || s.nodes != nodes)) report_error(a.err_word, SPEC_ERR_INDEX_RANGE);
    s.row_tiles = (s.nodes * g.group + kTileRows - 1) / kTileRows;
    s.tiles = (s.len + s.nodes + kTileKeys - 1) / kTileKeys;
    return s;
}

// Whole warp: the call's cost, and the sequence in which the part of CTA c begins with the offset in it (B: none).
__device__ Deal deal_out(const AttnArgs &g, int c, bool report, int &b_out, long long &off_out) {
    const int lane = threadIdx.x & 31;
    long long cost = 0, units = 0, mine = 0;
    for (int b = lane; b < g.a.B; b += 32) {
        const Seq s = seq_of(g, b, report);
        cost += g.a.Hkv * s.head_cost(0);
        if (s.tiles) units += g.a.Hkv * ((s.row_tiles + 1) / 2);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        cost += __shfl_xor_sync(0xffffffffu, cost, off);
        units += __shfl_xor_sync(0xffffffffu, units, off);
    }
    Deal d;
    d.unit_cost = cost >= (long long)kManyTiles * gridDim.x ? kUnitCost : 0;
    d.cost = cost = cost + units * d.unit_cost;
    const int apart = d.unit_cost + (g.a.T * g.group > kTileRows ? 2 : 1);       // the most between the begins of two tiles
    d.ctas = (int)min((long long)gridDim.x, cost > apart ? cost / apart : cost ? 1 : 0);
    b_out = g.a.B;
    off_out = 0;
    if (c >= d.ctas) return d;
    const long long pos = d.start(c);
    long long before = 0;
    for (int b0 = 0; b0 < g.a.B; b0 += 32) {
        const int b = b0 + lane;
        mine = b < g.a.B ? g.a.Hkv * seq_of(g, b, false).head_cost(d.unit_cost) : 0;
        long long upto = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += y;
        }
        upto += before;
        const unsigned hit = __ballot_sync(0xffffffffu, upto > pos);
        if (hit) {
            const int who = __ffs(hit) - 1;
            off_out = pos - __shfl_sync(0xffffffffu, upto - mine, who);
            b_out = b0 + who;
            return d;
        }
        before = __shfl_sync(0xffffffffu, upto, 31);
    }
    return d;
}

// A unit's tiles [t0, t1) that this CTA has.
struct Unit {
    int b, head, row0, rows;           // rows row0 .. row0 + rows - 1 of the head's nodes * group
    int len, nodes, tiles, t0, t1;
    int index;                         // counts the CTA's units
    long long begin;                   // in the cost of the call
    bool alone;                        // the head has no other rows
    __device__ bool two_tiles() const { return rows > kTileRows; }
    __device__ bool whole() const { return t0 == 0 && t1 == tiles; }
};

struct Walk {
    Seq s;
    int b, head, row_tile, index;      // row_tile: the unit's first
    int off, unit_cost;                // cost of the unit that is behind
    long long left, end;               // cost of this CTA that is ahead; where it ends
    __device__ Walk(const AttnArgs &g, const Shared *sh) {
        b = sh->start_b;
        left = sh->left;
        end = 0;
        index = head = row_tile = off = unit_cost = 0;
        s = {0, 0, 0, 0};
        if (b < g.a.B) {
            unit_cost = sh->deal.unit_cost;
            s = seq_of(g, b, false);
            const long long head_cost = s.head_cost(unit_cost);
            head = (int)(sh->start_off / head_cost);
            const long long in_head = sh->start_off - head * head_cost;
            const int pair_cost = 2 * s.tiles + unit_cost;               // of every unit of a head but the last
            row_tile = (int)(in_head / pair_cost) * 2;
            off = (int)(in_head - (long long)(row_tile / 2) * pair_cost);
            end = sh->deal.start(blockIdx.x + 1);
        }
    }
    // the tiles of a unit that begin before `upto` in it
    __device__ int tiles_before(int upto, int two) const {
        return upto <= 0 ? 0 : max(1, (upto - unit_cost + two) >> two);
    }
    __device__ bool next(const AttnArgs &g, Unit &u) {
        while (left > 0 && b < g.a.B) {
            if (row_tile >= s.row_tiles) {
                row_tile = 0;
                ++head;
            }
            if (head >= g.a.Hkv || s.row_tiles == 0) {
                head = 0;
                if (++b < g.a.B) s = seq_of(g, b, false);
                continue;
            }
            const int two = row_tile + 1 < s.row_tiles ? 1 : 0, cost = (s.tiles << two) + unit_cost;
            const int take = (int)min((long long)(cost - off), left);
            u.b = b;
            u.head = head;
            u.row0 = row_tile * kTileRows;
            u.rows = min(s.nodes * g.group - u.row0, 2 * kTileRows);
            u.len = s.len;
            u.nodes = s.nodes;
            u.tiles = s.tiles;
            u.t0 = tiles_before(off, two);
            u.t1 = tiles_before(off + take, two);
            u.begin = end - left - off;
            u.alone = s.row_tiles <= 2;
            left -= take;
            off += take;
            if (off == cost) {
                row_tile += 2;
                off = 0;
            }
            if (u.t0 == u.t1) continue;                  // what is left of a tile that begins in the CTA before
            u.index = index++;
            return true;
        }
        return false;
    }
};

// What block c of tree_combine_kernel joins: the unit whose first tiles, but not all, CTA c has.  rows 0: nothing.
struct __align__(16) Join {
    int b, head, row0, rows, parts, slot, pad[2];       // slot: of the first part; part i > 0 is in slot 2 (c + i)
};

// ---- loads -----------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void arrive_when_copied(uint64_t *bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A tile is 128 rows of 8 (D <= 64) or 16 chunks of 16 bytes: chunk c of row r lies at half c / 8, row pitch 128, column
// (c % 8) ^ (r % 8) of the row (the 128-byte swizzle of the MMA's descriptors).  A warp copies kRows rows at a time, in kPasses;
// lane l knows where row own_row() comes from and hands that to the lanes that copy it.
template <int kHalves>
struct TileMap {
    static constexpr int kChunks = 8 * kHalves, kRows = 32 / kChunks, kPasses = 32 / kRows, kStep = 4 * kRows;
    int warp, lane, chunk, row;        // row: of pass 0
    __device__ TileMap() {
        const int t = threadIdx.x - kFirstLoader;
        warp = t >> 5;
        lane = t & 31;
        chunk = lane % kChunks;
        row = warp * kRows + lane / kChunks;
    }
    __device__ int own_row() const { return lane / kRows * kStep + warp * kRows + lane % kRows; }
    // src: where own_row() starts, null: zeros.  cols: columns of a row in memory; the chunks up to a multiple of 16 are zeros.
    __device__ void copy(uint32_t tile, const uint16_t *src, int cols) const {
        const bool wanted = chunk * 8 < (cols + 15) / 16 * 16, there = chunk * 8 < cols;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const uint16_t *p = (const uint16_t *)__shfl_sync(0xffffffffu, (unsigned long long)src, i * kRows + lane / kChunks);
            const int r = row + i * kStep;
            const bool real = there && p != nullptr;
            if (wanted) copy16(address(tile, r), real ? p + chunk * 8 : nullptr, real);
        }
    }
    __device__ uint32_t address(uint32_t tile, int r) const {
        return tile + (chunk >> 3) * kHalfBytes + r * 128 + (((chunk & 7) ^ (r & 7)) << 4);
    }
};

// Where key `key` of a unit lies: page and token of the cache, or node of the tree.
struct KeyPlace {
    int page, token;                   // page -1: a node (token), -2: nothing
};
__device__ __forceinline__ KeyPlace key_place(const spec_tree_attention_t &a, const Unit &u, int key) {
    KeyPlace p = {-2, 0};
    if (key < u.len) {
        const int page = key / a.page_size, id = a.block_table[u.b * a.table_stride + page];
        if (id >= 0 && id < a.n_pages) p = {id, key - page * a.page_size};
        else report_error(a.err_word, SPEC_ERR_INDEX_RANGE);
    } else if (key < u.len + u.nodes) {
        p = {-1, key - u.len};
    }
    return p;
}
__device__ __forceinline__ const uint16_t *row_of(KeyPlace p, int b, int head, const void *cache, const int64_t *cs,
                                                  const void *tree, const int64_t *ts) {
    if (p.page >= 0) return (const uint16_t *)cache + p.page * cs[0] + p.token * cs[1] + head * cs[2];
    if (p.page == -1) return (const uint16_t *)tree + b * ts[0] + p.token * ts[1] + head * ts[2];
    return nullptr;
}

__device__ __forceinline__ void mbar_arrive_n(uint64_t *bar, int n) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(n) : "memory");
}
// Tiles [t0, boxed) of a unit lie in the cache and come by TMA.
__device__ __forceinline__ int boxed_tiles(const AttnArgs &g, const Unit &u) {
    return g.box_tokens ? min(u.t1, max(u.t0, u.len / kTileKeys)) : u.t0;
}

// The boxes of a tile are dealt to the warps: box i is piece i / kHalves of 128 / box_tokens, columns 64 * (i % kHalves).  Lane l
// of a warp looks up the page of the warp's box l, a tile ahead.  Nothing here divides but where a page holds several tiles:
// with a division per box and lookups that the copies wait for, four warps brought in 2.8 TB/s.
constexpr int kMaxBoxes = (32 + kBoxWarps - 1) / kBoxWarps;              // of a warp: pages of 8 tokens, two halves
template <int kHalves>
__device__ __forceinline__ int box_page(const AttnArgs &g, const Unit &u, int tile, int warp, int lane) {
    const spec_tree_attention_t &a = g.a;
    const int piece = (warp + kBoxWarps * lane) / kHalves;
    if (piece >= g.box_pieces) return 0;
    const int index = a.page_size > kTileKeys ? tile / (a.page_size / kTileKeys) : tile * g.box_pieces + piece;
    const int id = a.block_table[u.b * a.table_stride + index];
    if (id >= 0 && id < a.n_pages) return id;
    report_error(a.err_word, SPEC_ERR_INDEX_RANGE);
    return a.n_pages;                                    // behind the tensor: the box reads as zeros
}
template <int kHalves>
__device__ __forceinline__ void load_boxes(const AttnArgs &g, const CUtensorMap *map, const Unit &u, int tile, int page, int warp,
                                           uint32_t dst, uint64_t *bar, uint64_t policy) {
    const int boxes = g.box_pieces * kHalves, bytes = g.box_tokens * 128;
    const int token = g.a.page_size > kTileKeys ? tile % (g.a.page_size / kTileKeys) * kTileKeys : 0;
    int id[kMaxBoxes];
#pragma unroll
    for (int i = 0; i < kMaxBoxes; ++i) id[i] = __shfl_sync(0xffffffffu, page, i);
    if (tc::elect_one()) {
        int arrivals = kLoadThreads;
        if (warp < boxes) {
            tc::mbar_arrive_expect_tx(bar, (boxes - warp + kBoxWarps - 1) / kBoxWarps * bytes);
            --arrivals;
        }
        mbar_arrive_n(bar, arrivals);
#pragma unroll
        for (int i = 0; i < kMaxBoxes; ++i) {
            const int box = warp + kBoxWarps * i, piece = box / kHalves, half = box % kHalves;
            if (box >= boxes) break;
            asm volatile(
                "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint "
                "[%0], [%1, {%2, %3, %4, %5}], [%6], %7;"
                ::"r"(dst + half * kHalfBytes + piece * bytes), "l"((uint64_t)map), "r"(half * 64), "r"(token), "r"(u.head),
                "r"(id[i]), "r"(smem_u32(bar)), "l"(policy) : "memory");
        }
    }
    __syncwarp();
}

// K of a tile goes ahead of V of the tile before.  Every tile of a unit takes the next slot, whoever fills it, so a role passes over
// the slots that the other one fills.  A barrier's parity tells its phases apart only for those that are at most one phase away
// from it: row_role turns to the last tiles of a unit when box_role has asked for those before them (boxes_asked), and box_role to
// the next unit when row_role has a slot for each of the last ones (rows_asked).
template <int kSlots>
__device__ __forceinline__ void pass_over(int n, int &slot, uint32_t &parity) {
    slot += n;
    parity ^= (slot / kSlots) & 1;
    slot %= kSlots;
}

// Returns where the warp has ended: the slots and parities that would have been next.
__device__ __forceinline__ int pack_end(int ks, uint32_t kp, int vs, uint32_t vp) { return ks | vs << 8 | (int)(kp << 16 | vp << 17); }

template <int kHalves>
__device__ int box_role(const AttnArgs &g, Shared *sh, uint32_t k_tiles, uint32_t v_tiles) {
    using R = Ring<kHalves>;
    const int warp = (threadIdx.x >> 5) - kBoxWarp, lane = threadIdx.x & 31;
    int ks = 0, vs = 0;                                  // slots, and the parity of their `empty` that means free
    uint32_t kp = 1, vp = 1, rows_parity = 0;
    uint64_t once = tc::evict_first_policy(), normal;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(normal));
    Walk walk(g, sh);
    Unit u;
    while (walk.next(g, u)) {
        // keys that no other rows of the head read leave L2 first: 13B trees 120.3 -> 118.9 us, 131072 tokens 117.7 -> 116.3 (keeping
        // those that are read again with priority gains nothing: more than L2 holds comes in between)
        const uint64_t policy = u.alone ? once : normal;
        const int boxed = boxed_tiles(g, u);
        int page = u.t0 < boxed ? box_page<kHalves>(g, u, u.t0, warp, lane) : 0, before = 0;
        for (int t = u.t0; t <= boxed; ++t) {
            const int now = page;
            if (t < boxed) {
                if (t + 1 < boxed) page = box_page<kHalves>(g, u, t + 1, warp, lane);   // (ahead of the wait)
                if (!warp_wait(&sh->k_empty[ks], kp, sh, g.a.err_word)) return pack_end(ks, kp, vs, vp);
                load_boxes<kHalves>(g, &g.k_map, u, t, now, warp, k_tiles + ks * R::kBytes, &sh->k_full[ks], policy);
                pass_over<R::kK>(1, ks, kp);
            } else if (boxed < u.t1 && lane == 0) {
                mbar_arrive(&sh->boxes_asked);
            }
            if (t > u.t0) {
                if (!warp_wait(&sh->v_empty[vs], vp, sh, g.a.err_word)) return pack_end(ks, kp, vs, vp);
                load_boxes<kHalves>(g, &g.v_map, u, t - 1, before, warp, v_tiles + vs * R::kBytes, &sh->v_full[vs], policy);
                pass_over<R::kV>(1, vs, vp);
            }
            before = now;
        }
        if (boxed < u.t1) {
            if (!warp_wait(&sh->rows_asked, rows_parity, sh, g.a.err_word)) return pack_end(ks, kp, vs, vp);
            rows_parity ^= 1;
            pass_over<R::kK>(u.t1 - boxed, ks, kp);
            pass_over<R::kV>(u.t1 - boxed, vs, vp);
        }
    }
    return pack_end(ks, kp, vs, vp);
}

// A wait has run out somewhere in the CTA: boxes that are still on their way would land in shared memory that is somebody else's by
// then.  Whole warp, a lane per slot: the last fill that the warp knows of belongs to the round before the next one's or, in slots
// before that one, to the same (one that was never filled is free at once).  Bounded like the other waits: a tile that some warps
// did not come to ask for never completes its phase.
template <int kHalves>
__device__ void await_boxes(Shared *sh) {
    using R = Ring<kHalves>;
    const int lane = threadIdx.x & 31, end = sh->ended[(threadIdx.x >> 5) - kBoxWarp];
    const bool of_k = lane < R::kK;
    const int slot = of_k ? lane : lane - R::kK, next = of_k ? end & 0xff : end >> 8 & 0xff;
    const uint32_t parity = (end >> (of_k ? 16 : 17) & 1) ^ (slot < next ? 1 : 0);
    if (of_k || slot < R::kV)
        for (const uint64_t start = now_ns();
             !try_wait(of_k ? &sh->k_full[slot] : &sh->v_full[slot], parity) && now_ns() - start < kWaitMaxNs;) {}
    __syncwarp();
}

// Rows of the tree in a tile of V.  Not every query sees them, and 0 * inf would reach those that do not: what is not finite becomes zero
// in the tile, and the rows that do see it take it from memory (add_not_finite).  Every thread looks at the chunks that it
// copied itself, after they have arrived and before it says so.
template <int kDtype, int kHalves>
__device__ __forceinline__ bool finite_values(const TileMap<kHalves> &map, uint32_t tile, int first, int end, int cols) {
    constexpr uint32_t kExp = kDtype == SPEC_BF16 ? 0x7f80u : 0x7c00u;       // eight or five exponent bits
    bool bad = false;
    if (map.chunk * 8 < cols) {
#pragma unroll 4
        for (int i = 0; i < TileMap<kHalves>::kPasses; ++i) {
            const int r = map.row + i * TileMap<kHalves>::kStep;
            const uint32_t at = map.address(tile, r);
            uint32_t x[4];
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(at) : "memory");
            bool found = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) found |= (x[e] & kExp) == kExp || (x[e] >> 16 & kExp) == kExp;
            if (found && r >= first && r < end) {
                bad = true;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] &= ((x[e] & kExp) == kExp ? 0u : 0x0000ffffu) | ((x[e] >> 16 & kExp) == kExp ? 0u : 0xffff0000u);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
            }
        }
    }
    return !bad;
}

template <int kDtype, int kHalves>
__device__ void row_role(const AttnArgs &g, Shared *sh, uint32_t q_tiles, uint32_t k_tiles, uint32_t v_tiles) {
    using R = Ring<kHalves>;
    const spec_tree_attention_t &a = g.a;
    const TileMap<kHalves> map;
    int qs = 0, ks = 0, vs = 0;
    uint32_t qp = 1, kp = 1, vp = 1, boxes_parity = 0;
    auto arrive_all_copied = [](uint64_t *bar) {
#pragma unroll
        for (int i = 0; i < kBoxWarps; ++i) arrive_when_copied(bar);
    };
    Walk walk(g, sh);
    Unit u;
    while (walk.next(g, u)) {
        for (int i = 0; i < (u.two_tiles() ? 2 : 1); ++i) {
            if (!warp_wait(&sh->q_empty[qs], qp, sh, a.err_word)) return;
            const int r = i * kTileRows + map.own_row(), node = (u.row0 + r) / g.group;
            const uint16_t *src = nullptr;
            if (r < u.rows)
                src = (const uint16_t *)a.q + u.b * a.q_stride[0] + node * a.q_stride[1] +
                      (u.head * g.group + u.row0 + r - node * g.group) * a.q_stride[2];
            map.copy(q_tiles + qs * R::kBytes, src, a.D);
            arrive_when_copied(&sh->q_full[qs]);
            if (++qs == R::kQ) qs = 0, qp ^= 1;
        }
        const int boxed = boxed_tiles(g, u);
        pass_over<R::kK>(boxed - u.t0, ks, kp);
        pass_over<R::kV>(boxed - u.t0, vs, vp);
        if (boxed == u.t1) continue;
        KeyPlace here = key_place(a, u, boxed * kTileKeys + map.own_row()), before = {};
        if (!warp_wait(&sh->boxes_asked, boxes_parity, sh, a.err_word)) return;
        boxes_parity ^= 1;
        for (int t = boxed; t <= u.t1; ++t) {
            const KeyPlace now = here;
            if (t < u.t1) {
                if (t + 1 < u.t1) here = key_place(a, u, (t + 1) * kTileKeys + map.own_row());
                if (!warp_wait(&sh->k_empty[ks], kp, sh, a.err_word)) return;
                map.copy(k_tiles + ks * R::kBytes, row_of(now, u.b, u.head, a.k_cache, a.kc_stride, a.k, a.k_stride), a.D);
                arrive_all_copied(&sh->k_full[ks]);
                pass_over<R::kK>(1, ks, kp);
            }
            if (t > boxed) {
                if (!warp_wait(&sh->v_empty[vs], vp, sh, a.err_word)) return;
                if (t == u.t1 && map.lane == 0) mbar_arrive(&sh->rows_asked);
                const uint32_t tile = v_tiles + vs * R::kBytes;
                map.copy(tile, row_of(before, u.b, u.head, a.v_cache, a.vc_stride, a.v, a.v_stride), a.D);
                const int tree = u.len - (t - 1) * kTileKeys;            // the tree's first row
                if (tree < kTileKeys) {
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    if (!finite_values<kDtype>(map, tile, tree, tree + u.nodes, a.D)) sh->not_finite[u.index % kUnitFlags] = 1;
                    fence_async_proxy();
                    mbar_arrive_n(&sh->v_full[vs], kBoxWarps);
                } else {
                    arrive_all_copied(&sh->v_full[vs]);
                }
                pass_over<R::kV>(1, vs, vp);
            }
            before = now;
        }
    }
}

// ---- MMAs ------------------------------------------------------------------------------------------------------------
// Descriptors: 128-byte swizzle.  Q and K are K-major (rows of 128 bytes, groups of 8 rows 1024 bytes apart).  V is MN-major: 64
// columns of a key are contiguous, 8 keys make a 1024-byte group, the next 64 columns are kHalfBytes away.
__device__ __forceinline__ uint64_t v_desc(uint32_t saddr) {
    return tc::make_smem_desc(saddr) | (uint64_t)(kHalfBytes >> 4) << 16;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t desc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(desc), "r"((uint32_t)add) : "memory");
}

template <int kHalves>
__device__ bool mma_role(const AttnArgs &g, Shared *sh, int stream, uint32_t q_tiles, uint32_t k_tiles, uint32_t v_tiles) {
    using R = Ring<kHalves>;
    int32_t *err = g.a.err_word;
    const uint32_t s_cols = sh->tmem_base + stream * 128, o_cols = sh->tmem_base + 256 + stream * 128;
    const uint32_t desc_qk = g.desc_qk, desc_pv = g.desc_pv;
    const int k_steps = (g.a.D + 15) / 16;
    int qs = 0, ks = 0, vs = 0;
    uint32_t qp = 0, kp = 0, vp = 0;
    uint32_t count = 0;                                  // steps of the stream in the units before; buffers go by it
    Walk walk(g, sh);
    Unit u;
    while (walk.next(g, u)) {
        // two: step i is half i & 1 of tile i / 2; else half `stream` of tile i
        const bool two = u.two_tiles();
        const int steps = (u.t1 - u.t0) * (two ? 2 : 1), boxed = boxed_tiles(g, u) - u.t0;
        const int q = two && stream ? qs ^ 1 : qs;       // the stream's query tile
        const uint32_t q_parity = two && stream && qs == 1 ? qp ^ 1 : qp;
        if (!two) {
            if (++qs == R::kQ) qs = 0, qp ^= 1;
        } else {
            qp ^= 1;
        }
        const uint64_t qd = tc::make_smem_desc(q_tiles + q * R::kBytes);
        auto scores = [&](int i) -> bool {
            const int half = two ? i & 1 : stream;
            const uint32_t buf = (count + i) & 1;
            if (i == 0 && !wait(&sh->q_full[q], q_parity, sh, err)) return false;
            if (!wait(&sh->k_full[ks], kp, sh, err)) return false;
            if (i == 0 || (two ? i >> 1 : i) >= boxed) fence_async_proxy();      // Q and such tiles are written by ordinary copies
            // (Unrolled, with descriptors that differ by constants: a loop that builds them took 140 cycles an MMA, twice its time.)
            const uint64_t kd = tc::make_smem_desc(k_tiles + ks * R::kBytes + half * kStepKeys * 128);
            const uint32_t d = s_cols + buf * 64;
#pragma unroll
            for (int n = 0; n < 4 * kHalves; ++n) {
                constexpr int kHalf = kHalfBytes >> 4;
                const int off = (n >> 2) * kHalf + (n & 3) * 2;
                if (n < k_steps) mma_ss(d, qd + off, kd + off, desc_qk, n > 0);
            }
            umma_commit(&sh->s_full[stream][buf]);
            if (!two || half) {
                umma_commit(&sh->k_empty[ks]);
                if (++ks == R::kK) ks = 0, kp ^= 1;
            }
            if (i == steps - 1) {                        // a slot of Q is free when both streams say so
                umma_commit(&sh->q_empty[q]);
                if (two) umma_commit(&sh->q_empty[q ^ 1]);
            }
            return true;
        };
        if (!scores(0) || (steps > 1 && !scores(1))) return false;
        for (int i = 0; i < steps; ++i) {
            const int half = two ? i & 1 : stream;
            const uint32_t at = count + i, buf = at & 1;
            if (!wait(&sh->v_full[vs], vp, sh, err)) return false;
            if ((two ? i >> 1 : i) >= boxed) fence_async_proxy();
            if (!wait(&sh->p_full[stream][buf], at >> 1 & 1, sh, err)) return false;
            tc_fence_after();
            const uint64_t vd = v_desc(v_tiles + vs * R::kBytes + half * kStepKeys * 128);
            const uint32_t pa = s_cols + buf * 64;
#pragma unroll
            for (int n = 0; n < kStepKeys / 16; ++n) mma_ts(o_cols, pa + n * 8, vd + n * (2048 >> 4), desc_pv, i > 0 || n > 0);
            umma_commit(&sh->pv_done[stream][buf]);
            if (!two || half) {
                umma_commit(&sh->v_empty[vs]);
                if (++vs == R::kV) vs = 0, vp ^= 1;
            }
            if (i + 2 < steps && !scores(i + 2)) return false;
        }
        count += steps;
    }
    return true;
}

// ---- softmax ---------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <int kDtype>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    if (kDtype == SPEC_BF16) return pack_bf16x2(lo, hi);
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int kDtype>
__device__ __forceinline__ float number(uint32_t x, int which) {
    if (kDtype == SPEC_BF16) return __uint_as_float(which ? x & 0xffff0000u : x << 16);
    return __half2float(__ushort_as_half((unsigned short)(which ? x >> 16 : x & 0xffffu)));
}

// Which of the 32 keys from `first - len` on (in nodes of the tree; negative: the cache) the row of `node` sees.
struct RowMask {
    const uint32_t *words;             // null: a chain
    int n_words, nodes, node;
    __device__ uint32_t word(int i) const { return i < 0 ? 0xffffffffu : i < n_words ? words[i] : 0u; }
    __device__ uint32_t bits(int first) const {
        uint32_t m = 0xffffffffu;
        int end = nodes;
        if (words != nullptr) m = __funnelshift_r(word(first >> 5), word((first >> 5) + 1), first & 31);
        else end = min(nodes, node + 1);
        const int keep = end - first;
        return keep >= 32 ? m : keep <= 0 ? 0u : m & ((1u << keep) - 1);
    }
};

struct Row {
    float top;                         // running maximum (times scale log2 e) that exponents are taken against
    float sum;
};

__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, float *v, int at) {
#define V(i) "=f"(v[at + i])
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : V(0), V(1), V(2), V(3), V(4), V(5), V(6), V(7), V(8), V(9), V(10), V(11), V(12), V(13), V(14), V(15), V(16), V(17),
          V(18), V(19), V(20), V(21), V(22), V(23), V(24), V(25), V(26), V(27), V(28), V(29), V(30), V(31)
        : "r"(taddr) : "memory");
#undef V
}
// Nothing may use a register before the wait, so each passes through a statement behind it.
template <int kN>
__device__ __forceinline__ void tmem_ld_wait(float (&v)[kN]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int c = 0; c < kN; c += 8)
        asm volatile("" : "+f"(v[c]), "+f"(v[c + 1]), "+f"(v[c + 2]), "+f"(v[c + 3]), "+f"(v[c + 4]), "+f"(v[c + 5]), "+f"(v[c + 6]),
                          "+f"(v[c + 7]));
}

// Two lanes of fp32 arithmetic in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(r)
        : "l"(*(unsigned long long *)&a), "l"(*(unsigned long long *)&b), "l"(*(unsigned long long *)&c));
    return *(float2 *)&r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*(unsigned long long *)&a), "l"(*(unsigned long long *)&b));
    return *(float2 *)&r;
}

// One step of a row: probabilities in place of the scores.  The maximum follows the steps lazily: probabilities are taken against an
// older one as long as none exceeds 2^8 of it, which costs no precision in fp32 sums nor in the 16-bit probabilities and
// saves nearly every pass over the accumulated output (a pass waits for the products of the step before).  The probabilities are
// rounded to the 16 bits that the tensor cores take beside the values, each by half a step at most (in fp16 by 2^-32 of the
// greatest if that is more: see kLift); their sum is not.
template <int kDtype, int kHalves>
__device__ __forceinline__ bool softmax_step(const AttnArgs &g, Shared *sh, uint32_t s_addr, uint32_t o_addr, bool first,
                                             uint64_t *pv_done, uint32_t pv_parity, bool masked, uint64_t seen, Row &row) {
    float x[kStepKeys];
    tmem_ld32_async(s_addr, x, 0);
    tmem_ld32_async(s_addr + 32, x, 32);
    tmem_ld_wait(x);
    if (masked) {
#pragma unroll
        for (int i = 0; i < kStepKeys; ++i)
            if (!(seen >> i & 1)) x[i] = -INFINITY;
    }
    float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < kStepKeys; i += 2) top4[i / 2 % 4] = fmaxf(fmaxf(x[i], x[i + 1]), top4[i / 2 % 4]);
    float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
    top = top == -INFINITY ? top : top * g.scale_log2;
    float shrink = 1.f;
    if (first) {
        row.top = top;
    } else if (top > row.top + kRescaleAbove) {
        shrink = ex2_approx(row.top - top);
        row.top = top;
    }
    if (__any_sync(0xffffffffu, shrink != 1.f)) {
        if (!warp_wait(pv_done, pv_parity, sh, g.a.err_word)) return false;
        tc_fence_after();
        row.sum *= shrink;
#pragma unroll 1
        for (int c = 0; c < 4 * kHalves; ++c) {
            float o[16];
            uint32_t r[16];
            tc::tmem_ld16(o_addr + c * 16, o);
#pragma unroll
            for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(o[i] * shrink);
            tmem_st16(o_addr + c * 16, r);
        }
    }
    const float base = row.top == -INFINITY ? 0.f : row.top - kLift<kDtype>;
    const float2 scale = make_float2(g.scale_log2, g.scale_log2), minus = make_float2(-base, -base);
    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
    for (int c = 0; c < kStepKeys / 32; ++c) {
        uint32_t p[16];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            float2 y = fma2(make_float2(x[c * 32 + i], x[c * 32 + i + 1]), scale, minus);
            y.x = ex2_approx(y.x);
            y.y = ex2_approx(y.y);
            sum[i / 2 % 2] = add2(sum[i / 2 % 2], y);
            p[i / 2] = pack2<kDtype>(y.x, y.y);
        }
        tmem_st16(s_addr + c * 16, p);
    }
    sum[0] = add2(sum[0], sum[1]);
    row.sum += sum[0].x + sum[0].y;
    tmem_wait_st();
    return true;
}

// What finite_values kept out of the products: values that are not finite, of the nodes that the row sees, are added to the row's
// result in memory, which its own thread has just written (columns col0 .. col0 + 31).
template <int kDtype>
__device__ __forceinline__ void add_not_finite(const spec_tree_attention_t &a, const Unit &u, const RowMask &mask, int col0,
                                            uint16_t *out, float *part) {
    const int first = max(u.t0 * kTileKeys - u.len, 0), end = min(u.t1 * kTileKeys - u.len, u.nodes);
    for (int n = first; n < end; ++n) {
        if (!(mask.bits(n) & 1)) continue;
        const uint16_t *v = (const uint16_t *)a.v + u.b * a.v_stride[0] + n * a.v_stride[1] + u.head * a.v_stride[2];
        for (int i = col0; i < min(col0 + 32, a.D); ++i) {
            const float x = number<kDtype>(v[i], 0);
            if (fabsf(x) < INFINITY) continue;
            if (part != nullptr) part[i] += x;
            else out[i] = (uint16_t)pack2<kDtype>(number<kDtype>(out[i], 0) + x, 0.f);
        }
    }
}

// A barrier of the softmax threads whose wait is bounded like the others.
__device__ __forceinline__ bool softmax_meet(Shared *sh, uint32_t &parity, int32_t *err) {
    tc_fence_before();
    mbar_arrive(&sh->meet);
    if (!warp_wait(&sh->meet, parity, sh, err)) return false;
    tc_fence_after();
    parity ^= 1;
    return true;
}

template <int kDtype, int kHalves>
__device__ bool softmax_role(const AttnArgs &g, Shared *sh) {
    const spec_tree_attention_t &a = g.a;
    const int stream = threadIdx.x >> 7, lane_row = threadIdx.x & 127;
    const uint32_t lanes = sh->tmem_base + ((uint32_t)(lane_row & ~31) << 16);
    uint32_t count = 0, meet = 0;                        // steps of this stream over all units; parity
    Walk walk(g, sh);
    Unit u;
    while (walk.next(g, u)) {
        const bool two = u.two_tiles();
        const int r = two ? stream * kTileRows + lane_row : lane_row;
        const bool active = (r & ~31) < u.rows;          // of the warp
        const int node = (u.row0 + min(r, u.rows - 1)) / g.group, head = u.row0 + r - node * g.group;
        const int n_words = (a.T + 31) / 32;
        const RowMask mask = {a.mask == nullptr ? nullptr : a.mask + ((size_t)u.b * a.T + node) * n_words, n_words, u.nodes, node};
        Row row = {-INFINITY, 0.f};
        bool first = true;
        for (int key = u.t0 * kTileKeys + (two ? 0 : stream * kStepKeys); key < u.t1 * kTileKeys; key += two ? kStepKeys : kTileKeys) {
            const uint32_t buf = count & 1;
            const int key0 = key - u.len;
            const bool masked = key0 + kStepKeys > 0;
            uint64_t seen = 0;
            if (masked) seen = (uint64_t)mask.bits(key0 + 32) << 32 | mask.bits(key0);
            if (!warp_wait(&sh->s_full[stream][buf], count >> 1 & 1, sh, a.err_word)) return false;
            tc_fence_after();
            if (active && !softmax_step<kDtype, kHalves>(g, sh, lanes + stream * 128 + buf * 64, lanes + 256 + stream * 128, first,
                                                         &sh->pv_done[stream][buf ^ 1], (count - 1) >> 1 & 1, masked, seen, row))
                return false;
            first = false;
            tc_fence_before();
            mbar_arrive(&sh->p_full[stream][buf]);
            ++count;
        }
        // (A buffer's products are done when its next scores are there, so that this phase is the current one or the last.)
        if (!warp_wait(&sh->pv_done[stream][(count - 1) & 1], (count - 1) >> 1 & 1, sh, a.err_word)) return false;
        row.top -= kLift<kDtype>;                        // what the exponents were taken against
        // the two streams of one query tile are joined: each warp group takes every other 32 columns
        float w[2] = {1.f, 0.f};
        if (!two) {
            sh->stat[stream][lane_row][0] = row.top;
            sh->stat[stream][lane_row][1] = row.sum;
            if (!softmax_meet(sh, meet, a.err_word)) return false;
            const float top0 = sh->stat[0][lane_row][0], top1 = sh->stat[1][lane_row][0];
            const float top = fmaxf(top0, top1), base = top == -INFINITY ? 0.f : top;
            w[0] = ex2_approx(top0 - base);
            w[1] = ex2_approx(top1 - base);
            row.top = top;
            row.sum = sh->stat[0][lane_row][1] * w[0] + sh->stat[1][lane_row][1] * w[1];
        }
        tc_fence_after();
        const bool bad = sh->not_finite[u.index % kUnitFlags] != 0;
        if (active) {
            const float inv = row.sum == 0.f ? 0.f : 1.f / row.sum;
            const float lse = row.sum == 0.f ? -INFINITY : row.top * kLn2 + logf(row.sum);
            uint16_t *out = (uint16_t *)a.out + u.b * a.out_stride[0] + node * a.out_stride[1] +
                            (u.head * g.group + head) * a.out_stride[2];
            const size_t part = ((size_t)(2 * blockIdx.x + (u.index ? 1 : 0))) * g.part_rows + r;
            float *part_out = g.part_out + part * a.D;
            const bool whole = u.whole();
            w[0] *= inv;
            w[1] *= inv;
            // 32 columns at a time, of both streams, behind one wait: a load of TMEM takes several hundred cycles while MMAs run
#pragma unroll 1
            for (int c = two ? 0 : stream * 32; c < a.D; c += two ? 32 : 64) {
                float o[64];
                tmem_ld32_async(lanes + 256 + (two ? stream * 128 : 0) + c, o, 0);
                tmem_ld32_async(lanes + 384 + c, o, 32);
                tmem_ld_wait(o);
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = !two ? fmaf(o[32 + i], w[1], o[i] * w[0]) : o[i] * w[0];
                if (r < u.rows) {
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        if (c + i >= a.D) continue;
                        if (whole) {
                            uint4 y;
                            y.x = pack2<kDtype>(o[i], o[i + 1]);
                            y.y = pack2<kDtype>(o[i + 2], o[i + 3]);
                            y.z = pack2<kDtype>(o[i + 4], o[i + 5]);
                            y.w = pack2<kDtype>(o[i + 6], o[i + 7]);
                            *(uint4 *)(out + c + i) = y;
                        } else {
                            *(float4 *)(part_out + c + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                            *(float4 *)(part_out + c + i + 4) = make_float4(o[i + 4], o[i + 5], o[i + 6], o[i + 7]);
                        }
                    }
                    if (bad) add_not_finite<kDtype>(a, u, mask, c, out, whole ? nullptr : part_out);
                }
                __syncwarp();
            }
            if (r < u.rows && (two || stream == 0)) {
                if (!u.whole()) g.part_lse[part] = lse;
                else if (a.lse != nullptr) a.lse[((size_t)u.b * a.T + node) * a.Hq + u.head * g.group + head] = lse;
            }
        }
        if (!softmax_meet(sh, meet, a.err_word)) return false;       // nobody writes O, stat or the flag while somebody may still read them
        if (threadIdx.x == 0) {
            sh->not_finite[u.index % kUnitFlags] = 0;
            // where its last tile begins
            const long long last = u.begin + (u.tiles == 1 ? 0 : sh->deal.unit_cost + ((long long)(u.tiles - 1) << (two ? 1 : 0)));
            if (u.t0 == 0 && !u.whole())
                g.joins[blockIdx.x] = {u.b, u.head, u.row0, u.rows,
                                       sh->deal.owner(last) - (int)blockIdx.x + 1,
                                       2 * (int)blockIdx.x + (u.index ? 1 : 0), {}};
        }
    }
    return true;
}

template <int kDtype, int kHalves>
__global__ void __launch_bounds__(kThreads, 1) tree_attention_kernel(const __grid_constant__ AttnArgs g) {
    extern __shared__ __align__(1024) uint8_t smem[];
    using R = Ring<kHalves>;
    const uint32_t q_tiles = smem_u32(smem), k_tiles = q_tiles + R::kQ * R::kBytes, v_tiles = k_tiles + R::kK * R::kBytes;
    Shared *sh = (Shared *)(smem + (R::kQ + R::kK + R::kV) * R::kBytes);
    const int warp = threadIdx.x >> 5;
    griddep_launch();
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh->q_full[i], kLoadThreads);
            mbar_init(&sh->q_empty[i], 2);
            for (int j = 0; j < 2; ++j) {
                mbar_init(&sh->s_full[i][j], 1);
                mbar_init(&sh->p_full[i][j], kTileRows);
                mbar_init(&sh->pv_done[i][j], 1);
            }
        }
        for (int i = 0; i < R::kK; ++i) {
            mbar_init(&sh->k_full[i], kTileArrivals);
            mbar_init(&sh->k_empty[i], 2);
        }
        for (int i = 0; i < R::kV; ++i) {
            mbar_init(&sh->v_full[i], kTileArrivals);
            mbar_init(&sh->v_empty[i], 2);
        }
        mbar_init(&sh->meet, kSoftmaxThreads);
        mbar_init(&sh->drained, 2);
        mbar_init(&sh->boxes_asked, kBoxWarps);
        mbar_init(&sh->rows_asked, kLoadThreads / 32);
        sh->abort_flag = 0;
        for (int i = 0; i < kUnitFlags; ++i) sh->not_finite[i] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_proxy();
    }
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)),
                     "r"((uint32_t)kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    griddep_wait();
    if (warp == 1) {
        int b;
        long long off;
        const Deal d = deal_out(g, blockIdx.x, blockIdx.x == 0, b, off);
        if ((threadIdx.x & 31) == 0) {
            sh->start_b = b;
            sh->start_off = off;
            sh->left = (int)blockIdx.x < d.ctas ? d.start(blockIdx.x + 1) - d.start(blockIdx.x) : 0;
            sh->deal = d;
            g.joins[blockIdx.x] = Join{};                // (softmax_role writes what there is to join)
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        softmax_role<kDtype, kHalves>(g, sh);
    } else if (warp < kBoxWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kMmaRegs));
        if (warp < kMmaWarp + 2 && tc::elect_one()) {
            mma_role<kHalves>(g, sh, warp - kMmaWarp, q_tiles, k_tiles, v_tiles);
            umma_commit(&sh->drained);                   // what was issued ends before TMEM and shared memory go
            for (const uint64_t start = now_ns(); !try_wait(&sh->drained, 0) && now_ns() - start < kWaitMaxNs;) {}
        }
        __syncwarp();
    } else if (warp < kBoxWarp + kBoxWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kBoxRegs));
        const int end = box_role<kHalves>(g, sh, k_tiles, v_tiles);
        if ((threadIdx.x & 31) == 0) sh->ended[warp - kBoxWarp] = end;
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRowRegs));
        row_role<kDtype, kHalves>(g, sh, q_tiles, k_tiles, v_tiles);
        asm volatile("cp.async.wait_all;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (sh->abort_flag) {                    // (nobody sets it any more)
        if (warp >= kBoxWarp && warp < kBoxWarp + kBoxWarps) await_boxes<kHalves>(sh);
        __syncthreads();
    }
    if (warp == 8) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sh->tmem_base), "r"((uint32_t)kTmemCols) : "memory");
    }
}

// ---- joining the parts of a unit -------------------------------------------------------------------------------------
// Block c joins the unit that CTA c began and others ended, if there is one: CTA c left it in joins[c].  blockIdx.y takes
// kJoinRows of its rows, a warp per row; a row's weights are worked out by its warp, and its sums have the loads of eight parts in
// flight.
constexpr int kJoinRows = 8;
constexpr int kJoinThreads = 32 * kJoinRows;
constexpr int kMaxCtas = 256;

template <int kDtype>
__global__ void __launch_bounds__(kJoinThreads) tree_combine_kernel(const __grid_constant__ AttnArgs g) {
    __shared__ float weight[kJoinRows][kMaxCtas];
    const spec_tree_attention_t &a = g.a;
    griddep_launch();
    griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x;
    const Join j = g.joins[c];
    const int b = j.b, head = j.head, row0 = j.row0, n = j.parts, r = blockIdx.y * kJoinRows + warp;
    if (r >= j.rows) return;
    // part i's rows
    auto place = [&](int i) { return (size_t)(i ? 2 * (c + i) : j.slot) * g.part_rows + r; };
    float top = -INFINITY, sum = 0.f;
    for (int i = lane; i < n; i += 32) {
        const float lse = g.part_lse[place(i)];
        weight[warp][i] = lse;
        top = fmaxf(top, lse);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    for (int i = lane; i < n; i += 32) {
        const float lse = weight[warp][i], w = lse == -INFINITY ? 0.f : __expf(lse - top);
        // (a part whose weight is nothing still carries what is not finite; one without a key carries nothing)
        weight[warp][i] = lse == -INFINITY ? -1.f : w;
        sum += w;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncwarp();
    const int col = lane * 4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (col < a.D) {
#pragma unroll 8
        for (int i = 0; i < n; ++i) {
            const float4 o = *(const float4 *)(g.part_out + place(i) * a.D + col);
            const float w = weight[warp][i];
            if (w < 0.f) continue;
            acc.x += fabsf(o.x) < INFINITY ? o.x * w : o.x;
            acc.y += fabsf(o.y) < INFINITY ? o.y * w : o.y;
            acc.z += fabsf(o.z) < INFINITY ? o.z * w : o.z;
            acc.w += fabsf(o.w) < INFINITY ? o.w * w : o.w;
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int node = (row0 + r) / g.group, h = head * g.group + row0 + r - node * g.group;
    if (col < a.D) {
        uint2 y;
        y.x = pack2<kDtype>(acc.x * inv, acc.y * inv);
        y.y = pack2<kDtype>(acc.z * inv, acc.w * inv);
        *(uint2 *)((uint16_t *)a.out + b * a.out_stride[0] + node * a.out_stride[1] + h * a.out_stride[2] + col) = y;
    }
    if (lane == 0 && a.lse != nullptr)
        a.lse[((size_t)b * a.T + node) * a.Hq + h] = sum == 0.f ? -INFINITY : top + logf(sum);
}

bool strides_ok(const int64_t (&s)[3]) { return s[0] >= 0 && s[1] >= 0 && s[2] >= 0 && !(s[0] % 8) && !(s[1] % 8) && !(s[2] % 8); }

int check_shape(int B, int T, int Hq, int Hkv, int D) {
    if (B <= 0 || T <= 0 || Hq <= 0 || Hkv <= 0 || D <= 0) return SPEC_ERR_INVALID_ARG;
    if (D % 8 != 0 || D > 128 || Hq % Hkv != 0 || T > SPEC_MAX_TREE_NODES || Hq > 65535 || B > (1 << 20)) return SPEC_ERR_SHAPE;
    return SPEC_OK;
}

int part_rows(int T, int Hq, int Hkv) {
    const long long rows = (long long)T * (Hq / Hkv);
    return rows < 2 * kTileRows ? (int)rows : 2 * kTileRows;
}
size_t aligned(size_t bytes) { return (bytes + kWsAlign - 1) / kWsAlign * kWsAlign; }
size_t part_lse_bytes(int T, int Hq, int Hkv) { return aligned((size_t)2 * num_sms() * part_rows(T, Hq, Hkv) * 4); }
size_t join_bytes() { return aligned((size_t)num_sms() * sizeof(Join)); }

// The cache as a TMA tensor whose boxes are a page, or 128 tokens of one, by 64 columns of a head.  Pages have to tile 128 keys
// or be tiled by them, in whole groups of 8 rows (the swizzle's period).  False: not such a cache, or strides that TMA does not take.
// By TMA and row by row, us: 131072 tokens 111 to 121, four sequences of 20000 to 40000 100 to 107, 13B trees with pages of 8, 16 and 128
// 110, 110, 106 to 112 each, 64 chains of 4 tokens, grouped heads, 125 to 134, trees of 65 to 129 nodes 393 to 414; short units, where
// the first tile's way counts, are the exception: 32 sequences of 100 to 700 tokens 129 to 121, heads of 64 46.5 to 45.3.
bool cache_map(const spec_tree_attention_t &a, const void *base, const int64_t (&stride)[3], int box_tokens, CUtensorMap *map) {
    static const auto encode = []() -> decltype(&cuTensorMapEncodeTiled) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return nullptr;
        return (decltype(&cuTensorMapEncodeTiled))fn;
    }();
    if (encode == nullptr) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)a.D, (cuuint64_t)a.page_size, (cuuint64_t)a.Hkv, (cuuint64_t)a.n_pages};
    cuuint64_t bytes[3];
    const int64_t strides[3] = {stride[1], stride[2], stride[0]};
    for (int i = 0; i < 3; ++i) {
        if (strides[i] == 0 && dims[i + 1] > 1) return false;
        bytes[i] = strides[i] ? (cuuint64_t)strides[i] * 2 : ((cuuint64_t)a.D * 2 + 15) / 16 * 16;
    }
    const cuuint32_t box[4] = {64, (cuuint32_t)box_tokens, 1, 1}, step[4] = {1, 1, 1, 1};
    return encode(map, a.dtype == SPEC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
                  const_cast<void *>(base), dims, bytes, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kDtype, int kHalves>
int launch(const AttnArgs &g, cudaStream_t st) {
    const int ctas = num_sms() < kMaxCtas ? num_sms() : kMaxCtas;
    auto kernel = tree_attention_kernel<kDtype, kHalves>;
    SPEC_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<kHalves>()));
    SPEC_CUDA_TRY(launch_pdl(kernel, dim3(ctas), dim3(kThreads), smem_bytes<kHalves>(), st, g));
    SPEC_CUDA_TRY(launch_pdl(tree_combine_kernel<kDtype>, dim3(ctas, (g.part_rows + kJoinRows - 1) / kJoinRows),
                             dim3(kJoinThreads), 0, st, g));
    return SPEC_OK;
}

}  // namespace
}  // namespace spec

using namespace spec;

extern "C" {

size_t spec_tree_attention_workspace_bytes(int B, int T, int Hq, int Hkv, int D) {
    if (check_shape(B, T, Hq, Hkv, D) != SPEC_OK) return 0;
    return join_bytes() + part_lse_bytes(T, Hq, Hkv) + aligned((size_t)2 * num_sms() * part_rows(T, Hq, Hkv) * D * 4);
}

int spec_tree_attention(const spec_tree_attention_t *a, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!a || !a->q || !a->k || !a->v || !a->k_cache || !a->v_cache || !a->block_table || !a->seq_len || !a->out)
        return SPEC_ERR_INVALID_ARG;
    if (a->dtype != SPEC_BF16 && a->dtype != SPEC_F16) return SPEC_ERR_INVALID_ARG;
    const int rc = check_shape(a->B, a->T, a->Hq, a->Hkv, a->D);
    if (rc != SPEC_OK) return rc;
    if (a->page_size <= 0 || a->n_pages <= 0 || a->max_pages <= 0 || !(fabsf(a->scale) < INFINITY)) return SPEC_ERR_INVALID_ARG;
    if (a->table_stride < a->max_pages) return SPEC_ERR_SHAPE;
    const void *ptrs[] = {a->q, a->k, a->v, a->k_cache, a->v_cache, a->out};
    for (const void *p : ptrs)
        if ((uintptr_t)p % 16 != 0) return SPEC_ERR_INVALID_ARG;
    if ((uintptr_t)a->err_word % 4 != 0) return SPEC_ERR_INVALID_ARG;
    if (!strides_ok(a->q_stride) || !strides_ok(a->k_stride) || !strides_ok(a->v_stride) || !strides_ok(a->kc_stride) ||
        !strides_ok(a->vc_stride) || !strides_ok(a->out_stride))
        return SPEC_ERR_SHAPE;
    if (!workspace || ((uintptr_t)workspace % kWsAlign) != 0 ||
        workspace_bytes < spec_tree_attention_workspace_bytes(a->B, a->T, a->Hq, a->Hkv, a->D))
        return SPEC_ERR_WORKSPACE;
    AttnArgs g;
    g.a = *a;
    g.group = a->Hq / a->Hkv;
    // (not zero: what a row does not see is minus infinity times this)
    g.scale_log2 = a->scale == 0.f ? 1e-30f : fabsf(a->scale) * kLog2e;
    const bool bf16 = a->dtype == SPEC_BF16;
    const uint32_t type = bf16 ? 1u << 7 | 1u << 10 : 0u;              // A and B: bf16 or fp16
    const uint32_t common = 1u << 4 | type | (uint32_t)(kTileRows >> 4) << 24;
    g.desc_qk = common | (uint32_t)(kStepKeys >> 3) << 17 | (a->scale < 0.f ? 1u << 13 : 0u);       // a negative scale negates Q
    g.desc_pv = common | (uint32_t)((a->D + 15) / 16 * 2) << 17 | 1u << 16;                         // V is MN-major
    g.part_rows = part_rows(a->T, a->Hq, a->Hkv);
    g.joins = (Join *)workspace;
    g.part_lse = (float *)((char *)workspace + join_bytes());
    g.part_out = (float *)((char *)g.part_lse + part_lse_bytes(a->T, a->Hq, a->Hkv));
    const long long most = (long long)a->max_pages * a->page_size;
    g.max_len = (int)(most < INT_MAX - 4096 ? most : INT_MAX - 4096);
    g.box_tokens = a->page_size % 8 ? 0 : kTileKeys % a->page_size == 0 ? a->page_size : a->page_size % kTileKeys == 0 ? kTileKeys : 0;
    if (g.box_tokens && (!cache_map(*a, a->k_cache, a->kc_stride, g.box_tokens, &g.k_map) ||
                         !cache_map(*a, a->v_cache, a->vc_stride, g.box_tokens, &g.v_map)))
        g.box_tokens = 0;
    g.box_pieces = g.box_tokens ? kTileKeys / g.box_tokens : 0;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (a->D <= 64) return bf16 ? launch<SPEC_BF16, 1>(g, st) : launch<SPEC_F16, 1>(g, st);
    return bf16 ? launch<SPEC_BF16, 2>(g, st) : launch<SPEC_F16, 2>(g, st);
}

}  // extern "C"
