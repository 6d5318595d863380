// What a serving program does around the base model's forward pass over a tree of drafted tokens, apart from the attention
// (tree_attention.cu): merging the candidates into the tree, block tables and slots of a paged cache, the greedy walk
// down the tree's logits, and the copy of the accepted keys and values to the cache (Sec. 3.1, Sec. 4.1 of arXiv 2404.19124
// describe the tree; the cache and the constraints are the serving program's).
#include <limits.h>
#include <math.h>

#include <cuda_fp16.h>

#include "spec_common.cuh"

namespace spec {

namespace {

__device__ __forceinline__ int warp_inclusive_sum(int x) {
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, off);
        if ((threadIdx.x & 31) >= off) x += y;
    }
    return x;
}

// Inclusive sum over the block's threads; `total` receives the whole.  `part`: 33 ints of shared memory.
__device__ int block_inclusive_sum(int x, int *part, int &total) {
    const int warp = threadIdx.x >> 5, warps = (blockDim.x + 31) >> 5;
    x = warp_inclusive_sum(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 31) part[warp] = x;
    __syncthreads();
    if (warp == 0) {
        const int mine = threadIdx.x < warps ? part[threadIdx.x] : 0;
        const int sum = warp_inclusive_sum(mine);
        part[threadIdx.x] = sum - mine;
        if (threadIdx.x == 31) part[32] = sum;
    }
    __syncthreads();
    total = part[32];
    return x + part[warp];
}

// ---- the candidates' tree ------------------------------------------------------------------------------------------
// One CTA per sequence.  Level by level, candidates with the same first j + 1 tokens find each other through a hash table in
// shared memory whose entries keep the lowest of them (a table of pairs (lowest candidate with the same j tokens, token)); an entry
// (k, j) whose lowest candidate is k itself is a new node, and its number is its rank in (k, j) order, a prefix sum.
// All of it is latency: 3 n + 5 barriers.
constexpr int kPlanMaxThreads = 1024;

struct PlanSmem {            // offsets in bytes
    int keys, low, first, number, parent, total;
    int slots;               // of the hash table, a power of two
};
__host__ __device__ constexpr PlanSmem plan_smem(int K, int n, int T) {
    PlanSmem s{};
    s.slots = 32;
    while (s.slots < 2 * K) s.slots *= 2;
    s.keys = 0;
    s.low = s.slots * 8;
    s.first = s.low + s.slots * 4;          // [K, n] lowest candidate with the same prefix, -1 behind the end
    s.number = s.first + K * n * 4;         // [K, n] number of a new node
    s.parent = s.number + K * n * 4;        // [T]
    s.total = s.parent + T * 4;
    return s;
}
// The most that any call asks for.  A kernel's limit belongs to the process: every call sets the same one, so that calls from
// several host threads do not lower each other's.
constexpr int kPlanMostSmem = plan_smem(SPEC_MAX_LEAVES, SPEC_MAX_TREE_ENTRIES / SPEC_MAX_LEAVES, SPEC_MAX_TREE_NODES).total;
static_assert(kPlanMostSmem <= 220 * 1024 && SPEC_MAX_TREE_ENTRIES % SPEC_MAX_LEAVES == 0, "shared memory of a CTA");

__global__ void __launch_bounds__(kPlanMaxThreads)
tree_plan_kernel(const int32_t *cand, const int32_t *last_tok, const int32_t *seq_len, int K, int n, int T, int32_t *tok,
                 int32_t *pos, int32_t *parent, uint32_t *mask, int32_t *node_of, int32_t *n_nodes) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int part[33];
    griddep_launch();
    griddep_wait();
    const PlanSmem lay = plan_smem(K, n, T);
    unsigned long long *keys = (unsigned long long *)(smem + lay.keys);
    int *low = (int *)(smem + lay.low), *first = (int *)(smem + lay.first), *number = (int *)(smem + lay.number);
    int *up = (int *)(smem + lay.parent);                // (number: the tokens first, then the entries of the table)
    const int b = blockIdx.x, t = threadIdx.x, threads = blockDim.x;
    cand += (size_t)b * K * n;
    tok += (size_t)b * T;
    pos += (size_t)b * T;
    parent += (size_t)b * T;
    node_of += (size_t)b * K * (n + 1);

    const int length = seq_len[b], root = last_tok[b];
    for (int i = t; i < K * n; i += threads) number[i] = cand[i];        // one latency of HBM, not one per level
    for (int j = 0; j < n; ++j) {
        for (int i = t; i < lay.slots; i += threads) {
            keys[i] = 0;
            low[i] = INT_MAX;
        }
        __syncthreads();
        for (int k = t; k < K; k += threads) {
            const int with = j == 0 ? 0 : first[k * n + j - 1], c = number[k * n + j];
            int at = -1;
            if (with >= 0 && c >= 0) {
                const unsigned long long key = ((unsigned long long)(with + 1) << 32) | (uint32_t)c;
                at = (int)((key * 0x9e3779b97f4a7c15ull) >> 40) & (lay.slots - 1);
                for (;;) {                      // at most half of the slots are taken
                    const unsigned long long was = atomicCAS(&keys[at], 0ull, key);
                    if (was == 0 || was == key) break;
                    at = (at + 1) & (lay.slots - 1);
                }
                atomicMin(&low[at], k);
            }
            number[k * n + j] = at;
        }
        __syncthreads();
        for (int k = t; k < K; k += threads) {
            const int at = number[k * n + j];
            first[k * n + j] = at < 0 ? -1 : low[at];
        }
        __syncthreads();
    }
    // every thread numbers a run of consecutive entries
    const int run = (K * n + threads - 1) / threads, begin = min(t * run, K * n), end = min(begin + run, K * n);
    int fresh = 0, total;
    for (int i = begin; i < end; ++i) fresh += first[i] == i / n;
    int next = 1 + block_inclusive_sum(fresh, part, total) - fresh;
    for (int i = begin; i < end; ++i)
        if (first[i] == i / n) number[i] = next++;
    const int nodes = min(1 + total, T);
    __syncthreads();
    for (int i = t; i < K * n; i += threads) {
        const int k = i / n, j = i - k * n;
        const int node = first[i] < 0 ? -1 : number[first[i] * n + j];
        node_of[k * (n + 1) + j + 1] = node < T ? node : -1;
        if (j == 0) node_of[k * (n + 1)] = 0;
        if (first[i] == k && node < T) {
            const int above = j == 0 ? 0 : number[first[i - 1] * n + j - 1];
            tok[node] = cand[i];
            parent[node] = above;
            pos[node] = length + j + 1;
            up[node] = above;
        }
    }
    for (int i = t; i < T; i += threads) {
        if (i != 0 && i < nodes) continue;
        tok[i] = i == 0 ? root : 0;
        parent[i] = -1;
        pos[i] = length;
        up[i] = -1;
    }
    if (t == 0) n_nodes[b] = nodes;
    __syncthreads();
    const int words = (T + 31) / 32;
    mask += (size_t)b * T * words;
    for (int i = t; i < T * words; i += threads) {
        const int node = i / words, w = i - node * words;
        uint32_t bits = 0;
        if (node < nodes)
            for (int at = node; at >= 0; at = up[at])
                if (at >> 5 == w) bits |= 1u << (at & 31);
        mask[i] = bits;
    }
}

// ---- block tables and slots ----------------------------------------------------------------------------------------
// The prefix sum that deals the free pages needs all sequences, so one CTA grows the tables; it writes the slots too while
// they are few, otherwise a second kernel does with the whole GPU.  One kernel against two, us on the device: 64 sequences of 32, 64, 96
// and 128 slots 5.3 to 6.9, 6.2 to 6.9, 7.2 to 7.0, 8.4 to 7.0; one sequence of 4096 and 6144 6.3 to 6.8, 8.0 to 7.1; 1024 of 1 and 4
// 7.7 to 8.5, 11.3 to 10.0.
constexpr int kOneKernelSlots = 4096;
constexpr int kTableThreads = 1024;
constexpr int kSlotThreads = 256;

struct TableArgs {
    const int32_t *seq_len, *n_new;          // n_new null: max_new everywhere
    int B, page, max_new;
    int32_t *table;                          // rows `stride` apart
    long long stride;
    int max_pages;
    const int32_t *n_pages, *free_pages, *free_count;
    int n_free;                              // entries of free_pages
    int64_t *slots;                          // [B, max_new]
    int32_t *n_pages_out, *free_count_out, *err;
};

__device__ __forceinline__ int in_range(int x, int lo, int hi, int32_t *err) {
    if (x < lo || x > hi) report_error(err, SPEC_ERR_INDEX_RANGE);
    return min(max(x, lo), hi);
}

// The slot of new token j of a sequence that has `held` pages.
__device__ __forceinline__ int64_t slot_of(const TableArgs &a, int b, int j) {
    const int length = max(a.seq_len[b], 0), fresh = a.n_new == nullptr ? a.max_new : min(a.n_new[b], a.max_new);
    const unsigned at = (unsigned)length + (unsigned)j, page = at / (unsigned)a.page;        // both below 2^31: the sum fits
    if (j >= fresh || page >= (unsigned)a.n_pages_out[b]) return -1;
    const int id = a.table[b * a.stride + page];
    if (id < 0) {
        report_error(a.err, SPEC_ERR_INDEX_RANGE);
        return -1;
    }
    return (int64_t)id * a.page + (at - page * (unsigned)a.page);
}

__global__ void __launch_bounds__(kTableThreads) page_tables_kernel(const TableArgs a, int with_slots) {
    __shared__ int part[33];
    __shared__ int held_s[kTableThreads], grow_s[kTableThreads], first_s[kTableThreads];
    griddep_launch();
    griddep_wait();
    const int t = threadIdx.x, lane = t & 31;
    const int avail = in_range(*a.free_count, 0, a.n_free, a.err);
    long long asked = 0;                     // pages that the sequences before this block of them ask for
    int taken = 0;                           // ... and get
    for (int b0 = 0; b0 < a.B; b0 += kTableThreads) {
        const int b = b0 + t, count = min(a.B - b0, kTableThreads);
        int held = 0, need = 0;
        if (b < a.B) {
            const int length = in_range(a.seq_len[b], 0, INT_MAX, a.err);
            const int fresh = a.n_new == nullptr ? a.max_new : in_range(a.n_new[b], 0, a.max_new, a.err);
            held = in_range(a.n_pages[b], 0, a.max_pages, a.err);
            const long long want = ((long long)length + fresh + a.page - 1) / a.page;
            if (want > a.max_pages) report_error(a.err, SPEC_ERR_PAGES);
            else need = max((int)want - held, 0);
        }
        int total;                           // at most B max_pages, which the host keeps within 32 bits
        const int before = block_inclusive_sum(need, part, total) - need;
        const bool fits = asked + before + need <= avail;
        if (b < a.B) {
            if (!fits && need > 0) report_error(a.err, SPEC_ERR_PAGES);
            held_s[t] = held;
            grow_s[t] = fits ? need : 0;
            first_s[t] = (int)(avail - 1 - asked - before);    // only read where it fits
            a.n_pages_out[b] = held + grow_s[t];
        }
        // The sums rise with the sequence: behind one that does not fit, only sequences that ask for nothing are served.
        int dealt;
        block_inclusive_sum(b < a.B ? grow_s[t] : 0, part, dealt);
        __syncthreads();
        for (int i = t >> 5; i < count; i += kTableThreads / 32)
            for (int p = lane; p < grow_s[i]; p += 32)
                a.table[(b0 + i) * a.stride + held_s[i] + p] = a.free_pages[first_s[i] - p];
        asked += total;
        taken += dealt;
        __syncthreads();
    }
    if (t == 0) *a.free_count_out = avail - taken;
    if (with_slots)
        for (int i = t; i < a.B * a.max_new; i += kTableThreads) a.slots[i] = slot_of(a, i / a.max_new, i % a.max_new);
}

__global__ void __launch_bounds__(kSlotThreads) page_slots_kernel(const TableArgs a) {
    griddep_launch();
    griddep_wait();
    for (long long i = (long long)blockIdx.x * kSlotThreads + threadIdx.x; i < (long long)a.B * a.max_new;
         i += (long long)gridDim.x * kSlotThreads)
        a.slots[i] = slot_of(a, (int)(i / a.max_new), (int)(i % a.max_new));
}

// ---- the greedy walk -----------------------------------------------------------------------------------------------
// A cluster of CTAs per sequence; the vocabulary goes to them in blocks of 4096 tokens in turn.  Per step every CTA finds the
// maximum of its blocks of the current node's row, the CTAs exchange theirs through distributed shared memory, and all of them
// look up the child that carries the winner.  Only the rows on the path are read, so a step is latency: the loads of a row (1.5 us
// at a vocabulary of 32000), one exchange (1 us), one look at the tree, which lies in shared memory (0.5 us).
//
// Constraints.  The tokens that penalties or biases touch are few.  Each CTA counts those of its blocks once, in a table in
// shared memory, and marks them in a bitmap: the pass over the row leaves them out (and what the grammar forbids), and every
// listed token is looked at by itself.  The table is hashed while that is smaller, which lets four CTAs share an SM for
// histories of a few thousand tokens, else it has an entry per token.  64 sequences, a vocabulary of 128256, histories of up to
// 2048 tokens, a grammar: 53 us (34 without constraints); a table of 130 KB and checks per element took 278.
constexpr int kWalkThreads = 256;
constexpr int kWalkWarps = kWalkThreads / 32;
constexpr int kWalkCtasPerSm = 4;            // by registers
constexpr int kWalkMaxCluster = 16;
constexpr size_t kWalkMostSmem = 200 * 1024; // what a CTA may ask for
constexpr int kBlockTokens = 4096;
constexpr int kNoToken = INT_MAX;
constexpr uint32_t kSeen = 1u << 31;         // of a token's count: it is in the history (the rest: times it was generated)
constexpr uint32_t kFree = 0xffffffffu;      // of a key

struct WalkArgs {
    spec_tree_verify_t v;
    int log_ctas;
    int cap;                                 // entries of the table: somewhat more than max_list (hashed) or the CTA's tokens; 0: no constraints by token
    int hashed, max_list, part;              // part: tokens of a CTA, whole blocks
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_sync() {
    cluster_arrive();
    cluster_wait();
}
__device__ __forceinline__ void store_peer(const void *p, uint32_t rank, float x, int y) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(a), "r"(__float_as_uint(x)), "r"(y) : "memory");
}

template <int kDtype> struct Logit;
template <> struct Logit<SPEC_BF16> {
    static constexpr int kBytes = 2;
    static __device__ __forceinline__ float get(const uint4 &v, int i) {
        const uint32_t w = (&v.x)[i >> 1];
        return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
    }
    static __device__ __forceinline__ float at(const void *row, int i) { return bf16_bits_to_float(((const uint16_t *)row)[i]); }
    // the greatest of a vector; NaN only if all are
    static __device__ __forceinline__ float most(const uint4 &v) {
        uint32_t a, b;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
        asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
        asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
        return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
    }
};
template <> struct Logit<SPEC_F16> {
    static constexpr int kBytes = 2;
    static __device__ __forceinline__ float get(const uint4 &v, int i) {
        const uint32_t w = (&v.x)[i >> 1];
        return __half2float(__ushort_as_half((unsigned short)(i & 1 ? w >> 16 : w & 0xffffu)));
    }
    static __device__ __forceinline__ float at(const void *row, int i) {
        return __half2float(__ushort_as_half(((const unsigned short *)row)[i]));
    }
    static __device__ __forceinline__ float most(const uint4 &v) {
        uint32_t a, b;
        asm("max.f16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
        asm("max.f16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
        asm("max.f16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
        const __half2 h = *(__half2 *)&a;
        return fmaxf(__low2float(h), __high2float(h));
    }
};
template <> struct Logit<SPEC_F32> {
    static constexpr int kBytes = 4;
    static __device__ __forceinline__ float get(const uint4 &v, int i) { return __uint_as_float((&v.x)[i]); }
    static __device__ __forceinline__ float at(const void *row, int i) { return ((const float *)row)[i]; }
    static __device__ __forceinline__ float most(const uint4 &v) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
};

struct Best {
    float value;
    int tok;
    __device__ __forceinline__ void offer(float x, int t) {
        x = x != x ? -INFINITY : x;          // a NaN counts as minus infinity
        if (x > value || (x == value && t < tok)) {
            value = x;
            tok = t;
        }
    }
    __device__ __forceinline__ void join_warp() {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const float ov = __shfl_xor_sync(0xffffffffu, value, off);
            const int ot = __shfl_xor_sync(0xffffffffu, tok, off);
            offer(ov, ot);
        }
    }
};

// The tokens of this CTA that penalties or biases touch.
struct WalkTable {
    uint32_t *key;        // [cap] hashed only: token, kFree
    uint32_t *count;      // [cap] kSeen and the times generated
    uint32_t *bias;       // [cap] entry of the bias list + 1, 0: none
    uint32_t *marked;     // [part / 32]
    int *list;            // [max_list] entries in use
    int *n_list;
};

// Number of a token among the CTA's own.
__device__ __forceinline__ int local_token(const WalkArgs &a, int t) {
    return (t / kBlockTokens >> a.log_ctas) * kBlockTokens + t % kBlockTokens;
}
__device__ __forceinline__ bool owns(const WalkArgs &a, uint32_t rank, int t) {
    return (unsigned)t < (unsigned)a.v.V && (t / kBlockTokens & ((1 << a.log_ctas) - 1)) == (int)rank;
}

// The entry of a token, which is made and listed if there is none.
__device__ __forceinline__ int table_entry(const WalkArgs &a, const WalkTable &w, int t) {
    const int local = local_token(a, t);
    int at = local;
    if (a.hashed) {
        at = (int)__umulhi((uint32_t)t * 0x9e3779b1u, (uint32_t)a.cap);
        for (;;) {                                       // there are fewer tokens than entries
            const uint32_t was = atomicCAS(&w.key[at], kFree, (uint32_t)t);
            if (was == kFree || was == (uint32_t)t) break;
            at = at + 1 == a.cap ? 0 : at + 1;
        }
    }
    const uint32_t bit = 1u << (local & 31);
    if (!(atomicOr(&w.marked[local >> 5], bit) & bit)) w.list[atomicAdd(w.n_list, 1)] = at;
    return at;
}

__device__ __forceinline__ float walk_adjust(const WalkArgs &a, const WalkTable &w, int b, int at, float x, float rep, float freq,
                                             float pres) {
    // Each step rounds once, in the order of the definition: no contraction into fused multiply-adds.
    if (a.v.hist_tok != nullptr) {
        const uint32_t c = w.count[at];
        if (c & kSeen) x = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
        const uint32_t times = c & ~kSeen;
        if (times) x = __fsub_rn(__fsub_rn(x, __fmul_rn(freq, (float)times)), pres);
    }
    if (a.v.bias_tok != nullptr && w.bias[at]) x = __fadd_rn(x, a.v.bias_val[(size_t)b * a.v.max_bias + w.bias[at] - 1]);
    return x;
}

// Eight consecutive bits of a bit field of `bytes` bytes, from `first` on, which is a multiple of 4 or, unless kAligned, anything.
template <bool kAligned>
__device__ __forceinline__ uint32_t bits_from(const uint32_t *field, int first, int bytes) {
    const uint8_t *p = (const uint8_t *)field;
    uint32_t x = p[first >> 3];
    if (kAligned) return x >> (first & 4);
    if (first & 7) {
        if ((first >> 3) + 1 < bytes) x |= (uint32_t)p[(first >> 3) + 1] << 8;
        x >>= first & 7;
    }
    return x & 0xffu;
}

// A vector with what `use` does not keep at minus infinity.  keep: for each of 256 values of `use` the 16-bit elements that stay.
template <int kDtype>
__device__ __forceinline__ void blank(uint4 &x, uint32_t use, const uint4 *keep) {
    if (kDtype == SPEC_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (!(use >> i & 1)) (&x.x)[i] = 0xff800000u;
    } else {
        constexpr uint32_t kNone = kDtype == SPEC_BF16 ? 0xff80ff80u : 0xfc00fc00u;
        const uint4 k = keep[use];
        x.x = (x.x & k.x) | (kNone & ~k.x);
        x.y = (x.y & k.y) | (kNone & ~k.y);
        x.z = (x.z & k.z) | (kNone & ~k.z);
        x.w = (x.w & k.w) | (kNone & ~k.w);
    }
}

// The maximum over this CTA's blocks of a row, of the tokens that `allow` (null: all) and `marked` (null: none) leave.  A thread's
// vectors rise and four of them (and the grammar's bits) are in flight.  It keeps the first vector with the greatest maximum, without a
// branch, and looks for the element at the end: a branch for every new maximum is taken by some lane nearly always.
// kAligned: the row begins at a vector, so that no vector holds elements of two blocks or two bytes of bits.  Otherwise the vectors
// in which blocks end come last and may lie before the one that the thread has kept: equal maxima are told apart by their place (and a
// vector that two blocks share is the first one's end).
template <int kDtype, bool kAligned>
__device__ __forceinline__ void scan_row(const WalkArgs &a, const char *row, uint32_t rank, const uint32_t *allow, int words,
                                         const uint32_t *marked, const uint4 *keep, Best &best) {
    constexpr int kPer = 16 / Logit<kDtype>::kBytes, kPerThread = kBlockTokens / kPer / kWalkThreads, kAhead = 4;
    constexpr uint32_t kAll = (1u << kPer) - 1;
    const int V = a.v.V;
    const int skew = kAligned ? 0 : (int)(((uintptr_t)row & 15) / Logit<kDtype>::kBytes);        // elements behind a vector's start
    const uint4 *vec = (const uint4 *)(row - skew * Logit<kDtype>::kBytes);
    const int blocks = (V + kBlockTokens - 1) / kBlockTokens;
    const int turns = (blocks - (int)rank + (1 << a.log_ctas) - 1) >> a.log_ctas;
    uint4 best_x = make_uint4(0, 0, 0, 0);
    float best_top = -INFINITY;
    uint32_t best_use = 0;
    int best_e0 = 0;
    auto first_of = [&](int turn) { return ((turn << a.log_ctas) + (int)rank) * kBlockTokens; };
    // use: the grammar's bits from max(e0, begin) on; ends: a vector in which a block ends
    auto look = [&](uint4 x, int e0, int begin, int turn, uint32_t use, bool ends) {
        const int from = kAligned ? e0 : max(e0, begin);
        if (marked != nullptr) use &= ~bits_from<kAligned>(marked, turn * kBlockTokens + from - begin, a.part / 8);
        use = use << (from - e0) & kAll;
        if (!kAligned && e0 + kPer > begin + kBlockTokens) use &= kAll >> (e0 + kPer - begin - kBlockTokens);
        if (e0 + kPer > V) use &= kAll >> (e0 + kPer - V);
        if (e0 < 0 || e0 + kPer > V) {                   // a vector that reaches beyond the row: the memory there may be nobody's
            uint32_t y[4] = {0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                if (e0 + e < 0 || e0 + e >= V) continue;
                if (Logit<kDtype>::kBytes == 2) y[e / 2] |= (uint32_t)((const uint16_t *)row)[e0 + e] << 16 * (e % 2);
                else y[e] = ((const uint32_t *)row)[e0 + e];
            }
            x = make_uint4(y[0], y[1], y[2], y[3]);
        }
        if (use != kAll) blank<kDtype>(x, use, keep);
        const float top = fmaxf(Logit<kDtype>::most(x), -INFINITY);
        const bool take = use != 0 && (best_use == 0 || top > best_top || (ends && top == best_top && e0 <= best_e0));
        best_top = take ? top : best_top;
        best_use = take ? use : best_use;
        best_e0 = take ? e0 : best_e0;
        best_x.x = take ? x.x : best_x.x;
        best_x.y = take ? x.y : best_x.y;
        best_x.z = take ? x.z : best_x.z;
        best_x.w = take ? x.w : best_x.w;
    };
    for (int turn0 = 0; turn0 < turns; turn0 += kAhead / kPerThread) {
        uint4 x[kAhead];
        uint32_t use[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int turn = turn0 + k / kPerThread, begin = first_of(turn);
            const int e0 = begin - skew + ((int)threadIdx.x + k % kPerThread * kWalkThreads) * kPer;
            use[k] = kAll;
            x[k] = make_uint4(0, 0, 0, 0);
            if (turn >= turns || e0 >= V) continue;
            if (e0 >= 0 && e0 + kPer <= V) x[k] = __ldg((const uint4 *)((const char *)vec + (long long)(e0 + skew) * Logit<kDtype>::kBytes));
            if (allow != nullptr) use[k] = bits_from<kAligned>(allow, kAligned ? e0 : max(e0, begin), words * 4);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int turn = turn0 + k / kPerThread, begin = first_of(turn);
            const int e0 = begin - skew + ((int)threadIdx.x + k % kPerThread * kWalkThreads) * kPer;
            if (turn < turns && e0 < V) look(x[k], e0, begin, turn, use[k], false);
        }
    }
    if (!kAligned)                                       // the vectors in which blocks end
        for (int turn = threadIdx.x; turn < turns; turn += kWalkThreads) {
            const int begin = first_of(turn), e0 = begin - skew + kBlockTokens;
            if (e0 >= V) continue;
            const uint4 x = e0 + kPer <= V ? __ldg((const uint4 *)((const char *)vec + (long long)(e0 + skew) * Logit<kDtype>::kBytes))
                                           : make_uint4(0, 0, 0, 0);
            look(x, e0, begin, turn, allow != nullptr ? bits_from<kAligned>(allow, e0, words * 4) : kAll, true);
        }
    if (best_use == 0) return;
#pragma unroll
    for (int e = 0; e < kPer; ++e)                       // (a NaN counts as minus infinity)
        if (best_use >> e & 1) best.offer(Logit<kDtype>::get(best_x, e), best_e0 + e);
}

template <int kDtype>
__global__ void __launch_bounds__(kWalkThreads, kWalkCtasPerSm) tree_walk_kernel(const WalkArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ Best warp_best[kWalkWarps];
    __shared__ __align__(8) Best peer_best[2][kWalkMaxCluster];
    __shared__ uint4 keep[kDtype == SPEC_F32 ? 1 : 256];
    __shared__ int child[3], n_list;                     // child: of three steps in turn, so that none is cleared while it is read
    griddep_launch();
    cluster_arrive();                        // (waited for before the walk: a CTA's shared memory is there once it has begun)
    griddep_wait();
    const spec_tree_verify_t &v = a.v;
    const int t = threadIdx.x, lane = t & 31, ranks = 1 << a.log_ctas;
    const uint32_t rank = cluster_rank();
    const int b = blockIdx.x >> a.log_ctas;
    const int V = v.V, words = (V + 31) / 32;
    int *tok = (int *)smem, *parent = tok + v.T;
    WalkTable w;
    w.key = (uint32_t *)(parent + v.T);
    w.count = w.key + (a.hashed ? a.cap : 0);
    w.bias = w.count + (v.hist_tok != nullptr ? a.cap : 0);
    w.marked = w.bias + (v.bias_tok != nullptr ? a.cap : 0);
    w.list = (int *)(w.marked + (a.cap ? a.part / 32 : 0));
    w.n_list = &n_list;
    const int nodes = min(v.n_nodes[b], v.T);
    const float rep = v.repetition != nullptr ? v.repetition[b] : 1.f;
    const float freq = v.frequency != nullptr ? v.frequency[b] : 0.f;
    const float pres = v.presence != nullptr ? v.presence[b] : 0.f;
    for (int i = t; i < nodes; i += kWalkThreads) {
        tok[i] = v.tok[(size_t)b * v.T + i];
        parent[i] = v.parent[(size_t)b * v.T + i];
    }
    if (t == 0) {
        n_list = 0;
        child[0] = INT_MAX;
    }
    if (kDtype != SPEC_F32 && t < 256) {
#pragma unroll
        for (int i = 0; i < 4; ++i) (&keep[t].x)[i] = (t >> 2 * i & 1) * 0xffffu | (t >> (2 * i + 1) & 1) * 0xffff0000u;
    }
    if (a.cap) {
        if (a.hashed)
            for (int i = t; i < a.cap; i += kWalkThreads) w.key[i] = kFree;
        for (uint32_t *p = w.count + t; p < (uint32_t *)w.list; p += kWalkThreads) *p = 0;
        __syncthreads();
        if (v.hist_tok != nullptr) {
            const int size = min(v.hist_len[b], v.max_hist), prompt = v.prompt_len == nullptr ? 0 : v.prompt_len[b];
            const int32_t *hist = v.hist_tok + (size_t)b * v.max_hist;
            constexpr int kAhead = 2;
            for (int i0 = 0; i0 < size; i0 += kWalkThreads * kAhead) {
                int h[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int i = i0 + k * kWalkThreads + t;
                    h[k] = i < size ? hist[i] : -1;
                    if (!owns(a, rank, h[k])) h[k] = -1;
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    // equal tokens of a warp are counted together: a few tokens make up most of a text
                    const unsigned same = __match_any_sync(0xffffffffu, h[k]);
                    const unsigned made = __ballot_sync(0xffffffffu, i0 + k * kWalkThreads + t >= prompt) & same;
                    if (h[k] >= 0 && lane == __ffs(same) - 1) {
                        const int at = table_entry(a, w, h[k]);
                        atomicOr(&w.count[at], kSeen);
                        if (made) atomicAdd(&w.count[at], (uint32_t)__popc(made));
                    }
                }
            }
        }
        if (v.bias_tok != nullptr) {
            const int size = v.bias_len == nullptr ? v.max_bias : min(v.bias_len[b], v.max_bias);
            for (int i = t; i < size; i += kWalkThreads) {
                const int h = v.bias_tok[(size_t)b * v.max_bias + i];
                if (owns(a, rank, h)) atomicMax(&w.bias[table_entry(a, w, h)], (uint32_t)i + 1);     // the list's last entry counts
            }
        }
    }
    __syncthreads();
    cluster_wait();

    int cur = 0, accepted = 0, token = -1;
    if (nodes > 0) {
        for (int step = 0;; ++step) {
            Best best = {-INFINITY, kNoToken};
            const char *row = (const char *)v.logits + ((long long)b * v.logits_stride[0] + (long long)cur * v.logits_stride[1]) *
                                                           Logit<kDtype>::kBytes;
            const uint32_t *allow = v.allow == nullptr ? nullptr : v.allow + ((size_t)b * v.T + cur) * words;
            const uint32_t *marked = a.cap ? w.marked : nullptr;
            if (((uintptr_t)row & 15) == 0) scan_row<kDtype, true>(a, row, rank, allow, words, marked, keep, best);
            else scan_row<kDtype, false>(a, row, rank, allow, words, marked, keep, best);
            if (a.cap) {
                const int n = n_list;
                for (int i = t; i < n; i += kWalkThreads) {
                    const int at = w.list[i];
                    const int h = a.hashed ? (int)w.key[at]
                                           : ((at / kBlockTokens << a.log_ctas) + (int)rank) * kBlockTokens + at % kBlockTokens;
                    if (allow == nullptr || (allow[h >> 5] >> (h & 31) & 1))
                        best.offer(walk_adjust(a, w, b, at, Logit<kDtype>::at(row, h), rep, freq, pres), h);
                }
            }
            best.join_warp();
            if (lane == 0) warp_best[t >> 5] = best;
            if (t == 0) child[(step + 1) % 3] = INT_MAX;
            __syncthreads();
            if (t < 32) {
                best = t < kWalkWarps ? warp_best[t] : Best{-INFINITY, kNoToken};
                best.join_warp();
                if (t < ranks) store_peer(&peer_best[step & 1][rank], t, best.value, best.tok);
            }
            cluster_sync();
            best = lane < ranks ? peer_best[step & 1][lane] : Best{-INFINITY, kNoToken};
            best.join_warp();
            token = best.tok == kNoToken ? -1 : best.tok;
            if (rank == 0 && t == 0) v.path[(size_t)b * (v.n + 1) + step] = cur;
            if (step == v.n || token < 0) break;
            for (int i = 1 + t; i < nodes; i += kWalkThreads)
                if (parent[i] == cur && tok[i] == token) atomicMin(&child[step % 3], i);
            if (v.hist_tok != nullptr && t == 0 && owns(a, rank, token)) {
                uint32_t *count = &w.count[table_entry(a, w, token)];
                *count = (*count | kSeen) + 1;
            }
            __syncthreads();
            if (child[step % 3] == INT_MAX) break;
            cur = child[step % 3];
            ++accepted;
        }
    }
    cluster_sync();                          // no CTA leaves while another may still write to its shared memory
    if (rank == 0) {
        if (t == 0) {
            v.accept_len[b] = accepted;
            v.last_node[b] = nodes > 0 ? cur : -1;
            v.next_tok[b] = token;
        }
        for (int j = (nodes > 0 ? accepted + 1 : 0) + t; j <= v.n; j += kWalkThreads) v.path[(size_t)b * (v.n + 1) + j] = -1;
    }
}

// ---- accepted keys and values --------------------------------------------------------------------------------------
// A thread copies 16 bytes of every accepted row, the loads of two rows in flight before the first store (more cost occupancy:
// 13.2 us with two, 14.3 with six, 15.9 with eight at 50 MB): bound by HBM for batches, by latency for few sequences.
constexpr int kCommitThreads = 256;
constexpr int kCommitRows = 2;

__device__ __forceinline__ uint4 ld_once(const uint4 *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

__global__ void __launch_bounds__(kCommitThreads) kv_commit_kernel(const spec_kv_commit_t c) {
    griddep_launch();
    griddep_wait();
    const int b = blockIdx.y, n1 = c.n + 1;
    // (a path that does not begin: a sequence without a node)
    const int rows = c.path[(size_t)b * n1] < 0 ? 0 : min(max(c.accept_len[b], -1), c.n) + 1;
    if (blockIdx.x == 0 && threadIdx.x == 0 && c.new_len != nullptr) {
        int stored = rows;                   // a length counts no tokens behind the last slot: there are none where pages ran out
        while (stored > 0 && c.slots[(size_t)b * n1 + stored - 1] == -1) --stored;
        c.new_len[b] = c.seq_len[b] + stored;
    }
    const int per_head = c.D / 8, per_row = c.H * per_head;
    const long long i = (long long)blockIdx.x * kCommitThreads + threadIdx.x;
    if (i >= 2ll * c.L * per_row) return;
    const int vec = (int)(i % per_row), layer = (int)(i / per_row) % c.L;
    const bool is_v = i / per_row >= c.L;
    const int head = vec / per_head, d = (vec - head * per_head) * 8;
    const int64_t *ss = is_v ? c.v_stride : c.k_stride, *ds = is_v ? c.vc_stride : c.kc_stride;
    const uint16_t *src = (const uint16_t *)(is_v ? c.v : c.k) + layer * ss[0] + b * ss[1] + head * ss[3] + d;
    uint16_t *dst = (uint16_t *)(is_v ? c.v_cache : c.k_cache) + layer * ds[0] + head * ds[3] + d;
    for (int j0 = 0; j0 < rows; j0 += kCommitRows) {
        uint4 x[kCommitRows];
        uint16_t *to[kCommitRows];
#pragma unroll
        for (int i = 0; i < kCommitRows; ++i) {
            to[i] = nullptr;
            if (j0 + i >= rows) continue;
            const int node = c.path[(size_t)b * n1 + j0 + i];
            const long long slot = c.slots[(size_t)b * n1 + j0 + i];
            if (node < 0 || node >= c.T || slot < 0 || slot >= (long long)c.n_pages * c.page_size) {
                report_error(c.err_word, SPEC_ERR_INDEX_RANGE);
                continue;
            }
            x[i] = ld_once((const uint4 *)(src + node * ss[2]));
            const unsigned page = (unsigned)slot / (unsigned)c.page_size;
            to[i] = dst + page * ds[1] + ((int)slot - (int)(page * c.page_size)) * ds[2];
        }
#pragma unroll
        for (int i = 0; i < kCommitRows; ++i)
            if (to[i] != nullptr) *(uint4 *)to[i] = x[i];
    }
}

template <int kDtype>
int launch_walk(const WalkArgs &a, size_t smem, cudaStream_t st) {
    auto kernel = tree_walk_kernel<kDtype>;
    const int ctas = 1 << a.log_ctas;
    // (the same for every call: see kPlanMostSmem)
    SPEC_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kWalkMostSmem));
    if (ctas > 8) SPEC_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    SPEC_CUDA_TRY(launch_pdl_cluster(kernel, dim3((unsigned)ctas * a.v.B), dim3(kWalkThreads), smem, ctas, st, a));
    return SPEC_OK;
}

// The table of a CTA (bytes per entry: key, count, bias), the bitmap and the list.
bool plan_walk_table(WalkArgs &a, int log_ctas, size_t &smem) {
    const spec_tree_verify_t &v = a.v;
    const long long blocks = ((long long)v.V + kBlockTokens - 1) / kBlockTokens;
    const long long part = (blocks + (1 << log_ctas) - 1) / (1 << log_ctas) * kBlockTokens;
    const size_t tree = (size_t)v.T * 8, per_entry = 4 * ((v.hist_tok ? 1 : 0) + (v.bias_tok ? 1 : 0));
    a.log_ctas = log_ctas;
    a.cap = a.hashed = a.max_list = a.part = 0;
    smem = tree;
    if (!per_entry) return true;
    const long long tokens = (long long)v.max_hist + v.max_bias + v.n;
    const long long listed = tokens < part ? tokens : part;
    long long cap = listed + listed / 3 + 8;             // three quarters full at most
    const bool hashed = cap * (per_entry + 4) < part * per_entry;
    if (!hashed) cap = part;
    smem = tree + (size_t)cap * (per_entry + (hashed ? 4 : 0)) + (size_t)part / 8 + (size_t)listed * 4;
    if (smem > kWalkMostSmem) return false;
    a.cap = (int)cap;
    a.hashed = hashed;
    a.max_list = (int)listed;
    a.part = (int)part;
    return true;
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace
}  // namespace spec

using namespace spec;

extern "C" {

int spec_tree_plan(const int32_t *cand_tok, const int32_t *last_tok, const int32_t *seq_len, int B, int K, int n, int T,
                   int32_t *tok, int32_t *pos, int32_t *parent, uint32_t *mask, int32_t *node_of, int32_t *n_nodes,
                   void *cuda_stream) {
    if (!cand_tok || !last_tok || !seq_len || !tok || !pos || !parent || !mask || !node_of || !n_nodes)
        return SPEC_ERR_INVALID_ARG;
    if (B <= 0 || K <= 0 || n <= 0 || T <= 0) return SPEC_ERR_INVALID_ARG;
    if (n > SPEC_MAX_TREE_DEPTH || T > SPEC_MAX_TREE_NODES || K > SPEC_MAX_LEAVES || (long long)K * n > SPEC_MAX_TREE_ENTRIES)
        return SPEC_ERR_SHAPE;
    const PlanSmem lay = plan_smem(K, n, T);
    if (lay.total > 40 * 1024)
        SPEC_CUDA_TRY(cudaFuncSetAttribute(tree_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPlanMostSmem));
    int threads = K * n > T * ((T + 31) / 32) ? K * n : T * ((T + 31) / 32);     // words of the masks are the most to write
    threads = threads >= kPlanMaxThreads ? kPlanMaxThreads : (threads + 31) / 32 * 32;
    SPEC_CUDA_TRY(launch_pdl(tree_plan_kernel, dim3(B), dim3(threads), (size_t)lay.total, (cudaStream_t)cuda_stream, cand_tok,
                             last_tok, seq_len, K, n, T, tok, pos, parent, mask, node_of, n_nodes));
    return SPEC_OK;
}

int spec_page_tables(const int32_t *seq_len, const int32_t *n_new, int B, int page_size, int max_new, int32_t *block_table,
                     int64_t table_stride, int max_pages, const int32_t *n_pages, const int32_t *free_pages,
                     const int32_t *free_count, int n_free, int64_t *slots, int32_t *n_pages_out, int32_t *free_count_out,
                     int32_t *err_word, void *cuda_stream) {
    if (!seq_len || !block_table || !n_pages || !free_pages || !free_count || !slots || !n_pages_out || !free_count_out)
        return SPEC_ERR_INVALID_ARG;
    if (B <= 0 || page_size <= 0 || max_new <= 0 || max_pages <= 0 || n_free <= 0) return SPEC_ERR_INVALID_ARG;
    if ((uintptr_t)err_word % 4 != 0) return SPEC_ERR_INVALID_ARG;
    if (table_stride < max_pages || (long long)B * max_new > INT_MAX || (long long)B * max_pages > INT_MAX) return SPEC_ERR_SHAPE;
    const TableArgs a = {seq_len, n_new, B, page_size, max_new, block_table, table_stride, max_pages, n_pages, free_pages,
                         free_count, n_free, slots, n_pages_out, free_count_out, err_word};
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int all = B * max_new;
    const bool one = all <= kOneKernelSlots;
    SPEC_CUDA_TRY(launch_pdl(page_tables_kernel, dim3(1), dim3(kTableThreads), 0, st, a, one ? 1 : 0));
    if (!one) {
        const int blocks = (all - 1) / kSlotThreads + 1, most = 8 * num_sms();
        SPEC_CUDA_TRY(launch_pdl(page_slots_kernel, dim3(blocks < most ? blocks : most), dim3(kSlotThreads), 0, st, a));
    }
    return SPEC_OK;
}

int spec_verify_tree(const spec_tree_verify_t *v, void *cuda_stream) {
    if (!v || !v->tok || !v->parent || !v->n_nodes || !v->logits || !v->accept_len || !v->last_node || !v->next_tok || !v->path)
        return SPEC_ERR_INVALID_ARG;
    if (v->B <= 0 || v->T <= 0 || v->V <= 0 || v->n < 0) return SPEC_ERR_INVALID_ARG;
    if (v->logits_dtype != SPEC_BF16 && v->logits_dtype != SPEC_F16 && v->logits_dtype != SPEC_F32) return SPEC_ERR_INVALID_ARG;
    if ((uintptr_t)v->logits % (v->logits_dtype == SPEC_F32 ? 4 : 2) != 0) return SPEC_ERR_INVALID_ARG;
    if (v->logits_stride[0] < 0 || v->logits_stride[1] < 0) return SPEC_ERR_INVALID_ARG;
    if (v->hist_tok && (!v->hist_len || v->max_hist <= 0)) return SPEC_ERR_INVALID_ARG;
    if (!v->hist_tok && (v->repetition || v->frequency || v->presence || v->prompt_len)) return SPEC_ERR_INVALID_ARG;
    if (v->bias_tok && (!v->bias_val || v->max_bias <= 0)) return SPEC_ERR_INVALID_ARG;
    if (v->n > SPEC_MAX_TREE_DEPTH || v->T > SPEC_MAX_TREE_NODES || v->B > (1 << 20) || v->V > (1 << 30) ||
        v->max_hist > (1 << 30) || v->max_bias > (1 << 30))
        return SPEC_ERR_SHAPE;
    WalkArgs a;
    a.v = *v;
    // A block per CTA, up to the 8 CTAs that any cluster may have, but no more CTAs than run at the same time (a second round
    // of clusters costs a whole walk, and fewer CTAs per sequence only some of the rows' latency); 16 where the table does not
    // fit otherwise.
    int most = 0, log_ctas = -1;
    while (most < 3 && ((long long)kBlockTokens << most) < v->V) ++most;
    size_t smem = 0;
    for (int l = most; l >= 0; --l) {
        if (!plan_walk_table(a, l, smem)) continue;
        log_ctas = l;
        const long long per_sm = 227 * 1024 / ((long long)smem + 6144);
        if (((long long)v->B << l) <= num_sms() * (per_sm < kWalkCtasPerSm ? per_sm : kWalkCtasPerSm)) break;
    }
    if (!plan_walk_table(a, log_ctas < 0 ? 4 : log_ctas, smem)) return SPEC_ERR_SHAPE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (v->logits_dtype == SPEC_BF16) return launch_walk<SPEC_BF16>(a, smem, st);
    if (v->logits_dtype == SPEC_F16) return launch_walk<SPEC_F16>(a, smem, st);
    return launch_walk<SPEC_F32>(a, smem, st);
}

int spec_kv_commit(const spec_kv_commit_t *c, void *cuda_stream) {
    if (!c || !c->k || !c->v || !c->k_cache || !c->v_cache || !c->path || !c->accept_len || !c->slots) return SPEC_ERR_INVALID_ARG;
    if ((c->new_len && !c->seq_len) || (uintptr_t)c->err_word % 4 != 0) return SPEC_ERR_INVALID_ARG;
    if (c->L <= 0 || c->B <= 0 || c->T <= 0 || c->n < 0 || c->H <= 0 || c->D <= 0 || c->page_size <= 0 || c->n_pages <= 0)
        return SPEC_ERR_INVALID_ARG;
    if (c->D % 8 != 0 || c->B > 65535 || (long long)c->L * c->H * c->D > INT_MAX / 4) return SPEC_ERR_SHAPE;
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_cache) || !aligned16(c->v_cache)) return SPEC_ERR_INVALID_ARG;
    for (int i = 0; i < 4; ++i) {
        if (c->k_stride[i] % 8 || c->v_stride[i] % 8 || c->kc_stride[i] % 8 || c->vc_stride[i] % 8) return SPEC_ERR_SHAPE;
        if (c->k_stride[i] < 0 || c->v_stride[i] < 0 || c->kc_stride[i] < 0 || c->vc_stride[i] < 0) return SPEC_ERR_INVALID_ARG;
    }
    if ((long long)c->n_pages * c->page_size > INT_MAX) return SPEC_ERR_SHAPE;
    const long long vecs = 2ll * c->L * c->H * (c->D / 8);
    SPEC_CUDA_TRY(launch_pdl(kv_commit_kernel, dim3((unsigned)((vecs + kCommitThreads - 1) / kCommitThreads), c->B),
                             dim3(kCommitThreads), 0, (cudaStream_t)cuda_stream, *c));
    return SPEC_OK;
}

}  // extern "C"
