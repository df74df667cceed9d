// Attention of one new token per sequence over a paged key/value cache.
//
//     O[b,h] = sum_j p_j V[b,g,j] / sum_j p_j,   p_j = exp(scale <q[b,h], K[b,g,j]>),   g = h / (H / Hkv),
//     LSE[b,h] = ln sum_j p_j,   j over the visible keys of sequence b: j < len, and with a window of W keys and s first
//     tokens that stay visible only j >= len - W or j < s.
//
// Every visible key's K and V row is read once: 4 D bytes per key and K/V head, 2 multiply-adds per value and query head.
// That is HBM-bound for every group size up to 16 query heads per K/V head, so all of the design serves the loads:
//
//   * A warp works on chunks of CK keys of one head.  The warps of a CTA take different heads of the same keys where there
//     are enough heads (a page holds its heads side by side, so a step of the CTA reads one contiguous piece of it, and no
//     warp has to wait for another), and neighbouring chunks where there are not.  Such a step is a tile; the tiles of all
//     (sequence, group of heads) pairs form one list, of which every CTA of a one-wave persistent grid takes an equal,
//     contiguous part, whatever the lengths are.  Each CTA lays the list out for itself from the device-side lengths (no
//     host copy of them, no plan to keep).  A pair inside one CTA's part is finished there; one that is cut by a border
//     leaves one fp32 partial result per CTA (at most two per CTA), and a second small kernel joins those.
//   * A few pairs of short sequences (one conversation) are a matter of latency: there a cluster of 8, 4, 2 or 1 CTAs
//     takes one pair, each an equal share of its tiles, and joins the parts through distributed shared memory: one launch, no
//     list to lay out.
//   * Each warp keeps a ring of its own in shared memory, filled by TMA boxes of up to CK rows x 128 bytes (a box lies in one
//     page), one mbarrier per stage, and no other synchronisation: 128 to 192 KB per SM are in flight.  Measured at
//     4 x 65536 keys of 8 heads x 128: per-thread 16-byte copies (cp.async) stop at 4.9 TB/s however deep the ring is, the TMA
//     reaches 6.4 TB/s, which is the card's copy rate.
//   * The products run on mma.sync m16n8k16, transposed: S^T = K Q^T (rows: 16 keys, columns: 8 query heads) and
//     O^T = V^T P^T (rows: 16 value dims).  With 8 to 16 query heads they need a few percent of its rate; a tcgen05
//     instruction takes 128 rows.  The contraction order over D, the order of the value dims and that of the keys are free:
//     a thread's 16 contiguous bytes serve two instructions, and the key order (see krow) makes the reads of the
//     128-byte-swizzled boxes free of bank conflicts for both operands.
//   * P is fed as two 16-bit parts (hi + lo), so its rounding does not show in O.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "attn_tc_common.cuh"

namespace attn_paged {

constexpr int kMaxCtas = 148;        // CTAs of the persistent grid (one per SM); sizes the workspace
constexpr int kStatusBadIndex = 13;  // ATTN_ERR_DEVICE_INDEX

// A page number, position or length that the device found out of range.  An earlier report of a timed-out wait stays.
__device__ __forceinline__ void report_bad_index(int* status) { atomicCAS(status, 0, kStatusBadIndex); }

template <int D, int GH>
struct DecodeCfg {
    static constexpr int NW = D == 256 ? 4 : 8;             // warps
    static constexpr int THREADS = NW * 32;
    static constexpr int CK = D == 64 ? 32 : 16;            // keys of a warp's chunk
    static constexpr int NPL = D / 64;                      // planes of 64 columns (128 bytes a row)
    static constexpr int PLANE = CK * 128;
    static constexpr int CHUNK_BYTES = 2 * NPL * PLANE;     // K, then V
    static constexpr int STAGE_BYTES = NW * CHUNK_BYTES;
    static constexpr int ROW = D + 4;                       // floats of a row in the merge buffer (16-byte rows, banks shifted)
    static constexpr int MERGE_BYTES = NW * GH * ROW * 4 + NW * GH * 8;
    // ring stages: three where they fit beside the merge buffer
    static constexpr int NSTAGE = 3 * STAGE_BYTES + MERGE_BYTES + 1024 + 512 <= 232448 ? 3 : 2;
    static constexpr int SMEM_BYTES = 1024 + NSTAGE * STAGE_BYTES + MERGE_BYTES + 8 * NW * NSTAGE + 16;
    static constexpr int TABLE_AT = SMEM_BYTES - 1024, TABLE_BYTES = 32 * 8;       // with common prefixes: SeqTable
    static_assert(SMEM_BYTES + (D == 256 ? 0 : TABLE_BYTES) <= 232448 && TABLE_AT % 8 == 0, "shared memory budget");
    // a partial result of one head: O [GH][D] (not normalised), then reference exponent and sum [GH][2], fp32
    static constexpr int PART_FLOATS = GH * (D + 2);
};

// What decides whether a group's common keys are worth a list of their own (see common_keys).
struct Sharing {
    int tile_tokens;            // sequences of a 128-row tile of queries
    int key_bytes;              // that plain decoding reads of a key, for all query heads of a K/V head
    int step_ns;                // a step of one tile of a list, where there are many lists
    int tile_ns;                // the same beside the kernel of the sequences' own keys
    int always;                 // no more lists than CTAs: all groups that have common keys
};

struct DecodeParams {
    const void* q;              // [B, H, D]
    void* o;
    float* lse;
    const int* block_table;
    const int* seq_lens;
    float* parts;
    int* status;
    int64_t table_stride;       // entries between the rows of block_table
    int B, H, Hkv, group, sub;  // query heads per K/V head; parts of at most 16 of them (each a head of its own from here on)
    int heads;                  // Hkv * sub
    int hpt_shift;              // log2 of the heads that a tile covers side by side (long lists); the other warps take further chunks
    int max_len;                // slots that a row of block_table covers
    int num_pages, page_shift;
    int box_shift;              // log2 of the rows of a TMA box: min(CK, page_size)
    int k_axes, v_axes;         // coordinate (1, 2 or 3) of the maps' slot, head and page axis: 2 bits each
    int window, sinks;
    float scale_log2;
    int grid;                   // CTAs of the first kernel
#ifdef ATTN_TEST_HOOKS
    int test_skip_step;         // test build only: the step of every warp whose copies are left out (-1: none)
#endif
    // PREFIX: the first keys of each group of neighbouring sequences are not worked on (attn_paged_tc.cuh), and every row leaves a
    // partial result
    const int* group_starts;    // [n_groups + 1]
    const int* prefix_lens;     // [n_groups]
    int n_groups, all_ctas;     // groups; CTAs that the two kernels share
    Sharing sharing;
    int64_t* plan;              // [2 (B + 1)], for the joining kernel (SeqPlan)
    float* rows;                // O [B * H][D], then reference exponent and sum [B * H][2], of pairs that one CTA has to itself
    int cluster;                // > 0: a cluster of so many CTAs (a power of two up to kCluster) per (sequence, head), no second kernel
};
constexpr int kCluster = 8;

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the same shared-memory address in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t map_rank(uint32_t addr, int rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 ld_cluster2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ int64_t warp_sum(int64_t x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

// Visible chunks of CK keys of one sequence: n_sink of them from key 0, then those from chunk `lo`.
struct SeqRange {
    int len, win_lo;   // keys >= win_lo are visible, and those < sinks
    int n_sink, lo, n_chunks;
};

// The common keys of a group: no more than its first sequence has, whose pages are read.
__device__ __forceinline__ int group_prefix(const int* seq_lens, int first, int prefix, int max_len) {
    const int len = __ldg(seq_lens + first);
    const int n = prefix < len ? prefix : len;
    return n < 0 ? 0 : (n > max_len ? max_len : n);
}

// PREFIX: the group that sequence b belongs to (-1: none): the last one that begins at or before it.
__device__ __forceinline__ int group_of(const int* starts, int n_groups, int b) {
    if (b < __ldg(starts) || b >= __ldg(starts + n_groups)) return -1;
    int lo = 0, hi = n_groups;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(starts + mid) <= b) lo = mid; else hi = mid;
    }
    return lo;
}

// The two kernels of a call with common prefixes run side by side, each on a part of the SMs (the second one's CTAs take the SMs that
// the first one's surplus CTAs leave at once): the first is bound by its tensor-core pipeline's latencies, the second by memory.
// Each works the parts out for itself from the lengths, in whole numbers, so both find the same.
//
// 128-key steps over so many keys, which may be 2^31 - 1.
__host__ __device__ __forceinline__ int key_steps(int keys) { return keys > 0 ? ((keys - 1) >> 7) + 1 : 0; }

// What a K/V head's lists of a group of n sequences take of one CTA, in ns: a step of one tile, and by itself each list (its fill and way out).
constexpr int kListNs = 8000;
__host__ __device__ __forceinline__ int64_t list_cost(int n, int prefix, const Sharing& s, int step_ns, int list_ns) {
    const int pairs = (n + 2 * s.tile_tokens - 1) / (2 * s.tile_tokens), tiles = 2 * pairs - (n - (pairs - 1) * 2 * s.tile_tokens <= s.tile_tokens ? 1 : 0);
    return static_cast<int64_t>(key_steps(prefix)) * tiles * step_ns + static_cast<int64_t>(pairs) * list_ns;
}
constexpr int kBusyListNs = 12000, kBusyBytesPerNs = 45;
// A CTA's memory rate, and what a pair costs by itself.  (With 2500 for a pair 1024 sequences in groups of 4 behind 2000 keys, 16 heads of 64:
// 1600 us instead of 1070, the CTAs of the own keys being the last.)
constexpr int kBytesPerNs = 40, kPairNs = 3600;

// The keys of group g that are worked on once for its n sequences; 0 where reading them for each sequence takes less: short prefixes of
// few sequences.  With all SMs at lists, memory sets a step's time, and a list by itself takes 10 to 13 us.  1024 sequences, 8 K/V heads
// of 128, without and with lists for all groups: groups of 1 behind 500 keys 378 and 1206 us, of 4 behind 150 163 and 238, of 4
// behind 500 381 and 323, of 16 361 and 156.  With no more lists than CTAs (Sharing::always) a list's CTAs have no other list to get to.
__device__ __forceinline__ int common_keys(const int* starts, const int* prefix_lens, const int* seq_lens, int g, int B, int max_len,
                                           const Sharing& s, int& n) {
    int first = __ldg(starts + g), end = __ldg(starts + g + 1);
    first = first < 0 ? 0 : (first > B ? B : first);
    end = end < first ? first : (end > B ? B : end);
    n = end - first;
    const int prefix = n > 0 ? group_prefix(seq_lens, first, __ldg(prefix_lens + g), max_len) : 0;
    if (prefix <= 0) return 0;
    return s.always || static_cast<int64_t>(n) * s.key_bytes * prefix / kBusyBytesPerNs > list_cost(n, prefix, s, s.step_ns, kBusyListNs) ? prefix : 0;
}

// PREFIX: how many first keys of sequence b the other kernel takes.
__device__ __forceinline__ int prefix_of(const int* starts, const int* prefix_lens, const int* seq_lens, int n_groups, int B, int max_len,
                                         const Sharing& s, int b) {
    const int g = group_of(starts, n_groups, b);
    int n = 0;
    return g < 0 ? 0 : common_keys(starts, prefix_lens, seq_lens, g, B, max_len, s, n);
}

// What the lists of group g take of one CTA.
__device__ __forceinline__ int64_t group_cost(const int* starts, const int* prefix_lens, const int* seq_lens, int g, int B, int max_len, int Hkv,
                                              const Sharing& s) {
    int n;
    const int prefix = common_keys(starts, prefix_lens, seq_lens, g, B, max_len, s, n);
    return prefix > 0 ? Hkv * list_cost(n, prefix, s, s.tile_ns, kListNs) : 0;
}
// CTAs of the first kernel out of `grid`, for lists that take `cost` ns, and own_bytes of keys and values of `pairs` pairs of a sequence and
// a group of heads for the second one.
__device__ __forceinline__ int prefix_ctas(int64_t cost, int64_t own_bytes, int64_t pairs, int grid) {
    if (own_bytes <= 0) return grid;
    const int64_t own = own_bytes / kBytesPerNs + pairs * kPairNs, n = (cost * grid + (cost + own) / 2) / (cost + own);
    return cost <= 0 ? 0 : (n < 1 ? 1 : (n > grid - 1 ? grid - 1 : static_cast<int>(n)));
}

// PREFIX: keys win_lo .. len - 1.
template <int CK>
__device__ __forceinline__ SeqRange visible(int len, int win_lo) {
    SeqRange r;
    r.len = len;
    r.win_lo = win_lo;
    r.lo = win_lo / CK;
    r.n_sink = 0;
    r.n_chunks = win_lo < len ? len / CK + (len % CK != 0) - r.lo : 0;
    return r;
}

template <int CK, bool PREFIX>
__device__ __forceinline__ SeqRange seq_range(const DecodeParams& p, int b) {
    SeqRange r;
    int len = p.seq_lens[b];
    len = len < 0 ? 0 : (len > p.max_len ? p.max_len : len);
    r.len = len;
    if constexpr (PREFIX) {
        const int prefix = prefix_of(p.group_starts, p.prefix_lens, p.seq_lens, p.n_groups, p.B, p.max_len, p.sharing, b);
        return visible<CK>(len, prefix < len ? prefix : len);
    }
    r.win_lo = (p.window > 0 && p.window < len) ? len - p.window : 0;
    r.lo = r.win_lo / CK;
    const int sink_chunks = p.sinks / CK + (p.sinks % CK != 0);
    r.n_sink = sink_chunks < r.lo ? sink_chunks : r.lo;
    r.n_chunks = r.n_sink + len / CK + (len % CK != 0) - r.lo;
    return r;
}

// Tiles of one sequence and group of heads; a tile has NW >> hpt_shift chunks.
template <int NW>
__device__ __forceinline__ int seq_tiles(const SeqRange& r, int hpt_shift) {
    constexpr int LOG_NW = NW == 8 ? 3 : 2;
    const int shift = LOG_NW - hpt_shift;
    return (r.n_chunks + (1 << shift) - 1) >> shift;
}

// One box of the cache: columns 64 * plane .., rows from `slot` of a page's head.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, uint32_t bar, int axes, int plane, int slot, int head, int page) {
    const int s = axes & 3, h = (axes >> 2) & 3;
    const int c1 = s == 1 ? slot : (h == 1 ? head : page);
    const int c2 = s == 2 ? slot : (h == 2 ? head : page);
    const int c3 = s == 3 ? slot : (h == 3 ? head : page);
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(64 * plane), "r"(c1), "r"(c2), "r"(c3)
        : "memory");
}

// a / b for a >= 0, b > 0: the 64-bit division takes several times as long as the 32-bit one
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// CTA c of `ctas` takes the tiles [total * c / ctas, total * (c + 1) / ctas).  No more CTAs than tiles: none is empty, so
// that a cut pair has a partial result from every CTA between its first and its last one.
__device__ __forceinline__ int cta_count(int64_t total, int grid) { return total < grid ? static_cast<int>(total) : grid; }

// The list's form follows from its length and from the parts that it cuts a pair into.  Heads side by side read whole pages
// and leave nothing to merge inside a CTA (64 sequences of up to 8192 keys, 8 heads of 128: 171 us against 205), but cut each
// pair into as many parts as there are CTAs on it, and joining those is what a short list or one of few sequences waits for
// (4 sequences of 2000 keys: 24 us against 17 with all warps on one head; 2 of 16000: 55 against 35; 16 of 2000: 34 either
// way).  So tiles side by side are taken when every CTA gets at least kLongList of them and a pair has about kFewParts parts
// at most.
constexpr int kLongList = 4, kFewParts = 10;
// With common prefixes only what the prefix leaves of each sequence is in the list, often a few keys: every pair then costs more by
// itself than by its tiles, and heads side by side are an eighth as many (64 sequences of one key behind 8192 common ones: 43 us, with
// one head per pair three times as long).
struct ListForm { int64_t total; int hpt_shift; };
template <bool PREFIX>
__device__ __forceinline__ ListForm list_form(const DecodeParams& p, int64_t total_side, int64_t total_one, int grid) {
    const int groups = p.heads >> p.hpt_shift;
    total_side *= groups;
    const bool few_parts = static_cast<int64_t>(p.B) * groups * kFewParts >= grid;
    const bool side = (PREFIX || total_side >= static_cast<int64_t>(kLongList) * grid) && few_parts;
    if (p.hpt_shift == 0 || side) return {total_side, p.hpt_shift};
    return {total_one * p.heads, 0};
}
__device__ __forceinline__ int64_t cta_begin(int64_t total, int c, int ctas) { return divide(total * c, ctas); }
__device__ __forceinline__ int cta_of_tile(int64_t total, int64_t t, int ctas) {
    return static_cast<int>(divide((t + 1) * ctas - 1, total));
}


__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}

// d += a b: m16n8k16, A row-major (a0: row lane/4, a1: row lane/4 + 8, a2 / a3: the same rows, k + 8), fp32 accumulators
template <int DTYPE>
__device__ __forceinline__ void mma16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (DTYPE == 0)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16-bit parts of a pair: hi = round(x), lo = round(x - hi)
template <int DTYPE>
__device__ __forceinline__ void split2(float x0, float x1, uint32_t& hi, uint32_t& lo) {
    hi = sm100::pack2<DTYPE>(x0, x1);
    float h0, h1;
    if constexpr (DTYPE == 0) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi));
        h0 = f.x; h1 = f.y;
    } else {
        h0 = __uint_as_float(hi << 16);
        h1 = __uint_as_float(hi & 0xffff0000u);
    }
    lo = sm100::pack2<DTYPE>(x0 - h0, x1 - h1);
}

// PREFIX: what the joining kernel needs to know about a sequence's part of the list: left in the workspace by the decode kernel's first
// CTA, [b]: {tiles in front of sequence b, tiles of one of its pairs}, behind the last sequence {tiles of the list, log2 of a tile's heads + 256 CTAs}.
struct SeqPlan {
    int64_t total, before;
    int hs, groups, n, ctas;
    static __device__ __forceinline__ SeqPlan read(const DecodeParams& p, int b) {
        const longlong2 mine = __ldcg(reinterpret_cast<const longlong2*>(p.plan) + b), all = __ldcg(reinterpret_cast<const longlong2*>(p.plan) + p.B);
        SeqPlan s;
        s.total = all.x;
        s.hs = static_cast<int>(all.y & 255);
        s.groups = p.heads >> s.hs;
        s.before = mine.x;
        s.n = static_cast<int>(mine.y);
        s.ctas = static_cast<int>(all.y >> 8);
        return s;
    }
};

// PREFIX: the visible keys of the first sequences of a CTA's part, worked out once by all of its threads: walking from one sequence to the
// next every warp would otherwise look for its group, a chain of loads (100 sequences in 3 groups, 16 heads of 64: 9 % longer).
struct SeqTable {
    static constexpr int SIZE = 32;
    const int2* at;       // shared memory: {len, win_lo}
    int first;
};

// Position in the tile list, advanced tile by tile.  Every warp of a CTA walks the same tiles; kvh and r0 are its own.
template <int NW, int CK, bool PREFIX>
struct TileWalk {
    int b, h, t, t_end;   // sequence, group of heads, tile inside the pair, tiles of the pair
    int kvh, r0;          // K/V head, first query head of the part inside its group
    int hs;               // log2 of the heads of a tile
    SeqRange r;
    SeqTable table;
    __device__ __forceinline__ void look(const DecodeParams& p) {
        if (PREFIX && b - table.first < SeqTable::SIZE) {
            const int2 x = table.at[b - table.first];
            r = visible<CK>(x.x, x.y);
        } else {
            r = seq_range<CK, PREFIX>(p, b);
        }
    }
    __device__ __forceinline__ void at(const DecodeParams& p, int hs_, int b_, int h_, int t_, const SeqTable& table_) {
        hs = hs_;
        b = b_;
        h = h_;
        t = t_;
        table = table_;
        look(p);
        t_end = seq_tiles<NW>(r, hs);
        split_head(p);
    }
    __device__ __forceinline__ void split_head(const DecodeParams& p) {
        const int head = (h << hs) + ((threadIdx.x >> 5) & ((1 << hs) - 1));
        kvh = p.sub == 1 ? head : head / p.sub;
        r0 = (head - kvh * p.sub) * 16;
    }
    // true: the next tile belongs to another pair
    __device__ __forceinline__ bool next(const DecodeParams& p, int groups) {
        if (++t < t_end) return false;
        t = 0;
        if (++h == groups) {
            h = 0;
            do {
                if (++b >= p.B) return true;      // the end of the list: not used again
                look(p);
                t_end = seq_tiles<NW>(r, hs);
            } while (t_end == 0);
        }
        split_head(p);
        return true;
    }
};

// The transpose of an 8 x 8 matrix of 16-bit values, a row of which lies on four lanes.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// P carries a factor 2^P_OFF where 16-bit floats run out of small numbers (fp16); the reference maximum may lag by 2^LAG.
template <int DTYPE> struct ExpRange { static constexpr float P_OFF = DTYPE == 0 ? 6.f : 0.f, LAG = 8.f; };

// GH: query heads of an item, 8 (up to 8 query heads per K/V head) or 16.  PREFIX: see DecodeParams; not with clusters or a window.
template <int D, int DTYPE, int GH, bool PREFIX>
__global__ void __launch_bounds__(DecodeCfg<D, GH>::THREADS, 1)
attn_paged_decode_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const DecodeParams p) {
    using C = DecodeCfg<D, GH>;
    constexpr int NW = C::NW, NSTAGE = C::NSTAGE, CK = C::CK, NPL = C::NPL;
    constexpr int NSUB = CK / 16;                   // groups of 16 keys: rows of one product
    constexpr int KI = D / 32, VI = D / 64;         // 16-byte pieces of a thread: per key row of K, per key row of V
    constexpr float P_OFF = ExpRange<DTYPE>::P_OFF, LAG = ExpRange<DTYPE>::LAG;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (sm100::smem_u32(smem_raw) & 1023u)) & 1023u);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    float* merge = reinterpret_cast<float*>(smem + NSTAGE * C::STAGE_BYTES);
    float2* merge_ml = reinterpret_cast<float2*>(merge + NW * GH * C::ROW);
    int64_t* scan = reinterpret_cast<int64_t*>(merge);       // at the beginning: [0..31] warp sums, [32..34] the start
    const uint32_t bars = sm100::smem_u32(smem) + NSTAGE * C::STAGE_BYTES + C::MERGE_BYTES;     // [warp][stage]: a chunk has arrived
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + NSTAGE * C::STAGE_BYTES + C::MERGE_BYTES + 8 * NW * NSTAGE);
    if (tid < NW * NSTAGE) {     // a thread per barrier: each fences its own
        sm100::mbar_init(bars + 8 * tid, 1);
        sm100::fence_barrier_init();
        sm100::fence_proxy_async_smem();
    }
    if (tid == 0) {
        *abort_flag = 0;
        sm100::prefetch_tensormap(&tmK);
        sm100::prefetch_tensormap(&tmV);
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    TileWalk<NW, CK, PREFIX> ld, cu;      // the copies run NSTAGE - 1 tiles ahead of the arithmetic
    int steps, hs = 0, groups = p.heads;
    const int shift = 31 - __clz(p.cluster | 1), rank = static_cast<int>(blockIdx.x) & ((1 << shift) - 1);
    if (p.cluster) {
        const int pair = static_cast<int>(blockIdx.x) >> shift, b = pair / p.heads;
        ld.at(p, 0, b, pair - b * p.heads, 0, SeqTable{nullptr, 0});
        ld.t = ld.t_end * rank >> shift;
        steps = (ld.t_end * (rank + 1) >> shift) - ld.t;
        if (pair == b * p.heads && rank == 0 && tid == 0 && p.seq_lens[b] > p.max_len) report_bad_index(p.status);
    } else {
    // ---- lay out the tile list: total tiles, and the pair and tile at which this CTA's part begins ----
    const int per = (p.B + C::THREADS - 1) / C::THREADS;     // consecutive sequences of a thread
    const int b0 = tid * per, b1 = b0 + per < p.B ? b0 + per : p.B;
    int64_t mine[2] = {0, 0};                                // tiles in either form of the list
    int64_t own = 0, cost = 0, seqs = 0;                     // PREFIX: keys of this kernel and the sequences that have any; the other one's cost
    SeqRange first_range = {};
    for (int b = b0; b < b1; ++b) {
        const SeqRange r = seq_range<CK, PREFIX>(p, b);
        if (b == b0) first_range = r;
        own += r.len - r.win_lo;
        seqs += r.len > r.win_lo ? 1 : 0;
        mine[0] += seq_tiles<NW>(r, p.hpt_shift);
        mine[1] += seq_tiles<NW>(r, 0);
        if (p.seq_lens[b] > p.max_len && blockIdx.x == 0) report_bad_index(p.status);
    }
    int64_t incl[2] = {mine[0], mine[1]};
#pragma unroll
    for (int off = 1; off < 32; off <<= 1)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const int64_t up = __shfl_up_sync(0xffffffffu, incl[f], off);
            if (lane >= off) incl[f] += up;
        }
    if (lane == 31) {
        scan[warp] = incl[0];
        scan[16 + warp] = incl[1];
    }
    int grid = p.grid;
    if constexpr (PREFIX) {
        for (int g = tid; g < p.n_groups; g += C::THREADS)
            cost += group_cost(p.group_starts, p.prefix_lens, p.seq_lens, g, p.B, p.max_len, p.Hkv, p.sharing);
        own = warp_sum(own);
        cost = warp_sum(cost);
        seqs = warp_sum(seqs);
        if (lane == 0) {
            scan[40 + warp] = own;
            scan[48 + warp] = cost;
            scan[56 + warp] = seqs;
        }
    }
    __syncthreads();
    if constexpr (PREFIX) {
        own = cost = seqs = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            own += scan[40 + w];
            cost += scan[48 + w];
            seqs += scan[56 + w];
        }
        grid = p.all_ctas - prefix_ctas(cost, own * (p.Hkv * D * 4), seqs * (p.heads >> p.hpt_shift), p.all_ctas);
        grid = grid < p.grid ? grid : p.grid;
    }
    int64_t before2[2] = {incl[0] - mine[0], incl[1] - mine[1]}, total2[2] = {0, 0};
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            if (w < warp) before2[f] += scan[16 * f + w];
            total2[f] += scan[16 * f + w];
        }
    const ListForm form = list_form<PREFIX>(p, total2[0], total2[1], grid);
    const int64_t total = form.total;
    hs = form.hpt_shift;
    groups = p.heads >> hs;
    const bool side = hs == p.hpt_shift;
    const int64_t before = side ? before2[0] : before2[1], my_tiles = side ? mine[0] : mine[1];
    const int ctas = cta_count(total, grid);
    if (PREFIX && blockIdx.x == 0) {
        longlong2* plan = reinterpret_cast<longlong2*>(p.plan);
        int64_t at = before;
        for (int b = b0; b < b1; ++b) {
            const int n = seq_tiles<NW>(b == b0 ? first_range : seq_range<CK, PREFIX>(p, b), hs);
            plan[b] = make_longlong2(at, n);
            at += n;
        }
        if (tid == 0) plan[p.B] = make_longlong2(total, hs | static_cast<int64_t>(ctas) << 8);
    }
    if (static_cast<int>(blockIdx.x) >= ctas) {
        if (PREFIX) asm volatile("griddepcontrol.wait;" ::: "memory");
        return;
    }
    const int64_t first = cta_begin(total, blockIdx.x, ctas);
    steps = static_cast<int>(cta_begin(total, blockIdx.x + 1, ctas) - first);
    // the thread whose sequences hold tile `first` finds it
    if (first >= before * groups && first < (before + my_tiles) * groups) {
        int64_t rem = first - before * groups;
        for (int b = b0; b < b1; ++b) {
            const int n = seq_tiles<NW>(b == b0 ? first_range : seq_range<CK, PREFIX>(p, b), hs);
            if (rem < static_cast<int64_t>(n) * groups) {
                scan[32] = b;
                scan[33] = rem / n;
                scan[34] = rem % n;
                break;
            }
            rem -= static_cast<int64_t>(n) * groups;
        }
    }
    __syncthreads();
    const SeqTable table{reinterpret_cast<const int2*>(smem + C::TABLE_AT), static_cast<int>(scan[32])};
    if (PREFIX) {
        for (int b = b0; b < b1; ++b)
            if (b >= table.first && b - table.first < SeqTable::SIZE) {
                const SeqRange r = b == b0 ? first_range : seq_range<CK, PREFIX>(p, b);
                reinterpret_cast<int2*>(smem + C::TABLE_AT)[b - table.first] = make_int2(r.len, r.win_lo);
            }
        __syncthreads();
    }
    ld.at(p, hs, static_cast<int>(scan[32]), static_cast<int>(scan[33]), static_cast<int>(scan[34]), table);
    }
    cu = ld;
    const int own_b = cu.b, own_kvh = cu.kvh, own_r0 = cu.r0;     // of a cluster's pair
    __syncthreads();          // the merge buffer takes over the scan's shared memory

    const uint32_t ring = sm100::smem_u32(smem) + warp * C::CHUNK_BYTES, my_bars = bars + 8 * warp * NSTAGE;
    // first key of this warp's chunk in the walk's tile; negative: no chunk
    auto chunk_key = [&](const TileWalk<NW, CK, PREFIX>& w) {
        const int ch = (w.t * NW + warp) >> hs;
        if (ch >= w.r.n_chunks) return -1;
        return (ch < w.r.n_sink ? ch : w.r.lo + ch - w.r.n_sink) * CK;
    };
    // page of key (chunk + lane % CK) of the copies' tile, where any key of its box is visible: -1: hidden, -2: not a page
    const int box = 1 << p.box_shift, slot_mask = (1 << p.page_shift) - 1;
    auto fetch_page = [&](int k0) {
        const int first_key = (k0 + (lane & (CK - 1))) & ~(box - 1);
        int page = -1;
        if (k0 >= 0 && first_key < ld.r.len && (first_key > ld.r.win_lo - box || first_key < p.sinks)) {
            page = __ldg(p.block_table + static_cast<int64_t>(ld.b) * p.table_stride + (first_key >> p.page_shift));
            if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages)) page = -2;
        }
        return page;
    };
    int loaded = 0;
    int key_next = chunk_key(ld), page_next = fetch_page(key_next);
    // visible keys of the chunks in flight, one bit per key
    uint32_t live_q[NSTAGE], phases = 0;
#pragma unroll
    for (int s = 0; s < NSTAGE; ++s) live_q[s] = 0;
    auto issue = [&](int stage, uint32_t& live_out) {
        live_out = 0;
        if (loaded < steps) {
            const int k0 = key_next, key = k0 + (lane & (CK - 1));
            int page = page_next;
            const bool seen = page >= 0 && key < ld.r.len && (key >= ld.r.win_lo || key < p.sinks);
            const uint32_t live = __ballot_sync(0xffffffffu, seen) & (CK == 32 ? 0xffffffffu : 0xffffu);
            live_out = live;
            if (live) {
                const uint32_t dst = ring + stage * C::STAGE_BYTES, bar = my_bars + 8 * stage;
                // pages that are loaded: the first lane of each box counts
                const uint32_t boxes = __ballot_sync(0xffffffffu, lane < CK && (lane & (box - 1)) == 0 && page >= 0);
                if (lane == 0) sm100::mbar_arrive_expect_tx(bar, __popc(boxes) * 2 * NPL * box * 128);
#ifdef ATTN_TEST_HOOKS
                if (loaded == p.test_skip_step) page = -1;      // this step's copies are left out
#endif
                __syncwarp();     // armed before the first copy; and every lane has read what this stage held
                for (int o0 = 0; o0 < 2 * NPL * (CK >> p.box_shift); o0 += 32) {
                    const int o = o0 + lane, row = (o / (2 * NPL)) << p.box_shift, pl = o % (2 * NPL);
                    const int pg = __shfl_sync(0xffffffffu, page, row & 31);
                    if (row < CK && pg >= 0) {
                        const bool is_v = pl >= NPL;
                        load_box(dst + pl * C::PLANE + row * 128, is_v ? &tmV : &tmK, bar, is_v ? p.v_axes : p.k_axes, is_v ? pl - NPL : pl,
                                 (k0 + row) & slot_mask, ld.kvh, pg);
                    }
                }
            }
            if (page == -2) report_bad_index(p.status);
            ld.next(p, groups);
            if (++loaded < steps) {
                key_next = chunk_key(ld);
                page_next = fetch_page(key_next);
            }
        }
    };
#pragma unroll
    for (int s = 0; s < NSTAGE - 1; ++s) issue(s, live_q[s]);

    // This lane's rows and pieces inside a 16-key group of a swizzled box (16-byte piece x of row r lies at piece x ^ (r % 8)).
    // Row g (+ 8) of a product is key krow (+ 8); with this order the eight lanes of a shared-memory phase read eight different
    // pieces for K (rows krow(2j), krow(2j+1), four pieces each) and for V (four rows, two pieces each).
    const int krow = g ^ ((g & 1) << 2), vrow0 = 2 * c, vrow1 = (2 * c + 1) ^ 4;
    const uint32_t k_off = krow * 128 + ((c ^ krow) << 4);                       // pieces c + 4: the same with bit 6 flipped
    const uint32_t v_off0 = NPL * C::PLANE + vrow0 * 128 + ((g ^ vrow0) << 4), v_off1 = NPL * C::PLANE + vrow1 * 128 + ((g ^ vrow1) << 4);

    constexpr int NT = GH / 8;            // groups of 8 query heads
    uint32_t qf[NT][KI][4];               // Q^T: this lane's 16-byte pieces of head 8 nt + g
    float acc[NT][VI][4][4];              // O^T: dims 64 i + 8 g + 2 x (+ 1: elements 2, 3) of heads 8 nt + 2 c, + 1
    float m[NT][2], l[NT][2];             // reference maximum of the raw scores and this lane's part of the sum, same heads
    auto start_pair = [&]() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int head = cu.r0 + 8 * nt + g;
            const bool used = head < p.group;
            const uint8_t* qp = static_cast<const uint8_t*>(p.q) +
                                ((static_cast<int64_t>(cu.b) * p.H + cu.kvh * p.group + (used ? head : 0)) * D + 8 * c) * 2;
#pragma unroll
            for (int i = 0; i < KI; ++i) {
                const uint4 w = __ldg(reinterpret_cast<const uint4*>(qp + i * 64));
                qf[nt][i][0] = used ? w.x : 0u;
                qf[nt][i][1] = used ? w.y : 0u;
                qf[nt][i][2] = used ? w.z : 0u;
                qf[nt][i][3] = used ? w.w : 0u;
            }
#pragma unroll
            for (int i = 0; i < VI; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[nt][i][x][e] = 0.f;
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.f;
        }
    };
    const float sc = p.scale_log2;
    start_pair();
    bool from_start = cu.t == 0;    // this CTA has the current pair from its first tile
    int n_pairs = 0;                // pairs that this CTA has left so far (0: a cut pair goes to slot 0)

    for (int s0 = 0; s0 < steps; s0 += NSTAGE) {
#pragma unroll
        for (int st = 0; st < NSTAGE; ++st) {
            const int s = s0 + st;
            if (s >= steps) break;
            __syncwarp();
            issue((st + NSTAGE - 1) % NSTAGE, live_q[(st + NSTAGE - 1) % NSTAGE]);
            uint32_t live = live_q[st];
            if (live) {
                // A copy that does not arrive ends in an error status: the rest of the loop goes on without its keys, and asks for
                // nothing more (its stage is not free).
                if (__all_sync(0xffffffffu, sm100::mbar_wait(my_bars + 8 * st, (phases >> st) & 1, abort_flag))) {
                    phases ^= 1u << st;
                } else {
                    live = 0;
                    loaded = steps;
                }
            }
            if (live) {
                const uint32_t src = ring + st * C::STAGE_BYTES;
                const bool full = live == (CK == 32 ? 0xffffffffu : 0xffffu);
                float sf[NSUB][NT][4];               // S^T: keys krow (0, 1) and krow + 8 (2, 3) of each group, heads 2 c, 2 c + 1
#pragma unroll
                for (int sub = 0; sub < NSUB; ++sub) {
                    float odd[NT][4];                // a second chain of products
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sf[sub][nt][e] = odd[nt][e] = 0.f;
#pragma unroll
                    for (int i = 0; i < KI; ++i) {
                        const uint32_t at = src + (i >> 1) * C::PLANE + sub * 2048 + ((i & 1) ? k_off ^ 64u : k_off);
                        const uint4 a = lds128(at), b = lds128(at + 1024);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma16816<DTYPE>(sf[sub][nt], a.x, b.x, a.y, b.y, qf[nt][i][0], qf[nt][i][1]);
                            mma16816<DTYPE>(odd[nt], a.z, b.z, a.w, b.w, qf[nt][i][2], qf[nt][i][3]);
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            sf[sub][nt][e] += odd[nt][e];
                            if (!full && !((live >> (16 * sub + krow + (e < 2 ? 0 : 8))) & 1)) sf[sub][nt][e] = -INFINITY;
                        }
                }
                // advance the reference maximum only when a score ran ahead of it by more than 2^LAG (or there is none yet)
                auto chunk_max = [&](float (&s)[NSUB][NT][4], int nt, int h) {
                    float x = fmaxf(s[0][nt][h], s[0][nt][2 + h]);
#pragma unroll
                    for (int sub = 1; sub < NSUB; ++sub) x = sm100::max3(x, s[sub][nt][h], s[sub][nt][2 + h]);
                    return x;
                };
                bool ahead = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        ahead |= m[nt][h] == -INFINITY || (chunk_max(sf, nt, h) - m[nt][h]) * sc > LAG;
                if (__any_sync(0xffffffffu, ahead)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float x = chunk_max(sf, nt, h);
#pragma unroll
                            for (int off = 4; off < 32; off <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
                            const float mn = fmaxf(m[nt][h], x);
                            const float alpha = m[nt][h] == -INFINITY ? 0.f : sm100::ex2_approx((m[nt][h] - mn) * sc);
                            m[nt][h] = mn;
                            l[nt][h] *= alpha;
#pragma unroll
                            for (int i = 0; i < VI; ++i)
#pragma unroll
                                for (int x4 = 0; x4 < 4; ++x4) {
                                    acc[nt][i][x4][h] *= alpha;
                                    acc[nt][i][x4][2 + h] *= alpha;
                                }
                        }
                }
                float off[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) off[nt][h] = P_OFF - (m[nt][h] == -INFINITY ? 0.f : m[nt][h] * sc);   // every score so far -inf: P = 0
#pragma unroll
                for (int sub = 0; sub < NSUB; ++sub) {
                    uint32_t hi[NT][2], lo[NT][2];   // P^T as B operand: keys vrow0, vrow1 (0) and + 8 (1) of head g
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float pr[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            pr[e] = sm100::ex2_approx(fmaf(sf[sub][nt][e], sc, off[nt][e & 1]));
                            // explicit zeros: with scale 0 the hidden scores' -inf * 0 is no number
                            if (!full) pr[e] = ((live >> (16 * sub + krow + (e < 2 ? 0 : 8))) & 1) ? pr[e] : 0.f;
                        }
                        l[nt][0] += pr[0] + pr[2];
                        l[nt][1] += pr[1] + pr[3];
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            uint32_t a, b;
                            split2<DTYPE>(pr[2 * n], pr[2 * n + 1], a, b);
                            hi[nt][n] = transpose8x8(a);
                            lo[nt][n] = transpose8x8(b);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < VI; ++i) {
                        const uint32_t at = src + i * C::PLANE + sub * 2048;
                        uint4 v[4] = {lds128(at + v_off0), lds128(at + v_off1), lds128(at + v_off0 + 1024), lds128(at + v_off1 + 1024)};
                        if (!full) {     // hidden slots may hold anything, infinities and NaN among it
#pragma unroll
                            for (int n = 0; n < 4; ++n)
                                if (!((live >> (16 * sub + ((n & 1) ? vrow1 : vrow0) + 8 * (n >> 1))) & 1)) v[n] = make_uint4(0u, 0u, 0u, 0u);
                        }
                        const uint32_t w[4][4] = {{v[0].x, v[0].y, v[0].z, v[0].w}, {v[1].x, v[1].y, v[1].z, v[1].w},
                                                  {v[2].x, v[2].y, v[2].z, v[2].w}, {v[3].x, v[3].y, v[3].z, v[3].w}};
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            // V^T: dims 2 x and 2 x + 1 of this lane's 8 as rows g and g + 8, key pairs side by side
                            const uint32_t a0 = __byte_perm(w[0][x], w[1][x], 0x5410), a1 = __byte_perm(w[0][x], w[1][x], 0x7632);
                            const uint32_t a2 = __byte_perm(w[2][x], w[3][x], 0x5410), a3 = __byte_perm(w[2][x], w[3][x], 0x7632);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma16816<DTYPE>(acc[nt][i][x], a0, a1, a2, a3, hi[nt][0], hi[nt][1]);
                                mma16816<DTYPE>(acc[nt][i][x], a0, a1, a2, a3, lo[nt][0], lo[nt][1]);
                            }
                        }
                    }
                }
            }
            // ---- end of the pair, or of this CTA's part ----
            const bool end_pair = cu.t + 1 == cu.t_end;
            if (end_pair || s + 1 == steps) {
                const bool whole = end_pair && from_start && !p.cluster;
                const int hpt = 1 << hs;
                float* part = p.parts + (2 * static_cast<int64_t>(blockIdx.x) + (n_pairs > 0 ? 1 : 0)) * hpt * C::PART_FLOATS;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) l[nt][h] += __shfl_xor_sync(0xffffffffu, l[nt][h], o);
                if (hpt == NW) {
                    // every warp has a head to itself: straight from the registers, 8 contiguous dims per lane and plane
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int row = 8 * nt + 2 * c + h;
                            if (cu.r0 + row >= p.group) continue;
                            const float mm = m[nt][h] * sc, sum = l[nt][h];      // sum 0: no key, mm is not used
                            const int64_t out_row = static_cast<int64_t>(cu.b) * p.H + cu.kvh * p.group + cu.r0 + row;
                            if (whole && !PREFIX) {
                                const float inv = sum != 0.f ? 1.f / sum : 0.f;
                                uint8_t* dst = static_cast<uint8_t*>(p.o) + (out_row * D + 8 * g) * 2;
#pragma unroll
                                for (int i = 0; i < VI; ++i) {
                                    uint32_t w[4];
#pragma unroll
                                    for (int x = 0; x < 4; ++x) w[x] = sm100::pack2<DTYPE>(acc[nt][i][x][h] * inv, acc[nt][i][x][2 + h] * inv);
                                    *reinterpret_cast<uint4*>(dst + 128 * i) = make_uint4(w[0], w[1], w[2], w[3]);
                                }
                                if (g == 0) p.lse[out_row] = sum != 0.f ? (mm - P_OFF) * 0.6931471805599453f + logf(sum) : -INFINITY;
                            } else {
                                float* dst = part + warp * C::PART_FLOATS + row * D;
                                float* ml = part + warp * C::PART_FLOATS + GH * D + 2 * row;
                                if (PREFIX && whole) {
                                    dst = p.rows + out_row * D;
                                    ml = p.rows + static_cast<int64_t>(p.B) * p.H * D + 2 * out_row;
                                }
#pragma unroll
                                for (int i = 0; i < VI; ++i)
#pragma unroll
                                    for (int x = 0; x < 4; x += 2)
                                        *reinterpret_cast<float4*>(dst + 64 * i + 8 * g + 2 * x) =
                                            make_float4(acc[nt][i][x][h], acc[nt][i][x][2 + h], acc[nt][i][x + 1][h], acc[nt][i][x + 1][2 + h]);
                                if (g == 0) *reinterpret_cast<float2*>(ml) = make_float2(mm, sum);
                            }
                        }
                } else {
                    // several warps share a head: through shared memory
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int row = 8 * nt + 2 * c + h;
                            if (g == 0) merge_ml[warp * GH + row] = make_float2(m[nt][h] * sc, l[nt][h]);
                            float* dst = merge + (warp * GH + row) * C::ROW + 8 * g;
#pragma unroll
                            for (int i = 0; i < VI; ++i)
#pragma unroll
                                for (int x = 0; x < 4; x += 2)
                                    *reinterpret_cast<float4*>(dst + 64 * i + 2 * x) =
                                        make_float4(acc[nt][i][x][h], acc[nt][i][x][2 + h], acc[nt][i][x + 1][h], acc[nt][i][x + 1][2 + h]);
                        }
                    __syncthreads();
                    const int rows = p.group < GH ? p.group : GH;         // of a head; the last part of a group may have fewer
                    for (int e = tid; e < hpt * rows * (D / 4); e += C::THREADS) {
                        const int d4 = e % (D / 4), x = e / (D / 4), row = x % rows, hh = x / rows;
                        const int head = (cu.h << hs) + hh, kvh = head / p.sub, r0 = (head - kvh * p.sub) * 16;
                        if (r0 + row >= p.group) continue;
                        float mm = -INFINITY;
                        for (int w = hh; w < NW; w += hpt) {
                            const float2 ml = merge_ml[w * GH + row];
                            if (ml.y != 0.f) mm = fmaxf(mm, ml.x);
                        }
                        float sum = 0.f;
                        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
                        for (int w = hh; w < NW; w += hpt) {
                            const float2 ml = merge_ml[w * GH + row];
                            if (ml.y == 0.f) continue;       // this warp saw no key of the pair
                            const float f = sm100::ex2_approx(ml.x - mm);
                            const float4 v = *reinterpret_cast<const float4*>(merge + (w * GH + row) * C::ROW + 4 * d4);
                            sum = fmaf(f, ml.y, sum);
                            o.x = fmaf(f, v.x, o.x);
                            o.y = fmaf(f, v.y, o.y);
                            o.z = fmaf(f, v.z, o.z);
                            o.w = fmaf(f, v.w, o.w);
                        }
                        const int64_t out_row = static_cast<int64_t>(cu.b) * p.H + kvh * p.group + r0 + row;
                        if (whole && !PREFIX) {
                            const float inv = sum != 0.f ? 1.f / sum : 0.f;
                            uint2 w;
                            w.x = sm100::pack2<DTYPE>(o.x * inv, o.y * inv);
                            w.y = sm100::pack2<DTYPE>(o.z * inv, o.w * inv);
                            reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.o) + out_row * D * 2)[d4] = w;
                            if (d4 == 0) p.lse[out_row] = sum != 0.f ? (mm - P_OFF) * 0.6931471805599453f + logf(sum) : -INFINITY;
                        } else {
                            // (a cluster's parts stay in shared memory, in the ring: every copy into it has been waited for)
                            float* dst = p.cluster ? reinterpret_cast<float*>(smem) : part + hh * C::PART_FLOATS;
                            float* ml = dst + GH * D + 2 * row;
                            dst += row * D;
                            if (PREFIX && whole) {
                                dst = p.rows + out_row * D;
                                ml = p.rows + static_cast<int64_t>(p.B) * p.H * D + 2 * out_row;
                            }
                            *reinterpret_cast<float4*>(dst + 4 * d4) = o;
                            if (d4 == 0) *reinterpret_cast<float2*>(ml) = make_float2(mm, sum);
                        }
                    }
                    __syncthreads();     // the merge buffer may be written again
                }
                ++n_pairs;
            }
            if (cu.next(p, groups) && s + 1 < steps) {
                start_pair();
                from_start = true;
            }
        }
    }
    __syncthreads();
    if (tid == 0 && *abort_flag != 0) attn_tc::report_timeout(p.status);
    // the end of this kernel stands for the end of the one on the common keys, too
    if (PREFIX) asm volatile("griddepcontrol.wait;" ::: "memory");
    if (p.cluster) {
        float* mine = reinterpret_cast<float*>(smem);
        if (steps == 0)
            for (int row = tid; row < GH; row += C::THREADS) *reinterpret_cast<float2*>(mine + GH * D + 2 * row) = make_float2(-INFINITY, 0.f);
        cluster_sync();
        // every p.cluster-th row of the pair from `rank`: this CTA joins it, a thread per 16-byte column
        const int rows = p.group - own_r0 < GH ? p.group - own_r0 : GH;
        const uint32_t base = sm100::smem_u32(smem);
        for (int row = rank; row < rows; row += p.cluster) {
            for (int d4 = tid; d4 < D / 4; d4 += C::THREADS) {
                float2 ml[kCluster];
                float4 v[kCluster];
#pragma unroll
                for (int k = 0; k < kCluster; ++k) {
                    ml[k] = make_float2(-INFINITY, 0.f);
                    v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (k >= p.cluster) continue;
                    const uint32_t from = map_rank(base, k);
                    ml[k] = ld_cluster2(from + (GH * D + 2 * row) * 4);
                    v[k] = ld_cluster4(from + (row * D + 4 * d4) * 4);
                }
                float mm = -INFINITY, sum = 0.f;
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int k = 0; k < kCluster; ++k)
                    if (ml[k].y != 0.f) mm = fmaxf(mm, ml[k].x);
#pragma unroll
                for (int k = 0; k < kCluster; ++k) {
                    if (ml[k].y == 0.f) continue;        // no key of the pair (its O is not set)
                    const float f = sm100::ex2_approx(ml[k].x - mm);
                    sum = fmaf(f, ml[k].y, sum);
                    o.x = fmaf(f, v[k].x, o.x);
                    o.y = fmaf(f, v[k].y, o.y);
                    o.z = fmaf(f, v[k].z, o.z);
                    o.w = fmaf(f, v[k].w, o.w);
                }
                const int64_t out_row = static_cast<int64_t>(own_b) * p.H + own_kvh * p.group + own_r0 + row;
                const float inv = sum != 0.f ? 1.f / sum : 0.f;
                uint2 w;
                w.x = sm100::pack2<DTYPE>(o.x * inv, o.y * inv);
                w.y = sm100::pack2<DTYPE>(o.z * inv, o.w * inv);
                reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.o) + out_row * D * 2)[d4] = w;
                if (d4 == 0) p.lse[out_row] = sum != 0.f ? (mm - P_OFF) * 0.6931471805599453f + logf(sum) : -INFINITY;
            }
        }
        cluster_sync();      // a peer may still read this CTA's part
    }
}

// One row (sequence and query head) out of np partial results, by one warp: ml_of(i) gives part i's reference exponent, which stands
// p_off too high, and its sum; row_of(i) its O.  The order of the parts is fixed.
template <int D, int DTYPE, class MlOf, class RowOf>
__device__ __forceinline__ void join_row(int np, int lane, float p_off, MlOf ml_of, RowOf row_of, void* out, float* lse) {
    constexpr int COLS = D / 4;                            // 16-byte columns of a partial row
    constexpr int TEAMS = COLS >= 32 ? 1 : 32 / COLS, PER = COLS >= 32 ? COLS / 32 : 1;
    // up to 32 parts at a time: a row of more is joined in rounds, like the rounds of an online softmax
    float mm = -INFINITY, sum = 0.f;
    float4 o[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    const int team = TEAMS > 1 ? lane / COLS : 0, col = TEAMS > 1 ? lane % COLS : lane;
    constexpr int BATCH = PER > 1 ? 4 : 8;                 // rows of a lane in flight
    for (int i0 = 0; i0 < np; i0 += 32) {
        const int m = np - i0 < 32 ? np - i0 : 32;
        float2 ml = make_float2(-INFINITY, 0.f);
        if (lane < m) ml = __ldcg(ml_of(i0 + lane));
        float4 v[BATCH][PER];
        auto load = [&](int x0) {
#pragma unroll
            for (int x = 0; x < BATCH; ++x) {
                const int i = x0 + x * TEAMS;
                if (i >= m) break;
                const int mine = i + team < m ? i + team : m - 1;            // (a weight of 0 below for the repeated one)
                const float4* src = reinterpret_cast<const float4*>(row_of(i0 + mine));
#pragma unroll
                for (int k = 0; k < PER; ++k) v[x][k] = __ldcg(src + col + 32 * k);
            }
        };
        load(0);                                           // on their way while the weights are worked out
        float mx = ml.y != 0.f ? ml.x : -INFINITY;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
        const float mn = fmaxf(mm, mx);
        const float keep = mm == -INFINITY ? 0.f : sm100::ex2_approx(mm - mn);
        const float f = ml.y != 0.f ? sm100::ex2_approx(ml.x - mn) : 0.f;
        float part_sum = f * ml.y;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) part_sum += __shfl_xor_sync(0xffffffffu, part_sum, off);
        sum = fmaf(sum, keep, part_sum);
        mm = mn;
#pragma unroll
        for (int k = 0; k < PER; ++k) { o[k].x *= keep; o[k].y *= keep; o[k].z *= keep; o[k].w *= keep; }
        for (int x0 = 0; x0 < m; x0 += BATCH * TEAMS) {
            if (x0 > 0) load(x0);
#pragma unroll
            for (int x = 0; x < BATCH; ++x) {
                const int i = x0 + x * TEAMS;
                if (i >= m) break;
                float w = __shfl_sync(0xffffffffu, f, i + team < m ? i + team : m - 1);
                if (i + team >= m) w = 0.f;
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (w != 0.f) {     // a part without a visible key adds nothing
                        o[k].x = fmaf(w, v[x][k].x, o[k].x);
                        o[k].y = fmaf(w, v[x][k].y, o[k].y);
                        o[k].z = fmaf(w, v[x][k].z, o[k].z);
                        o[k].w = fmaf(w, v[x][k].w, o[k].w);
                    }
            }
        }
    }
    if constexpr (TEAMS > 1) {
#pragma unroll
        for (int off = COLS; off < 32; off <<= 1) {
            o[0].x += __shfl_xor_sync(0xffffffffu, o[0].x, off);
            o[0].y += __shfl_xor_sync(0xffffffffu, o[0].y, off);
            o[0].z += __shfl_xor_sync(0xffffffffu, o[0].z, off);
            o[0].w += __shfl_xor_sync(0xffffffffu, o[0].w, off);
        }
    }
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    if (team == 0) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            uint2 w;
            w.x = sm100::pack2<DTYPE>(o[k].x * inv, o[k].y * inv);
            w.y = sm100::pack2<DTYPE>(o[k].z * inv, o[k].w * inv);
            reinterpret_cast<uint2*>(out)[col + 32 * k] = w;
        }
    }
    if (lane == 0) *lse = sum != 0.f ? (mm - p_off) * 0.6931471805599453f + logf(sum) : -INFINITY;
}

constexpr int kJoinWarps = 8;
// A row without a visible key.
template <int D>
__device__ __forceinline__ void empty_row(void* out, float* lse, int lane) {
    for (int e = lane; e < D / 4; e += 32) static_cast<uint2*>(out)[e] = make_uint2(0u, 0u);
    if (lane == 0) *lse = -INFINITY;
}

// Where the partial results of one sequence's heads lie: worked out by a whole block of kJoinWarps warps from the lengths.
template <int D, int GH>
struct JoinList {
    using C = DecodeCfg<D, GH>;
    int64_t total, before;     // tiles of the list, and of the sequences in front
    int hs, groups, n, ctas;   // log2 of a tile's heads, groups of heads, tiles of a pair of this sequence
    __device__ __forceinline__ JoinList(const DecodeParams& p, int b, int64_t (*red)[kJoinWarps]) {
        constexpr int NW = C::NW;
        const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
        int64_t sum4[4] = {0, 0, 0, 0};                    // tiles of the sequences before b and of all, in either form of the list
        for (int x = tid; x < p.B; x += kJoinWarps * 32) {
            const SeqRange r = seq_range<C::CK, false>(p, x);
            const int n0 = seq_tiles<NW>(r, p.hpt_shift), n1 = seq_tiles<NW>(r, 0);
            sum4[2] += n0;
            sum4[3] += n1;
            if (x < b) {
                sum4[0] += n0;
                sum4[1] += n1;
            }
        }
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            sum4[f] = warp_sum(sum4[f]);
            if (lane == 0) red[f][warp] = sum4[f];
        }
        __syncthreads();
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            sum4[f] = 0;
#pragma unroll
            for (int w = 0; w < kJoinWarps; ++w) sum4[f] += red[f][w];
        }
        const ListForm form = list_form<false>(p, sum4[2], sum4[3], p.grid);
        total = form.total;
        hs = form.hpt_shift;
        groups = p.heads >> hs;
        before = hs == p.hpt_shift ? sum4[0] : sum4[1];
        n = seq_tiles<NW>(seq_range<C::CK, false>(p, b), hs);
        ctas = cta_count(total, p.grid);
    }
};

// The parts of one row: head (of the K/V heads' parts of at most 16 query heads) and row of the pair.
struct RowParts {
    int count = 0;             // 1: one CTA has the pair to itself; 0: no keys
    int c0 = 0, hs = 0, hh = 0, head = 0, row = 0;
    bool odd = false;          // the pair is not c0's first (it is that of every CTA behind c0)
    template <class List>
    __device__ __forceinline__ void find(const DecodeParams& p, const List& l, int q_head) {       // (l.n > 0)
        const int kvh = q_head / p.group, in_group = q_head - kvh * p.group;
        row = in_group & 15;
        head = kvh * p.sub + (in_group >> 4);
        hs = l.hs;
        const int hg = head >> hs;
        hh = head - (hg << hs);
        const int64_t t0 = l.before * l.groups + static_cast<int64_t>(hg) * l.n, t1 = t0 + l.n;
        c0 = cta_of_tile(l.total, t0, l.ctas);
        count = cta_of_tile(l.total, t1 - 1, l.ctas) - c0 + 1;
        odd = cta_begin(l.total, c0, l.ctas) < t0;
    }
    template <int PART_FLOATS>
    __device__ __forceinline__ const float* at(const DecodeParams& p, int i) const {
        const int64_t slot = i == 0 ? 2 * c0 + (odd ? 1 : 0) : 2 * (c0 + i);
        return p.parts + ((slot << hs) + hh) * PART_FLOATS;
    }
};

// Joins the partial results of the pairs that more than one CTA of the first kernel worked on, and writes the rows of
// sequences without a visible key.  A warp per row (sequence and query head), eight rows of one sequence to a block; the
// list layout is worked out before the first kernel's results are waited for, and after that a row takes two dependent rounds
// of loads: the parts' exponents and sums, one per lane, then their rows.
template <int D, int DTYPE, int GH>
__global__ void __launch_bounds__(kJoinWarps * 32)
attn_paged_join_kernel(const DecodeParams p, int blocks_per_seq) {
    using C = DecodeCfg<D, GH>;
    constexpr float P_OFF = ExpRange<DTYPE>::P_OFF;
    __shared__ int64_t red[4][kJoinWarps];
    const int b = blockIdx.x / blocks_per_seq, lane = threadIdx.x & 31;
    const int q_head = (blockIdx.x - b * blocks_per_seq) * kJoinWarps + (threadIdx.x >> 5);
    const JoinList<D, GH> list(p, b, red);
    // Every block waits for the first kernel, also one without work: in a graph this kernel's end stands for both.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (q_head >= p.H) return;
    const int64_t out_row = static_cast<int64_t>(b) * p.H + q_head;
    uint8_t* out = static_cast<uint8_t*>(p.o) + out_row * D * 2;
    if (list.n == 0) {
        empty_row<D>(out, p.lse + out_row, lane);
        return;
    }
    RowParts parts;
    parts.find(p, list, q_head);
    if (parts.count == 1) return;                // finished by the first kernel
    auto part = [&](int i) { return parts.at<C::PART_FLOATS>(p, i); };
    join_row<D, DTYPE>(parts.count, lane, P_OFF, [&](int i) { return reinterpret_cast<const float2*>(part(i) + GH * D) + parts.row; },
                       [&](int i) { return part(i) + parts.row * D; }, out, p.lse + out_row);
}

}  // namespace attn_paged
