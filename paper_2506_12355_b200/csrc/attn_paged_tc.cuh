// Attention of many query rows over the paged cache on the tensor cores (tcgen05), in two forms:
//
//   prefill (PREFIX = false): the n new tokens of each sequence of length len; token i sees the keys j <= len - n + i.
//   prefix  (PREFIX = true):  one new token per sequence, and only the first P keys, which the sequences of a group have in common:
//                             a token sees the keys j < min(P, its sequence's length).  K and V of the prefix are read once for
//                             all rows of the group; attn_paged.cuh adds each sequence's other keys.
//
//     O = sum_j p_j V_j / sum_j p_j,   p_j = exp(scale <q, K_j>),   LSE = ln sum_j p_j
//
// A list is one K/V head and a pair of 128-row tiles of queries; row r of a tile is query head r % G of the K/V head's G, of token
// r / G (128 / G tokens to a tile, rounded down), which a TMA box brings in that order from [token][head][D].  Its steps are the
// 128-key tiles that its last token sees.  The steps of all lists, one after the other, each weighted by what it takes and each list
// with kListCost more for its fill and way out, are cut evenly over one CTA per SM, whatever the lengths are (each CTA works out its own
// part from the device-side lengths: no host copy, no plan to keep); a list that a border cuts leaves a partial result per CTA (at most
// two per CTA, fp32), which a second kernel joins in a fixed order.  (8 prompts of 100 - 4000 tokens, 16 heads of 64: 230 us; without
// kListCost 260, with all steps alike 243.  Prompts of up to 2000 tokens, 32 heads over 8 of 128: 172; without kListCost 197.)
//
// Inside a CTA it is the pipeline of attn_tc_pipe.cuh: TMA ring of K/V tiles, one MMA-issuing warp, two softmax groups in
// ping-pong, P back into tensor memory as the second product's operand, a lagging reference maximum.  What paging adds:
//   * A tile is 128 / page_size boxes per 64 columns, issued by as many lanes of a warp, K's by one warp and V's by another (a box
//     costs its warp about 95 cycles; one warp for both: 2048 tokens behind 14336 in pages of 16 507 us, of 8 706, two: 410 either
//     way); page numbers are read a step ahead.
//   * Slots that hold no key of the sequence (behind its end, or in a page whose number is out of range) may hold anything: their
//     scores are overwritten with -inf before the softmax, and their V rows with zeros before the product (0 * NaN is no number).
//   * A list of one tile (few query rows: a prefix call's usual case) keeps both softmax groups busy: its rows are in both Q tiles,
//     one takes the even steps and one the odd ones, and the epilogue adds up the two accumulators in tensor memory.
//   * All exponentials on the special-function unit, as under a window: rows may see only a few keys.
// Prefill: P is rounded to the type of Q, K and V before its product and the row sums add the unrounded values (see attn_tc_pipe.cuh).
// Prefix: P goes into its product in two 16-bit parts, as in attn_paged.cuh, so that a key counts the same whether it is read as a common
// one or not (rounded once, O was off by 2.3e-3 of its 2-norm in bf16 where its own rounding is 1.66e-3); the second parts lie in the
// other half of S's columns.
//
// What bounds it: a step of two tiles takes 1.9 us at D = 128 (1024 tensor cycles a tile, 1.25 PFLOP/s of visible pairs for the 2048
// tokens above) and 1.7 at D = 64 (its exponentials), a step of one tile 1.0; a list costs 5 us beside its steps (the way out 2.3,
// then the next list's first scores), and the first scores are there 7 us after the start, most of it instructions that come from L2.
// Prefix, all SMs at K and V that come from HBM: a step of two tiles 2.4 us, 1.9 at D = 64, of one 1.75 and 1.3 (with P rounded once: 2.0, 1.55,
// 1.4, 1.0).
#pragma once
#include "attn_paged.cuh"
#include "attn_tc_common.cuh"

namespace attn_paged_tc {

using namespace sm100;
using attn_paged::cta_begin;
using attn_paged::cta_count;
using attn_paged::cta_of_tile;
using attn_paged::divide;
using attn_paged::key_steps;
using attn_paged::report_bad_index;
using attn_tc::low_bits;

constexpr int kRows = 256;                        // rows of a list: two tiles
constexpr int kListCost = 4;                      // what a list costs beside its steps (see step_weight), about 4 us

template <int D>
struct Cfg {
    static constexpr int NBOX = D / 64;           // 64-column boxes (128 bytes a row)
    static constexpr int Q_BYTES = 128 * D * 2, KV_BYTES = 128 * D * 2;
    static constexpr int NSLOT = D == 128 ? 4 : 8, NGRP = NSLOT / 2;      // ring slots; a group is V_j and K_{j+1}
    static constexpr int OST_BYTES = 128 * 128;   // staging of a tile's output, 128 bytes a row
    static constexpr int TILE_BYTES = 2 * Q_BYTES + NSLOT * KV_BYTES + 2 * OST_BYTES;
    static constexpr int MISC_BYTES = 2048;
    static constexpr int SMEM_BYTES = 1024 + TILE_BYTES + MISC_BYTES;
    static constexpr int THREADS = 384, TMEM_COLS = 512;
    __host__ __device__ static constexpr int s_col(int t) { return t * 128; }
    __host__ __device__ static constexpr int o_col(int t) { return 256 + t * D; }
    static_assert(SMEM_BYTES <= 232448, "shared memory budget");
};

// floats of one partial result: O [256][D] (not normalised), then reference exponent and sum [256][2]
__host__ __device__ constexpr int64_t part_floats(int D) { return static_cast<int64_t>(kRows) * (D + 2); }

// What the joining kernels need to know about the lists, left in the workspace by the kernel that has worked it out.
struct Cut { int parts[2], tok, n_tok, kvh; };     // partial results of each tile (0: none)
struct PrefixPlan {
    int64_t start, stride;      // where step 0 of the sequence's list of K/V head 0 lies, and weight per head.  Behind the last sequence: the
                                // weight of all lists, and the CTAs that share it
    int64_t span;               // from step 0 to the last one (-1: no common keys)
    int row;                    // row of query head 0 of a K/V head
};

struct Params {
    void* o;                    // prefill: [tokens, H, D] and lse [tokens, H]
    float* lse;
    float* parts;               // [2 per CTA] partial results of lists that a border cuts
    Cut* cuts;                  // prefill: [CTA], the list whose first border lies behind the CTA
    PrefixPlan* plan;           // prefix: [tokens + 1]
    float* rows;                // prefix: O [tokens * H][D], then [tokens * H][2], of lists that one CTA has to itself
    const int* block_table;
    const int* seq_lens;
    const int* starts;          // [units + 1]: first token of each sequence (prefill), first sequence of each group (prefix)
    const int* prefix_lens;     // prefix: [units]
    int64_t table_stride;
    int units, tokens;          // sequences and their new tokens; groups and sequences
    int H, Hkv, group, tile_tokens;
    int twin_weight;            // of a step of one tile
    int max_len, num_pages, page_shift, box_shift, k_axes, v_axes;
    float scale, scale_log2;
    attn_paged::Sharing sharing;
    int row_bytes, head_groups; // prefix: of a key, K and V of all heads; groups of heads of a pair of the other kernel
    int grid;
    int* status;
#ifdef ATTN_TEST_HOOKS
    int test_skip_group;        // test build only: the ring group of every CTA whose copies are left out (-1: none)
#endif
};

// sum over i < n of floor((a i + b) / 128)
__host__ __device__ __forceinline__ int64_t floor_sum(uint32_t n, uint32_t a, uint32_t b) {
    uint32_t m = 128;
    int64_t sum = 0;
    while (n > 0) {
        sum += static_cast<int64_t>(n) * (n - 1) / 2 * (a / m) + static_cast<int64_t>(n) * (b / m);
        a %= m;
        b %= m;
        const uint64_t y = static_cast<uint64_t>(a) * n + b;
        if (y < m) break;
        n = static_cast<uint32_t>(y / m);
        b = static_cast<uint32_t>(y % m);
        const uint32_t x = m;
        m = a;
        a = x;
    }
    return sum;
}

// One sequence (prefill) or group (prefix).
template <bool PREFIX>
struct Unit {
    int tok0, n;       // its query tokens
    int base;          // prefill: the last key that token 0 sees
    int len;           // keys
    int pairs;
    __device__ __forceinline__ void load(const Params& p, int u) {
        tok0 = __ldg(p.starts + u);
        int end = __ldg(p.starts + u + 1);
        tok0 = tok0 < 0 ? 0 : (tok0 > p.tokens ? p.tokens : tok0);
        end = end < tok0 ? tok0 : (end > p.tokens ? p.tokens : end);
        n = end - tok0;
        if constexpr (PREFIX) {
            len = attn_paged::common_keys(p.starts, p.prefix_lens, p.seq_lens, u, p.tokens, p.max_len, p.sharing, n);
            base = 0;
        } else {
            len = __ldg(p.seq_lens + u);
            len = len > p.max_len ? p.max_len : len;
            base = len - n;
        }
        if (len <= 0) n = 0;
        const int t2 = 2 * p.tile_tokens;
        pairs = (n + t2 - 1) / t2;
    }
    // that of another lane of the warp
    __device__ __forceinline__ void from_lane(int lane) {
        tok0 = __shfl_sync(0xffffffffu, tok0, lane);
        n = __shfl_sync(0xffffffffu, n, lane);
        base = __shfl_sync(0xffffffffu, base, lane);
        len = __shfl_sync(0xffffffffu, len, lane);
        pairs = __shfl_sync(0xffffffffu, pairs, lane);
    }
    // steps of the first `tokens` query tokens (at least one, also where none of them sees a key)
    __host__ __device__ __forceinline__ int steps_of(int tokens) const {
        if (PREFIX) return key_steps(len);
        return ((base > 0 ? base : 0) + (tokens < n ? tokens : n) - 1) / 128 + 1;
    }
    __host__ __device__ __forceinline__ int pair_steps(const Params& p, int i) const { return steps_of((i + 1) * 2 * p.tile_tokens); }
    // Weights, in units of about 1 us: a step of two tiles counts 2, one of one tile (the last pair may have no more) as much at D = 128,
    // where it waits for the same K and V (with weight 1 32 prompts of 10 - 200 tokens behind 4096, 32 heads over 8: 330 us instead of
    // 277), and 1 at D = 64; each list counts kListCost more.
    __host__ __device__ __forceinline__ int step_weight(const Params& p, int i) const {
        return i == pairs - 1 && n - i * 2 * p.tile_tokens <= p.tile_tokens ? p.twin_weight : 2;
    }
    __host__ __device__ __forceinline__ int64_t weight_before(const Params& p, int i) const {
        const int t2 = 2 * p.tile_tokens, full = i < pairs ? i : pairs - 1;      // the last pair has a weight of its own
        if (i == 0) return 0;
        const int64_t steps = PREFIX ? static_cast<int64_t>(full) * key_steps(len)
                                     : floor_sum(full, t2, static_cast<uint32_t>(base > 0 ? base : 0) + t2 - 1) + full;
        return 2 * steps + static_cast<int64_t>(i) * kListCost + (i == pairs ? static_cast<int64_t>(step_weight(p, i - 1)) * steps_of(n) : 0);
    }
    __host__ __device__ __forceinline__ int64_t head_weight(const Params& p) const { return weight_before(p, pairs); }
};

// Position in the lists: unit, K/V head, pair, and how far into the pair's list in weights (what the list costs beside its steps comes
// first; a step belongs to whom its first weight does).  All lanes of a warp hold the same one.
template <bool PREFIX>
struct Walk {
    Unit<PREFIX> unit;
    int u, h, i, steps, weight;
    int64_t at;
    int64_t mine, before;      // weight of this lane's units (consecutive ones) and of those in front of them
    int per, first;            // units of a lane, and this lane's first
    // The total weight of all lists (prefix: after plan_sums()); all 32 lanes.
    __device__ __forceinline__ int64_t total(const Params& p, int lane, const volatile int64_t* sums) {
        per = (p.units + 31) / 32;
        first = lane * per;
        if constexpr (PREFIX) {
            mine = sums[lane];
        } else {
            const int end = first + per < p.units ? first + per : p.units;
            mine = 0;
            for (int x = first; x < end; ++x) {
                unit.load(p, x);
                mine += p.Hkv * unit.head_weight(p);
            }
        }
        before = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int64_t up = __shfl_up_sync(0xffffffffu, before, off);
            if (lane >= off) before += up;
        }
        const int64_t all = __shfl_sync(0xffffffffu, before, 31);
        before -= mine;
        return all;
    }
    // The CTAs that share the lists: of a prefix call those that prefix_ctas() gives it.
    static __device__ __forceinline__ int ctas(const Params& p, int64_t total, const volatile int64_t* sums) {
        const int n = PREFIX ? attn_paged::prefix_ctas(sums[32], sums[33] * p.row_bytes, sums[34] * p.head_groups, p.grid) : p.grid;
        // (a CTA's part holds the beginning of a step: two weights at least)
        return cta_count(total / 2, n);
    }
    // Position `pos` of all (below the total), after total().
    __device__ __forceinline__ void find(const Params& p, int lane, int64_t pos) {
        const bool here = pos >= before && pos < before + mine;
        const int owner = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
        int64_t rem = pos - before;
        if constexpr (PREFIX) {                        // 32 of the owner's units at a time
            rem = __shfl_sync(0xffffffffu, rem, owner);
            const int end = (owner + 1) * per < p.units ? (owner + 1) * per : p.units;
            for (u = owner * per;; u += 32) {
                int64_t n = 0;
                if (u + lane < end) {
                    unit.load(p, u + lane);
                    n = p.Hkv * unit.head_weight(p);
                }
                int64_t incl = n;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const int64_t up = __shfl_up_sync(0xffffffffu, incl, off);
                    if (lane >= off) incl += up;
                }
                const unsigned hit = __ballot_sync(0xffffffffu, rem < incl);
                if (hit != 0u) {
                    const int at = __ffs(hit) - 1;
                    rem -= __shfl_sync(0xffffffffu, incl - n, at);
                    unit.from_lane(at);
                    u += at;
                    break;
                }
                rem -= __shfl_sync(0xffffffffu, incl, 31);
            }
        } else {
            int x = first;
            if (here && per > 1)
                for (;; ++x) {
                    unit.load(p, x);
                    const int64_t n = p.Hkv * unit.head_weight(p);
                    if (rem < n) break;
                    rem -= n;
                }
            u = __shfl_sync(0xffffffffu, x, owner);
            rem = __shfl_sync(0xffffffffu, rem, owner);
            unit.from_lane(owner);
        }
        const int64_t per_head = unit.head_weight(p);
        h = static_cast<int>(divide(rem, per_head));
        rem -= h * per_head;
        // the last pair with weight_before <= rem, 32 candidates at a time
        int lo = 0, hi = unit.pairs;
        while (hi - lo > 1) {
            const int stride = (hi - lo + 31) / 32, mid = lo + lane * stride;
            const unsigned ok = __ballot_sync(0xffffffffu, mid < hi && unit.weight_before(p, mid) <= rem);
            lo += (31 - __clz(ok)) * stride;
            hi = lo + stride < hi ? lo + stride : hi;
        }
        i = lo;
        at = rem - unit.weight_before(p, i);
        steps = unit.pair_steps(p, i);
        weight = unit.step_weight(p, i);
    }
    // The first step of the list that begins at `pos` or behind it.
    __device__ __forceinline__ int step_from(int64_t pos) const {
        const int64_t x = pos - kListCost;
        return x <= 0 ? 0 : static_cast<int>((x + weight - 1) >> (weight - 1));
    }
    __device__ __forceinline__ int64_t list_weight() const { return kListCost + static_cast<int64_t>(weight) * steps; }
    // The next list (not called behind the last one).
    __device__ __forceinline__ void next(const Params& p) {
        at = 0;
        if (++i == unit.pairs) {
            i = 0;
            if (++h == p.Hkv) {
                h = 0;
                do unit.load(p, ++u);
                while (unit.pairs == 0 && u + 1 < p.units);
            }
        }
        steps = unit.pair_steps(p, i);
        weight = unit.step_weight(p, i);
    }
};

// What every CTA of a prefix call works out from the lengths, by all of its threads (by one warp, as in a prefill, 1024 sequences in as many
// groups take 38 us more).  sums, zero before: [0, 32): the weights of the units of each lane of Walk; [32]: the cost of all lists; [33], [34]:
// the keys that remain for the other kernel, and the sequences that have any.
__device__ __forceinline__ void plan_sums(const Params& p, int tid, int threads, unsigned long long* sums) {
    const int per = (p.units + 31) / 32;
    int64_t cost = 0, own = 0, seqs = 0;
    for (int u = tid; u < p.units; u += threads) {
        Unit<true> unit;
        unit.load(p, u);
        if (unit.n > 0) {
            atomicAdd(sums + u / per, static_cast<unsigned long long>(p.Hkv * unit.head_weight(p)));
            cost += p.Hkv * attn_paged::list_cost(unit.n, unit.len, p.sharing, p.sharing.tile_ns, attn_paged::kListNs);
        }
    }
    for (int b = tid; b < p.tokens; b += threads) {
        int len = __ldg(p.seq_lens + b);
        len = len < 0 ? 0 : (len > p.max_len ? p.max_len : len);
        const int prefix = attn_paged::prefix_of(p.starts, p.prefix_lens, p.seq_lens, p.units, p.tokens, p.max_len, p.sharing, b);
        own += len > prefix ? len - prefix : 0;
        seqs += len > prefix ? 1 : 0;
    }
    cost = attn_paged::warp_sum(cost);
    own = attn_paged::warp_sum(own);
    seqs = attn_paged::warp_sum(seqs);
    if ((tid & 31) == 0) {
        if (cost > 0) atomicAdd(sums + 32, static_cast<unsigned long long>(cost));
        if (own > 0) atomicAdd(sums + 33, static_cast<unsigned long long>(own));
        if (seqs > 0) atomicAdd(sums + 34, static_cast<unsigned long long>(seqs));
    }
}

// A CTA's share of one list, as the roles of the CTA get it.
struct Item {
    int kvh, tok, n_tok;       // K/V head; first token and the tokens from there to the end of the unit
    int n0, n1, n_max;         // steps of each tile in this share, and of the share
    bool twin;                 // one tile of queries, in both places: tile 0 takes the even steps, tile 1 the odd ones
    int tile0;                 // first key tile
    int base, len;             // last key that the first token sees (prefill); keys
    int slot;                  // partial result (-1: the whole list)
    int first_row;             // row of the block table
    __device__ __forceinline__ int n(int t) const { return t ? n1 : n0; }
};

__device__ __forceinline__ void reg_inc_softmax() { asm volatile("setmaxnreg.inc.sync.aligned.u32 216;"); }
__device__ __forceinline__ void reg_dec_service() { asm volatile("setmaxnreg.dec.sync.aligned.u32 64;"); }

// 16-bit parts of a pair of probabilities, as split2 of attn_paged.cuh makes them, but with the first parts cut off instead of rounded (an
// instruction less): the second part is then off by 2^-16 of the whole (bf16; fp16: 2^-22).
template <int DTYPE>
__device__ __forceinline__ void split_p(float p0, float p1, uint32_t& hi, uint32_t& lo) {
    constexpr uint32_t CUT = DTYPE == 0 ? 0xffffe000u : 0xffff0000u;
    const float h0 = __uint_as_float(__float_as_uint(p0) & CUT), h1 = __uint_as_float(__float_as_uint(p1) & CUT);
    hi = DTYPE == 0 ? pack2<DTYPE>(h0, h1) : __byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x7632);
    float d0, d1;
    unpack_f32x2(fma_f32x2(pack_f32x2(h0, h1), pack_f32x2(-1.f, -1.f), pack_f32x2(p0, p1)), d0, d1);
    lo = pack2<DTYPE>(d0, d1);
}

template <int D, int DTYPE, bool PREFIX>
__global__ void __launch_bounds__(Cfg<D>::THREADS, 1)
attn_paged_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                     const __grid_constant__ Params p) {
    using C = Cfg<D>;
    constexpr int NBOX = C::NBOX, NGRP = C::NGRP;
    constexpr float LAG = 8.f;                     // the reference maximum may lag by 2^LAG
    constexpr float P_OFF = attn_paged::ExpRange<DTYPE>::P_OFF;      // what the partial results of attn_paged.cuh carry
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
    auto sQ = [&](int t) { return smem_base + t * C::Q_BYTES; };
    auto sKV = [&](int slot) { return smem_base + 2 * C::Q_BYTES + slot * C::KV_BYTES; };
    auto sOst = [&](int t) { return smem_base + 2 * C::Q_BYTES + C::NSLOT * C::KV_BYTES + t * C::OST_BYTES; };
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem_gen + C::TILE_BYTES);
    enum {
        B_QFULL = 0,       // [2] Q tile t loaded
        B_QEMPTY = 2,      // [2] every S product of tile t of the item has finished
        B_SFULL = 4,       // [2] S_t ready
        B_PFULL = 6,       // [2] first three quarters of P_t written (128 threads)
        B_PFULL2 = 8,      // [2] the rest
        B_OFINAL = 10,     // [2] the item's last O_t += P_t V has finished
        B_OFREE = 12,      // [2] O_t is in registers (128 threads)
        B_SCHEDFULL = 14,  // [4] slot holds an item
        B_SCHEDEMPTY = 18, // [4] slot read by warps 8, 10 and the eight softmax warps
        B_MERGE = 22,      // tile 1's sums are in shared memory (128 threads)
        B_KVFULL = 23,     // [NGRP] V_{j-1} and K_j loaded (two warps' copies)
        B_KVEMPTY = 23 + NGRP,
        B_COUNT = 23 + 2 * NGRP
    };
    auto bar = [&](int i) { return smem_base + C::TILE_BYTES + i * 8; };
    constexpr int SCHED = PREFIX ? 12 : 16;
    volatile int* sched = reinterpret_cast<volatile int*>(bars + B_COUNT);             // [4][SCHED]
    // [8][8]: of the key tile in ring group g % 8: whether any of its keys' pages is out of range, and which keys as bits.  (The
    // producer is at most NGRP groups ahead of the tile that the softmax groups are working on.)
    volatile uint32_t* bad_ring = reinterpret_cast<volatile uint32_t*>(sched + 4 * SCHED);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(const_cast<uint32_t*>(bad_ring) + 64);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    float2* merge = reinterpret_cast<float2*>(smem_gen + C::TILE_BYTES + C::MISC_BYTES - 1024);     // [128]: reference and sum of tile 1's rows
    constexpr int SUMS_AT = 8 * B_COUNT + 4 * (4 * SCHED + 64 + 2);
    unsigned long long* sums = reinterpret_cast<unsigned long long*>(reinterpret_cast<uint8_t*>(bars) + SUMS_AT);       // prefix: [35], see plan_sums
    static_assert(SUMS_AT + (PREFIX ? 8 * 35 : 0) <= C::MISC_BYTES - 1024 && SUMS_AT % 8 == 0, "barriers and slots");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int tile_rows = p.tile_tokens * p.group;

    if (PREFIX) {
        if (tid < 35) sums[tid] = 0;
        __syncthreads();
    }
    if (tid == 0) {
        *abort_flag = 0;
        for (int t = 0; t < 2; ++t) {
            mbar_init(bar(B_QFULL + t), 1);
            mbar_init(bar(B_QEMPTY + t), 1);
            mbar_init(bar(B_SFULL + t), 1);
            mbar_init(bar(B_PFULL + t), 128);
            mbar_init(bar(B_PFULL2 + t), 128);
            mbar_init(bar(B_OFINAL + t), 1);
            mbar_init(bar(B_OFREE + t), 128);
        }
        for (int s = 0; s < 4; ++s) {
            mbar_init(bar(B_SCHEDFULL + s), 1);
            mbar_init(bar(B_SCHEDEMPTY + s), 10);
        }
        mbar_init(bar(B_MERGE), 128);
        for (int s = 0; s < NGRP; ++s) {
            mbar_init(bar(B_KVFULL + s), 2);
            mbar_init(bar(B_KVEMPTY + s), 1);
        }
        fence_barrier_init();
        fence_proxy_async_smem();
    }
    // rows that no box writes (128 is not a multiple of the group) must be numbers
    for (int e = tid; tile_rows < 128 && e < 2 * NBOX * (128 - tile_rows) * 8; e += C::THREADS) {
        const int plane = e / ((128 - tile_rows) * 8);
        *reinterpret_cast<uint4*>(smem_gen + (plane * 128 + tile_rows) * 128 + (e - plane * (128 - tile_rows) * 8) * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    if (tile_rows < 128) fence_proxy_async_smem();
    if (warp == 8) {
        tmem_alloc(smem_u32(tmem_slot), C::TMEM_COLS);
        tmem_relinquish();
    }
    if (warp == 9 && lane == 0) {
        prefetch_tensormap(&tmQ);
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
    }
    if constexpr (PREFIX) plan_sums(p, tid, C::THREADS, sums);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = *tmem_slot;

    // every wait of a warp ends for all of its lanes alike
    auto wait = [&](int b, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar(b), parity, abort_flag)) != 0; };
    // The k-th item of this CTA; false: there is none.
    auto next_item = [&](int k, bool hand_back, Item& it) -> bool {
        const int slot = k & 3;
        if (!wait(B_SCHEDFULL + slot, (k >> 2) & 1)) return false;
        volatile int* e = sched + slot * SCHED;
        const bool valid = e[0] != 0;
        it.kvh = e[1];
        it.tok = e[2];
        it.n_tok = e[3];
        it.n0 = e[4];
        it.n1 = e[5];
        it.tile0 = e[6];
        it.base = e[7];
        it.len = e[8];
        it.slot = e[9];
        it.first_row = e[10];
        it.n_max = e[11] >> 1;
        it.twin = e[11] & 1;
        __syncwarp();
        if (hand_back) mbar_arrive(bar(B_SCHEDEMPTY + slot));
        return valid;
    };

    // ---- what the two warps that load tiles share: page numbers of a tile's boxes, box 32 r + lane: -1: no key there, -2: not a page ----
    const int boxes = 128 >> p.box_shift, slot_mask = (1 << p.page_shift) - 1;
    auto fetch = [&](const Item& it, int tile, int* pg) {
        const int* table = p.block_table + static_cast<int64_t>(it.first_row) * p.table_stride;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int box = 32 * r + lane, key = tile * 128 + (box << p.box_shift);
            pg[r] = -1;
            if (box < boxes && key < it.len) {
                pg[r] = __ldg(table + (key >> p.page_shift));
                if (static_cast<unsigned>(pg[r]) >= static_cast<unsigned>(p.num_pages)) pg[r] = -2;
            }
        }
    };
    auto load_tile = [&](const Item& it, uint32_t dst, const CUtensorMap* map, int axes, uint32_t full, int tile, const int* pg) {
        int n = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) n += __popc(__ballot_sync(0xffffffffu, pg[r] >= 0));
        if (lane == 0) mbar_arrive_expect_tx(full, (n * NBOX << p.box_shift) * 128);
        __syncwarp();        // armed before the first copy
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (32 * r >= boxes) break;
            const int row = (32 * r + lane) << p.box_shift;
            if (pg[r] >= 0) {
#pragma unroll
                for (int pl = 0; pl < NBOX; ++pl)
                    attn_paged::load_box(dst + pl * 16384 + row * 128, map, full, axes, pl, (tile * 128 + row) & slot_mask, it.kvh, pg[r]);
            }
        }
    };

    const volatile int64_t* plan = reinterpret_cast<const volatile int64_t*>(sums);
    if (warp >= 8) {
        reg_dec_service();
        if (warp == 9) {
            // =========================== lists, TMA ===========================
            const bool leader = elect_one();
            Walk<PREFIX> walk;
            int64_t left = 0;
            const int64_t total = walk.total(p, lane, plan);
            const int ctas = walk.ctas(p, total, plan);
            if (static_cast<int>(blockIdx.x) < ctas) {
                const int64_t first = cta_begin(total, blockIdx.x, ctas);
                left = cta_begin(total, blockIdx.x + 1, ctas) - first;
                walk.find(p, lane, first);
            }
            // prefill: the list of this CTA that goes on in the next one: none as yet (also where a wait runs out later)
            if (!PREFIX && leader) p.cuts[blockIdx.x] = Cut{{0, 0}, 0, 0, 0};
            int kv_base = 0, q_uses[2] = {0, 0};
            for (int k = 0;; ++k) {
                const int slot = k & 3;
                if (!wait(B_SCHEDEMPTY + slot, ((k >> 2) & 1) ^ 1)) break;
                Item it;
                // this CTA's steps of the next list that it has any of
                int s0 = 0, s1 = 0;
                int64_t origin = 0;      // where the list begins, counted back from the end of this CTA's part
                while (left > 0) {
                    const int64_t end = walk.list_weight() < walk.at + left ? walk.list_weight() : walk.at + left;
                    s0 = walk.step_from(walk.at);
                    s1 = walk.step_from(end);
                    origin = left + walk.at;
                    left -= end - walk.at;
                    if (s1 > s0) break;
                    if (left > 0) walk.next(p);
                }
                if (s1 > s0) {
                    const int pair_tok = walk.i * 2 * p.tile_tokens;
                    it.kvh = walk.h;
                    it.tok = walk.unit.tok0 + pair_tok;
                    it.n_tok = walk.unit.n - pair_tok;
                    it.tile0 = s0;
                    it.base = walk.unit.base + pair_tok;
                    it.len = walk.unit.len;
                    it.first_row = PREFIX ? walk.unit.tok0 : walk.u;
                    it.twin = it.n_tok <= p.tile_tokens;
                    it.n_max = s1 - s0;
                    if (it.twin) {
                        it.n0 = (it.n_max + 1) >> 1;
                        it.n1 = it.n_max >> 1;
                    } else {
                        const int all0 = walk.unit.steps_of(pair_tok + p.tile_tokens);
                        it.n0 = (all0 < s1 ? all0 : s1) - s0;
                        it.n0 = it.n0 < 0 ? 0 : it.n0;
                        it.n1 = it.n_max;
                    }
                    it.slot = s0 == 0 && s1 == walk.steps ? -1 : 2 * static_cast<int>(blockIdx.x) + (s0 == 0 ? 1 : 0);
                    if (!PREFIX && s0 == 0 && s1 < walk.steps) {
                        if (leader) {
                            const int64_t start = cta_begin(total, blockIdx.x + 1, ctas) - origin + kListCost;        // where step 0 lies
                            const int me = static_cast<int>(blockIdx.x), last0 = walk.unit.steps_of(pair_tok + p.tile_tokens) - 1;
                            Cut c;
                            c.parts[0] = cta_of_tile(total, start + static_cast<int64_t>(walk.weight) * last0, ctas) - me + 1;
                            c.parts[1] = it.twin ? 0 : cta_of_tile(total, start + static_cast<int64_t>(walk.weight) * (walk.steps - 1), ctas) - me + 1;
                            c.tok = it.tok;
                            c.n_tok = it.n_tok;
                            c.kvh = it.kvh;
                            p.cuts[me] = c;
                        }
                    }
                    if (left > 0) walk.next(p);
                    if (leader) {
                        volatile int* e = sched + slot * SCHED;
                        e[1] = it.kvh;
                        e[2] = it.tok;
                        e[3] = it.n_tok;
                        e[4] = it.n0;
                        e[5] = it.n1;
                        e[6] = it.tile0;
                        e[7] = it.base;
                        e[8] = it.len;
                        e[9] = it.slot;
                        e[10] = it.first_row;
                        e[11] = 2 * it.n_max + (it.twin ? 1 : 0);
                        e[0] = 1;
                        mbar_arrive(bar(B_SCHEDFULL + slot));
                    }
                } else {
                    if (leader) {
                        sched[slot * SCHED] = 0;
                        mbar_arrive(bar(B_SCHEDFULL + slot));
                    }
                    break;
                }
                auto load_q = [&](int t) -> bool {
                    if (!wait(B_QEMPTY + t, (q_uses[t] & 1) ^ 1)) return false;
                    if (leader) {
                        mbar_arrive_expect_tx(bar(B_QFULL + t), NBOX * tile_rows * 128);
#pragma unroll
                        for (int bx = 0; bx < NBOX; ++bx)
                            asm volatile(
                                "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                                ::"r"(sQ(t) + bx * 16384), "l"(reinterpret_cast<uint64_t>(&tmQ)), "r"(bar(B_QFULL + t)), "r"(64 * bx), "r"(it.kvh * p.group),
                                "r"(it.tok + (it.twin ? 0 : t * p.tile_tokens)), "r"(0)
                                : "memory");
                    }
                    ++q_uses[t];
                    return true;
                };
                // Ring group i of an item: {V_{i-1}, K_i}, what the MMA warp needs together (see attn_tc_pipe.cuh).  K here, V by
                // warp 10.
                int pg[4], pg_next[4];
                fetch(it, it.tile0, pg_next);
                bool ok = it.n0 > 0 ? load_q(0) : true;
                for (int i = 0; i <= it.n_max && ok; ++i) {
                    const int group = kv_base + i, g = group % NGRP;
#pragma unroll
                    for (int r = 0; r < 4; ++r) pg[r] = pg_next[r];
                    if (i + 1 < it.n_max) fetch(it, it.tile0 + i + 1, pg_next);
                    if (!(ok = wait(B_KVEMPTY + g, ((group / NGRP) & 1) ^ 1))) break;
#ifdef ATTN_TEST_HOOKS
                    if (group == p.test_skip_group) continue;      // this group's barrier never completes
#endif
                    if (i == it.n_max) {
                        if (lane == 0) mbar_arrive(bar(B_KVFULL + g));
                        continue;
                    }
                    volatile uint32_t* bad = bad_ring + (group & 7) * 8;
                    bool any = false;
#pragma unroll
                    for (int r = 0; r < 4; ++r) any = any || pg[r] == -2;
                    any = __any_sync(0xffffffffu, any);
                    if (any) {       // rare: the tile's bits are put together word by word
                        if (lane == 0) report_bad_index(p.status);
                        for (int w = 0; w < 4; ++w) {
                            // key 32 w + lane lies in box (32 w + lane) >> box_shift, whose page number lane box % 32 has
                            const int box = (32 * w + lane) >> p.box_shift;
                            int page = -1;
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int x = __shfl_sync(0xffffffffu, pg[r], box & 31);
                                if (box >> 5 == r) page = x;
                            }
                            const uint32_t word = __ballot_sync(0xffffffffu, page == -2);
                            if (lane == 0) bad[1 + w] = word;
                        }
                    }
                    if (lane == 0) bad[0] = any ? 1u : 0u;
                    load_tile(it, sKV(2 * g + 1), &tmK, p.k_axes, bar(B_KVFULL + g), it.tile0 + i, pg);
                    if (i == 0 && it.n1 > 0) ok = load_q(1);
                }
                if (!ok) break;
                kv_base += it.n_max + 1;
            }
        } else if (warp == 10) {
            // =========================== V tiles ===========================
            int kv_base = 0;
            bool ok = true;
            for (int k = 0; ok; ++k) {
                Item it;
                if (!next_item(k, lane == 0, it)) break;
                int pg[4], pg_next[4];
                fetch(it, it.tile0, pg_next);
                for (int i = 0; i <= it.n_max; ++i) {
                    const int group = kv_base + i, g = group % NGRP;
#pragma unroll
                    for (int r = 0; r < 4; ++r) pg[r] = pg_next[r];
                    if (i > 0 && i < it.n_max) fetch(it, it.tile0 + i, pg_next);
                    if (!(ok = wait(B_KVEMPTY + g, ((group / NGRP) & 1) ^ 1))) break;
                    if (i == 0) {
                        if (lane == 0) mbar_arrive(bar(B_KVFULL + g));
                        continue;
                    }
                    bool any = false;
#pragma unroll
                    for (int r = 0; r < 4; ++r) any = any || pg[r] == -2;
                    if (__any_sync(0xffffffffu, any)) {      // rare: V rows of pages that are out of range become zeros
                        uint8_t* v = smem_gen + 2 * C::Q_BYTES + 2 * g * C::KV_BYTES;
                        for (int row = 0; row < 128; ++row) {
                            const int box = row >> p.box_shift;
                            int page = -1;
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int x = __shfl_sync(0xffffffffu, pg[r], box & 31);
                                if (box >> 5 == r) page = x;
                            }
                            if (page == -2 && lane < 8 * NBOX) *reinterpret_cast<uint4*>(v + (lane >> 3) * 16384 + row * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                        }
                        fence_proxy_async_smem();
                        __syncwarp();
                    }
                    load_tile(it, sKV(2 * g), &tmV, p.v_axes, bar(B_KVFULL + g), it.tile0 + i - 1, pg);
                }
                kv_base += it.n_max + 1;
            }
        } else if (warp == 8) {
            // =========================== MMA issuer ===========================
            const bool leader = elect_one();
            constexpr uint32_t IDESC_S = make_idesc_f16(128, 128, DTYPE, 0, 0);
            constexpr uint32_t IDESC_O = make_idesc_f16(128, D, DTYPE, 0, 1);
            constexpr uint32_t DESC_HI = smem_desc_hi_sw128(1024);
            const uint32_t q_lo[2] = {smem_desc_lo(sQ(0), 16), smem_desc_lo(sQ(1), 16)};
            const uint32_t k_lo0 = smem_desc_lo(sKV(0), 16);          // K-major
            const uint32_t v_lo0 = smem_desc_lo(sKV(0), 16384);       // MN-major
            auto issue_s = [&](int t, int s) {
                if (leader) {
                    const uint32_t a0 = q_lo[t], b0 = k_lo0 + s * (C::KV_BYTES >> 4);
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint32_t off = ((kk >> 2) * 16384 + (kk & 3) * 32) >> 4;
                        mma_f16_ss_lohi(tmem + C::s_col(t), a0 + off, b0 + off, DESC_HI, IDESC_S, kk > 0);
                    }
                }
            };
            // 16 keys at a time; from 8 on (prefix) with the second parts of P
            auto issue_pv = [&](int t, int s, bool accumulate, int kk_begin, int kk_end) {
                if (leader) {
                    const uint32_t b0 = v_lo0 + s * (C::KV_BYTES >> 4);
#pragma unroll
                    for (int kk = kk_begin; kk < kk_end; ++kk)
                        mma_f16_ts_lohi(tmem + C::o_col(t), tmem + C::s_col(t) + kk * 8, b0 + ((kk & 7) * 16 * 128 >> 4), DESC_HI, IDESC_O,
                                        (accumulate || kk > 0) ? 1u : 0u);
                }
            };
            auto commit = [&](int b) {
                if (leader) mma_commit(bar(b));
            };
            int kv_base = 0, it_base[2] = {0, 0}, uses[2] = {0, 0};
            bool ok = true;
            for (int k = 0; ok; ++k) {
                Item it;
                if (!next_item(k, leader, it)) break;
                // V rows behind the sequence's end, in the last tile, become zeros (the ring's slot is this warp's until it commits the
                // products that read it).  That is all this warp looks at: reading the tile's flag, too, costs 4 % of 120 steps.
                auto clear_v = [&](int j, int slot) {
                    const int valid = it.len - (it.tile0 + j) * 128;
                    if (valid >= 128) return;
                    uint8_t* v = smem_gen + 2 * C::Q_BYTES + slot * C::KV_BYTES;
                    const int from = valid < 0 ? 0 : valid;
#pragma unroll 1
                    for (int e = from * 8 + lane; e < 128 * 8; e += 32)
#pragma unroll
                        for (int pl = 0; pl < NBOX; ++pl) *reinterpret_cast<uint4*>(v + pl * 16384 + e * 16) = make_uint4(0u, 0u, 0u, 0u);
                    fence_proxy_async_smem();
                    __syncwarp();
                };
                // O_t += P_t V, the i-th step of the tile; false: a wait ran out
                auto do_pv = [&](int t, int i, int gslot) {
                    const uint32_t par = (it_base[t] + i) & 1;
                    if (!wait(B_PFULL + t, par)) return false;
                    // the previous item's O_t must be in registers before it is overwritten
                    if (i == 0 && uses[t] > 0 && !wait(B_OFREE + t, (uses[t] - 1) & 1)) return false;
                    tc_fence_after_sync();
                    issue_pv(t, 2 * gslot, i > 0, 0, PREFIX ? 4 : 6);
                    if constexpr (PREFIX) issue_pv(t, 2 * gslot, true, 8, 12);
                    if (!wait(B_PFULL2 + t, par)) return false;
                    tc_fence_after_sync();
                    issue_pv(t, 2 * gslot, true, PREFIX ? 4 : 6, 8);
                    if constexpr (PREFIX) issue_pv(t, 2 * gslot, true, 12, 16);
                    if (i + 1 == it.n(t)) commit(B_OFINAL + t);
                    return true;
                };
                auto do_s = [&](int t, int i, int gslot) {
                    issue_s(t, 2 * gslot + 1);
                    commit(B_SFULL + t);
                    if (i + 1 == it.n(t)) commit(B_QEMPTY + t);      // the last S of the item
                };
                ok = wait(B_KVFULL + kv_base % NGRP, (kv_base / NGRP) & 1);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (ok && it.n(t) > 0 && !(t == 1 && it.twin)) {
                        ok = wait(B_QFULL + t, uses[t] & 1);
                        tc_fence_after_sync();
                        if (ok) do_s(t, 0, kv_base % NGRP);
                    }
                }
                if (ok) commit(B_KVEMPTY + kv_base % NGRP);
                if (!it.twin) {
#pragma unroll 1
                    for (int j = 0; j < it.n_max && ok; ++j) {
                        const int grp = kv_base + j + 1, gslot = grp % NGRP;
                        if (!(ok = wait(B_KVFULL + gslot, (grp / NGRP) & 1))) break;
                        clear_v(j, 2 * gslot);
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            if (j < it.n(t) && !(ok = do_pv(t, j, gslot))) break;
                            if (j + 1 < it.n(t)) do_s(t, j + 1, gslot);
                        }
                        if (ok) commit(B_KVEMPTY + gslot);
                    }
                } else {
                    // tile 0 takes the even steps, tile 1 the odd ones; the next step's S first: it waits for no softmax
#pragma unroll 1
                    for (int j2 = 0; j2 < it.n0 && ok; ++j2) {
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            const int j = 2 * j2 + t;
                            if (j >= it.n_max) break;
                            const int grp = kv_base + j + 1, gslot = grp % NGRP;
                            if (!(ok = wait(B_KVFULL + gslot, (grp / NGRP) & 1))) break;
                            clear_v(j, 2 * gslot);
                            if (j + 1 < it.n_max) {
                                if (j == 0 && !(ok = wait(B_QFULL + 1, uses[1] & 1))) break;
                                tc_fence_after_sync();
                                do_s(t ^ 1, j2 + t, gslot);
                            }
                            if (!(ok = do_pv(t, j2, gslot))) break;
                            commit(B_KVEMPTY + gslot);
                        }
                    }
                }
                kv_base += it.n_max + 1;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    it_base[t] += it.n(t);
                    uses[t] += it.n(t) > 0 ? 1 : 0;
                }
            }
        } else {
            // =========================== checks, plans ===========================
            if constexpr (PREFIX) {
                // where the partial results of each sequence's rows will lie, a lane per sequence: by the CTAs that have no lists
                Walk<true> walk;
                const int64_t total = walk.total(p, lane, plan);
                const int ctas = walk.ctas(p, total, plan), free = ctas < p.grid ? ctas : 0, stride = p.grid - free;
                const int first = static_cast<int>(blockIdx.x) - free;
                if (first == 0 && lane == 0) p.plan[p.tokens] = PrefixPlan{total, ctas, 0, 0};
                for (int b0 = first; first >= 0 && b0 < p.tokens; b0 += 32 * stride) {
                    const int b = b0 + lane * stride, g = b < p.tokens ? attn_paged::group_of(p.starts, p.units, b) : -1;
                    int64_t start = __shfl_sync(0xffffffffu, walk.before, g < 0 ? 0 : g / walk.per);
                    PrefixPlan at = {0, 0, -1, 0};
                    if (g >= 0) {
                        Unit<true> unit;
                        for (int x = g / walk.per * walk.per; x < g; ++x) {
                            unit.load(p, x);
                            start += p.Hkv * unit.head_weight(p);
                        }
                        unit.load(p, g);
                        const int token = b - unit.tok0, pair = token / (2 * p.tile_tokens), in_pair = token - pair * 2 * p.tile_tokens;
                        if (token >= 0 && token < unit.n) {
                            const int t = in_pair >= p.tile_tokens ? 1 : 0;
                            at.start = start + unit.weight_before(p, pair) + kListCost;
                            at.stride = unit.head_weight(p);
                            at.span = static_cast<int64_t>(unit.step_weight(p, pair)) * (unit.pair_steps(p, pair) - 1);
                            at.row = t * 128 + (in_pair - t * p.tile_tokens) * p.group;
                        }
                    }
                    if (b < p.tokens) p.plan[b] = at;
                }
            } else {
                // lengths that are out of range (of a prefix call the second kernel reports them)
                for (int u = static_cast<int>(blockIdx.x) * 32 + lane; u < p.units; u += 32 * gridDim.x) {
                    const int len = __ldg(p.seq_lens + u), begin = __ldg(p.starts + u), end = __ldg(p.starts + u + 1);
                    if (len > p.max_len || (len > 0 && (begin < 0 || end > p.tokens || end - begin > len))) report_bad_index(p.status);
                }
            }
        }
    } else {
        // =========================== softmax groups ===========================
        reg_inc_softmax();
        const int t = warp >> 2, r = tid & 127, w4 = warp & 3;
        const uint32_t lane_off = static_cast<uint32_t>(w4 * 32) << 16;
        const uint32_t tS = tmem + C::s_col(t) + lane_off, tO = tmem + C::o_col(t) + lane_off;
        const float c = p.scale_log2;
        const int row_token = r / p.group, my_head = r % p.group;                        // of the tile; of the K/V head
        const uint32_t ost = sOst(t) + w4 * 4096;                                        // this warp's staging: 32 rows x 128 bytes
        int it_base = 0, uses = 0, kv_base = 0, merges = 0;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            Item it;
            if (!next_item(k, lane == 0, it)) break;
            const int n = it.n(t), group0 = kv_base;
            kv_base += it.n_max + 1;
            if (n <= 0) continue;
            const int my_token = it.twin ? row_token : t * p.tile_tokens + row_token;
            const bool live = r < tile_rows && my_token < it.n_tok;
            // last key that this row sees; rows without a token ask for no mask
            int lim = 0;
            if (live) {
                if constexpr (PREFIX) {
                    const int len = __ldg(p.seq_lens + it.tok + my_token);
                    lim = (len < it.len ? len : it.len) - 1;
                } else {
                    lim = it.base + my_token;
                }
            }
            const int lim_lo = __reduce_min_sync(0xffffffffu, live ? lim : 2147483647);
            const int lim_hi = __reduce_max_sync(0xffffffffu, live ? lim : -2147483647);
            if (!live) lim = 2147483647;
            const bool any_live = lim_hi > -2147483647;
            float m = 0.f, l = 0.f;
            bool unset = live, any_unset = any_live;       // the reference maximum is taken from the first tile that shows the row a key

            // O_t *= alpha, before step j (the last update of O finished before S was produced)
            auto rescale = [&](int j, float alpha) {
                if (j == 0) return;
#pragma unroll 1
                for (int ch = 0; ch < D / 32; ++ch) {
                    uint32_t orr[32];
                    tmem_ld_32x32b_x32(tO + ch * 32, orr);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; ++e) orr[e] = __float_as_uint(__uint_as_float(orr[e]) * alpha);
                    tmem_st_32x32b_x32(tO + ch * 32, orr);
                }
            };
            for (int j = 0; j < n; ++j) {
                if (!(ok = wait(B_SFULL + t, (it_base + j) & 1))) break;
                tc_fence_after_sync();
                if (!any_live) {                           // no row of this warp is a query's: whatever S holds may stand in as P
                    mbar_arrive(bar(B_PFULL + t));
                    mbar_arrive(bar(B_PFULL2 + t));
                    continue;
                }
                const int step = it.twin ? 2 * j + t : j, kv0 = (it.tile0 + step) * 128;
                const volatile uint32_t* bad = bad_ring + ((group0 + step) & 7) * 8;
                const bool some_bad = __any_sync(0xffffffffu, bad[0] != 0);
                if (__any_sync(0xffffffffu, kv0 + 127 > lim_lo || some_bad)) {
                    // hidden scores become -inf in tensor memory, so that masked tiles run the code of all others
#pragma unroll 1
                    for (int ch = 0; ch < 4; ++ch) {
                        const int a = kv0 + 32 * ch;
                        const uint32_t ok_keys = some_bad ? ~bad[1 + ch] : 0xffffffffu;
                        if (a + 31 <= lim_lo && ok_keys == 0xffffffffu) continue;
                        uint32_t tmp[32];
                        if (a > lim_hi || ok_keys == 0u) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) tmp[e] = 0xff800000u;
                        } else {
                            tmem_ld_32x32b_x32(tS + ch * 32, tmp);
                            tmem_ld_wait();
                            const uint32_t seen = low_bits(lim > a + 31 ? 32 : lim - a + 1) & ok_keys;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!(seen & (1u << e))) tmp[e] = 0xff800000u;
                        }
                        tmem_st_32x32b_x32(tS + ch * 32, tmp);
                    }
                    tmem_st_wait();
                }
                uint32_t sr[128];
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) tmem_ld_32x32b_x32(tS + ch * 32, sr + ch * 32);
                tmem_ld_wait();
                auto max_of = [&](float* mx, int e0, int e1) {
#pragma unroll
                    for (int e = e0; e < e1; e += 16)
#pragma unroll
                        for (int x = 0; x < 8; ++x) mx[x] = max3(mx[x], __uint_as_float(sr[e + 2 * x]), __uint_as_float(sr[e + 2 * x + 1]));
                };
                auto max8 = [&](const float* mx) {
                    return fmaxf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), fmaxf(fmaxf(mx[4], mx[5]), fmaxf(mx[6], mx[7])));
                };
                if constexpr (PREFIX) {
                    // The tile's maximum first, so that no exponential is taken twice and S leaves the registers as P's two parts come.  P
                    // carries 2^P_OFF, as in attn_paged.cuh: its small values keep their precision in fp16.
                    float mx[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) mx[x] = -INFINITY;
                    max_of(mx, 0, 128);
                    const float top = max8(mx);
                    const bool ahead = live && (unset ? top != -INFINITY : (top - m) * c > LAG);
                    float alpha = 1.f;
                    if (__any_sync(0xffffffffu, ahead)) {
                        if (ahead) {
                            if (!unset) alpha = ex2_approx((m - top) * c);
                            m = top;
                            unset = false;
                        }
                        rescale(j, alpha);
                    }
                    const float nmc = fmaf(-m, c, P_OFF);
                    const uint64_t c2 = pack_f32x2(c, c), nmc2 = pack_f32x2(nmc, nmc);
                    uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
                    for (int ch = 0; ch < 4; ++ch) {
                        uint32_t hi[16], lo[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float x0, x1;
                            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(sr[ch * 32 + e]), __uint_as_float(sr[ch * 32 + e + 1])), c2, nmc2), x0, x1);
                            const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
                            acc[(e / 2) & 3] = add_f32x2(acc[(e / 2) & 3], pack_f32x2(p0, p1));
                            split_p<DTYPE>(p0, p1, hi[e / 2], lo[e / 2]);
                        }
                        tmem_st_32x32b_x16(tS + ch * 16, hi);
                        tmem_st_32x32b_x16(tS + 64 + ch * 16, lo);
                        if (ch == 1) {
                            tmem_st_wait();
                            tc_fence_before_sync();
                            mbar_arrive(bar(B_PFULL + t));
                        }
                    }
                    float a0, a1, a2, a3;
                    unpack_f32x2(add_f32x2(acc[0], acc[1]), a0, a1);
                    unpack_f32x2(add_f32x2(acc[2], acc[3]), a2, a3);
                    l = l * alpha + ((a0 + a1) + (a2 + a3));
                    tmem_st_wait();
                    tc_fence_before_sync();
                    mbar_arrive(bar(B_PFULL2 + t));
                    continue;
                }
                if (any_unset) {
                    float mx[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) mx[x] = -INFINITY;
                    max_of(mx, 0, 128);
                    const float top = max8(mx);
                    if (unset && top != -INFINITY) {
                        m = top;
                        unset = false;
                    }
                    any_unset = __any_sync(0xffffffffu, unset);
                }
                // Exponentials against the reference maximum of the tiles before, this tile's maximum on the side; once more with a
                // new reference where a row has grown by more than 2^LAG.
                float alpha = 1.f;
#pragma unroll 1
                for (bool again = false;; again = true) {
                    const float nmc = -m * c;
                    const uint64_t c2 = pack_f32x2(c, c), nmc2 = pack_f32x2(nmc, nmc);
                    uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
                    float mx[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) mx[x] = -INFINITY;
                    auto exp_chunk = [&](int ch) {
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float x0, x1;
                            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(sr[ch * 32 + e]), __uint_as_float(sr[ch * 32 + e + 1])), c2, nmc2), x0, x1);
                            const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
                            acc[(e / 2) & 3] = add_f32x2(acc[(e / 2) & 3], pack_f32x2(p0, p1));
                            pk[e / 2] = pack2<DTYPE>(p0, p1);
                        }
                        tmem_st_32x32b_x16(tS + ch * 16, pk);
                    };
#pragma unroll
                    for (int ch = 0; ch < 3; ++ch) {
                        exp_chunk(ch);
                        max_of(mx, ch == 0 ? 0 : (ch == 1 ? 48 : 96), ch == 0 ? 48 : (ch == 1 ? 96 : 128));
                    }
                    if (!again) {
                        const float top = max8(mx);
                        const bool ahead = live && (top - m) * c > LAG;
                        if (__any_sync(0xffffffffu, ahead)) {
                            if (ahead) {
                                alpha = ex2_approx((m - top) * c);
                                m = top;
                            }
                            rescale(j, alpha);
                            continue;
                        }
                    }
                    tmem_st_wait();
                    tc_fence_before_sync();
                    mbar_arrive(bar(B_PFULL + t));         // first three quarters of P are in place
                    exp_chunk(3);
                    float a0, a1, a2, a3;
                    unpack_f32x2(add_f32x2(acc[0], acc[1]), a0, a1);
                    unpack_f32x2(add_f32x2(acc[2], acc[3]), a2, a3);
                    l = l * alpha + ((a0 + a1) + (a2 + a3));
                    break;
                }
                tmem_st_wait();
                tc_fence_before_sync();
                mbar_arrive(bar(B_PFULL2 + t));
            }
            if (!ok) break;
            it_base += n;

            // ---- epilogue: through this warp's part of the staging tile, so that rows leave in whole lines ----
            if (!(ok = wait(B_OFINAL + t, uses & 1))) break;
            ++uses;
            tc_fence_after_sync();
            // Twins: tile 1's group hands over its reference and sum, and tile 0's adds up both accumulators.
            const bool both = it.twin && it.n1 > 0;
            float f1 = 0.f, f0 = 1.f;
            if (both) {
                if (t == 1) {
                    merge[r] = make_float2(m, l);
                    tc_fence_before_sync();
                    mbar_arrive(bar(B_MERGE));
                    continue;
                }
                if (!(ok = wait(B_MERGE, merges & 1))) break;
                ++merges;
                tc_fence_after_sync();
                const float2 other = merge[r];
                const float top = l != 0.f ? (other.y != 0.f ? fmaxf(m, other.x) : m) : other.x;
                f0 = l != 0.f ? ex2_approx((m - top) * c) : 0.f;
                f1 = other.y != 0.f ? ex2_approx((other.x - top) * c) : 0.f;
                l = fmaf(f0, l, f1 * other.y);
                m = top;
            }
            const bool final_rows = !PREFIX && it.slot < 0;
            const bool seen = l != 0.f;                    // false: no visible key in this share (a sum that is no number stays one)
            // this row of [tokens][H]
            const int out_row = live ? (it.tok + my_token) * p.H + it.kvh * p.group + my_head : -1;
            float* part = p.parts + it.slot * part_floats(D);
            if (live) {
                if (final_rows) {
                    p.lse[out_row] = seen ? fmaf(m, p.scale, logf(l)) : -INFINITY;
                } else {
                    float2* ml = reinterpret_cast<float2*>(it.slot < 0 ? p.rows + static_cast<int64_t>(p.tokens) * p.H * D + 2 * static_cast<int64_t>(out_row)
                                                                       : part + kRows * D + 2 * (t * 128 + r));
                    *ml = make_float2(PREFIX ? m * c : fmaf(m, c, P_OFF), l);
                }
            }
            if (final_rows) {
                const float inv = seen ? 1.f / l : 0.f;
                f0 *= inv;
                f1 *= inv;
            }
            // Rows leave 128 bytes at a time, a quarter of a warp per row: row 4 x + lane / 8 goes to to + at[x] * row_bytes.
            uint8_t* to = (final_rows ? static_cast<uint8_t*>(p.o) : reinterpret_cast<uint8_t*>(it.slot < 0 ? p.rows : part)) + (lane & 7) * 16;
            const int row_bytes = final_rows ? 2 * D : 4 * D;
            int at[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const int row = 4 * x + (lane >> 3), other = __shfl_sync(0xffffffffu, out_row, row);
                at[x] = it.slot < 0 ? other : t * 128 + w4 * 32 + row;
            }
            auto stage = [&](int piece, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(ost + lane * 128 + ((piece ^ (lane & 7)) << 4)), "r"(a), "r"(b), "r"(c), "r"(d)
                             : "memory");
            };
#pragma unroll 1
            for (int col = 0; col < D; col += 32) {
                float o[32];
                {
                    uint32_t a[32];
                    tmem_ld_32x32b_x32(tO + col, a);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(a[e]) * f0;
                    if (both) {
                        tmem_ld_32x32b_x32(tO + D + col, a);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = fmaf(__uint_as_float(a[e]), f1, o[e]);
                    }
                }
                if (col + 32 == D) {                       // O is in registers
                    tc_fence_before_sync();
                    mbar_arrive(bar(B_OFREE + t));
                    if (both) mbar_arrive(bar(B_OFREE + 1));
                }
                if (final_rows) {
                    const int half = (col >> 3) & 4;
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        stage(half + g, pack2<DTYPE>(o[8 * g], o[8 * g + 1]), pack2<DTYPE>(o[8 * g + 2], o[8 * g + 3]), pack2<DTYPE>(o[8 * g + 4], o[8 * g + 5]),
                              pack2<DTYPE>(o[8 * g + 6], o[8 * g + 7]));
                    if (half == 0) continue;
                } else {
#pragma unroll
                    for (int g = 0; g < 8; ++g)
                        stage(g, __float_as_uint(o[4 * g]), __float_as_uint(o[4 * g + 1]), __float_as_uint(o[4 * g + 2]), __float_as_uint(o[4 * g + 3]));
                }
                __syncwarp();
                uint4 w[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int row = 4 * x + (lane >> 3);
                    w[x] = attn_paged::lds128(ost + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
                }
                __syncwarp();
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    if (at[x] >= 0) *reinterpret_cast<uint4*>(to + static_cast<int64_t>(at[x]) * row_bytes) = w[x];
                to += 128;
            }
        }
    }

    // ---- teardown (also reached after a timed-out wait) ----
    tc_fence_before_sync();
    __syncthreads();
    if (tid == 0 && *abort_flag != 0) attn_tc::report_timeout(p.status);
    __syncthreads();
    if (warp == 8) tmem_dealloc(tmem, C::TMEM_COLS);
}

// Joins the partial results of prefill lists that were cut: block (c, y) takes rows of the list whose first border is the one
// between CTAs c and c + 1 (its last list, and the first of the others).  A warp per row.
template <int D, int DTYPE>
__global__ void __launch_bounds__(attn_paged::kJoinWarps * 32)
attn_paged_prefill_join_kernel(const __grid_constant__ Params p) {
    constexpr float P_OFF = attn_paged::ExpRange<DTYPE>::P_OFF;
    const int lane = threadIdx.x & 31, c0 = blockIdx.x;
    const int row = blockIdx.y * attn_paged::kJoinWarps + (threadIdx.x >> 5), t = row >> 7, r = row & 127;
    const int in_tile = r / p.group, token = t * p.tile_tokens + in_tile;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Cut* cut = p.cuts + c0;
    const int n = __ldcg(cut->parts + t), tok = __ldcg(&cut->tok), n_tok = __ldcg(&cut->n_tok), kvh = __ldcg(&cut->kvh);
    if (n == 0 || in_tile >= p.tile_tokens || token >= n_tok) return;
    const int64_t out_row = static_cast<int64_t>(tok + token) * p.H + kvh * p.group + r - in_tile * p.group;
    auto part = [&](int i) { return p.parts + (2 * (c0 + i) + (i == 0 ? 1 : 0)) * part_floats(D); };
    attn_paged::join_row<D, DTYPE>(n, lane, P_OFF, [&](int i) { return reinterpret_cast<const float2*>(part(i) + kRows * D) + row; },
                                   [&](int i) { return part(i) + row * D; }, static_cast<uint8_t*>(p.o) + out_row * (2 * D), p.lse + out_row);
}

// Joins what the two kernels of a call with shared prefixes have left for each row: the parts of its sequence's own keys
// (attn_paged.cuh) and those of the prefix.  A warp per row, eight rows of one sequence to a block, as in attn_paged_join_kernel.
template <int D, int DTYPE, int GH>
__global__ void __launch_bounds__(attn_paged::kJoinWarps * 32)
attn_paged_prefix_join_kernel(const __grid_constant__ attn_paged::DecodeParams p, const __grid_constant__ Params pre, int blocks_per_seq) {
    using C = attn_paged::DecodeCfg<D, GH>;
    constexpr float P_OFF = attn_paged::ExpRange<DTYPE>::P_OFF;
    const int b = blockIdx.x / blocks_per_seq, lane = threadIdx.x & 31;
    const int q_head = (blockIdx.x - b * blocks_per_seq) * attn_paged::kJoinWarps + (threadIdx.x >> 5);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (q_head >= p.H) return;
    const int64_t out_row = static_cast<int64_t>(b) * p.H + q_head;
    uint8_t* out = static_cast<uint8_t*>(p.o) + out_row * D * 2;
    const int64_t n_rows = static_cast<int64_t>(p.B) * p.H;
    const PrefixPlan* plan = pre.plan + b;
    const int64_t total = __ldcg(&pre.plan[p.B].start), ctas = __ldcg(&pre.plan[p.B].stride);
    const int64_t first = __ldcg(&plan->start), stride = __ldcg(&plan->stride);
    const int64_t span = __ldcg(&plan->span);
    const int kvh = q_head / pre.group, row = __ldcg(&plan->row) + q_head - kvh * pre.group;
    const attn_paged::SeqPlan list = attn_paged::SeqPlan::read(p, b);
    int n_pre = 0, c0 = 0;
    if (span >= 0) {
        const int64_t start = first + kvh * stride;
        c0 = cta_of_tile(total, start, static_cast<int>(ctas));
        n_pre = cta_of_tile(total, start + span, static_cast<int>(ctas)) - c0 + 1;
    }
    attn_paged::RowParts own;
    if (list.n > 0) own.find(p, list, q_head);
    const int n_own = own.count;
    if (n_own + n_pre == 0) {
        attn_paged::empty_row<D>(out, p.lse + out_row, lane);
        return;
    }
    // Part i of the sequence's own keys and part i of the prefix: the first one's O, and how far the others lie (see RowParts::at and
    // Item::slot); exponent and sum at a fixed distance.
    const float *own0 = p.rows + out_row * D, *pre0 = pre.rows + out_row * D;
    int64_t own_ml = (n_rows - out_row) * D + 2 * out_row, pre_ml = own_ml;
    const int64_t own_stride = static_cast<int64_t>(C::PART_FLOATS) << own.hs;
    if (n_own > 1) {
        own0 = own.at<C::PART_FLOATS>(p, 0) + own.row * D;
        own_ml = GH * D + 2 * own.row - own.row * D;
    }
    if (n_pre > 1) {
        pre0 = pre.parts + (2 * c0 + 1) * part_floats(D) + row * D;
        pre_ml = kRows * D + 2 * row - row * D;
    }
    auto part = [&](int i) {
        const int j = i < n_own ? i : i - n_own;
        const int64_t stride = i < n_own ? own_stride : part_floats(D);
        const int away = j == 0 ? 0 : 2 * j - (i < n_own ? (own.odd ? 1 : 0) : 1);
        return (i < n_own ? own0 : pre0) + away * stride;
    };
    attn_paged::join_row<D, DTYPE>(n_own + n_pre, lane, P_OFF,
                                   [&](int i) { return reinterpret_cast<const float2*>(part(i) + (i < n_own ? own_ml : pre_ml)); }, part, out,
                                   p.lse + out_row);
}

}  // namespace attn_paged_tc
