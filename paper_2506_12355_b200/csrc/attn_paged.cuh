// Attention of one new token per sequence over a paged key/value cache.
//
//     O[b,h] = sum_j p_j V[b,g,j] / sum_j p_j,   p_j = exp(scale <q[b,h], K[b,g,j]>),   g = h / (H / Hkv),
//     LSE[b,h] = ln sum_j p_j,   j over the visible keys of sequence b: j < len, and with a window of W keys and s first
//     tokens that stay visible only j >= len - W or j < s.
//
// Every visible key's K and V row is read once: 4 D bytes per key and K/V head, 2 multiply-adds per value and query head.
// That is HBM-bound for every group size up to 16 query heads per K/V head, so all of the design serves the loads:
//
//   * Key axis cut into tiles of 16 keys per warp; the tiles of all (sequence, K/V head) pairs form one list, of which
//     every CTA of a one-wave persistent grid takes an equal, contiguous part, whatever the lengths are.  The list is
//     laid out from the device-side lengths by each CTA for itself (no host copy of the lengths, no plan to keep).
//     A (sequence, head) pair inside one CTA's part is finished there; one that is cut by a border leaves one fp32
//     partial result per CTA (at most two per CTA), and a second small kernel joins those.
//   * A thread copies exactly the 16-byte pieces that it will feed to the tensor core itself (cp.async into its own slots of
//     a ring in shared memory), so there is no synchronisation between copy and use, pages of any power-of-two size and
//     any strides cost the same, and 128 KB and more per SM are in flight.
//   * The products run on mma.sync m16n8k16.  With 16 query rows they need a few percent of its rate; a tcgen05
//     instruction takes 128 rows, 112 of which would be padding, and K/V tiles staged for it by one thread.
//     First product: A = Q (rows: query heads), B = K (columns: keys).  The contraction order over D is free, so that a
//     thread's 16 contiguous bytes serve two instructions.  The accumulator layout of S is the A layout of the second
//     product (B = V, columns: value dims, again in the order in which 16-byte pieces deliver them).
//   * P is fed as two 16-bit parts (hi + lo), so its rounding does not show in O.  With up to 8 query heads per K/V head
//     the low parts take rows 8 .. 15 of the same instructions.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "sm100_ptx.cuh"

namespace attn_paged {

constexpr int kMaxCtas = 148;        // CTAs of the persistent grid (one per SM); sizes the workspace
constexpr int kStatusBadIndex = 13;  // ATTN_ERR_DEVICE_INDEX

// A page number, position or length that the device found out of range.  An earlier report of a timed-out wait stays.
__device__ __forceinline__ void report_bad_index(int* status) { atomicCAS(status, 0, kStatusBadIndex); }

template <int D, int GH>
struct DecodeCfg {
    static constexpr int NW = D == 256 ? 4 : 8;             // warps
    static constexpr int THREADS = NW * 32;
    static constexpr int NCH = D / 8;                       // 16-byte pieces of a thread's share of 16 keys (K and V)
    static constexpr int STAGE_BYTES = NW * NCH * 512;
    // ring stages: as many as fit beside the merge buffer
    static constexpr int NSTAGE = D == 64 ? (GH == 8 ? 6 : 5) : (D == 128 ? (GH == 8 ? 3 : 2) : 2);
    static constexpr int ROW = D + 4;                       // floats of a row in the merge buffer (16-byte rows, banks shifted)
    static constexpr int MERGE_BYTES = NW * GH * ROW * 4 + NW * GH * 8;
    static constexpr int SMEM_BYTES = NSTAGE * STAGE_BYTES + MERGE_BYTES + 64;
    static_assert(SMEM_BYTES <= 232448, "shared memory budget");
    // a partial result: O [GH][D] (not normalised), then reference exponent and sum [GH][2], fp32
    static constexpr int PART_FLOATS = GH * (D + 2);
};

struct DecodeParams {
    const void* q;              // [B, H, D]
    const uint8_t* k_cache;     // [pages, Hkv, slots, D] through byte strides
    const uint8_t* v_cache;
    void* o;
    float* lse;
    const int* block_table;
    const int* seq_lens;
    float* parts;
    int* status;
    int64_t k_page, k_head, k_slot, v_page, v_head, v_slot;   // byte strides
    int64_t table_stride;       // entries between the rows of block_table
    int B, H, Hkv, group, sub;  // query heads per K/V head; parts of at most 16 of them
    int max_len;                // slots that a row of block_table covers
    int num_pages, page_shift;
    int window, sinks;
    float scale_log2;
    int grid;                   // CTAs of the first kernel
};

// Visible chunks of 16 keys of one sequence: n_sink of them from key 0, then those from chunk `lo`.
struct SeqRange {
    int len, win_lo;   // keys >= win_lo are visible, and those < sinks
    int n_sink, lo, n_chunks;
};

__device__ __forceinline__ SeqRange seq_range(const DecodeParams& p, int b) {
    SeqRange r;
    int len = p.seq_lens[b];
    len = len < 0 ? 0 : (len > p.max_len ? p.max_len : len);
    r.len = len;
    r.win_lo = (p.window > 0 && p.window < len) ? len - p.window : 0;
    r.lo = r.win_lo >> 4;
    const int sink_chunks = (p.sinks >> 4) + ((p.sinks & 15) != 0);
    r.n_sink = sink_chunks < r.lo ? sink_chunks : r.lo;
    r.n_chunks = r.n_sink + ((len + 15) >> 4) - r.lo;
    return r;
}

template <int NW>
__device__ __forceinline__ int seq_tiles(const SeqRange& r) { return (r.n_chunks + NW - 1) / NW; }

// CTA c of `ctas` takes the tiles [total * c / ctas, total * (c + 1) / ctas).  No more CTAs than tiles: none is empty, so
// that a cut pair has a partial result from every CTA between its first and its last one.
__device__ __forceinline__ int cta_count(int64_t total, int grid) { return total < grid ? static_cast<int>(total) : grid; }
__device__ __forceinline__ int64_t cta_begin(int64_t total, int c, int ctas) { return total * c / ctas; }
__device__ __forceinline__ int cta_of_tile(int64_t total, int64_t t, int ctas) {
    return static_cast<int>(((t + 1) * ctas - 1) / total);
}

__device__ __forceinline__ int64_t warp_sum(int64_t x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool live) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

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

// Position in the tile list, advanced tile by tile.  Every warp of a CTA walks the same tiles.
template <int NW>
struct TileWalk {
    int b, h, t, t_end;   // sequence, K/V head (times head part), tile inside the pair, tiles of the pair
    SeqRange r;
    __device__ __forceinline__ void next(const DecodeParams& p, int heads) {
        if (++t < t_end) return;
        t = 0;
        if (++h < heads) return;
        h = 0;
        do {
            if (++b >= p.B) return;      // the end of the list: not used again
            r = seq_range(p, b);
            t_end = seq_tiles<NW>(r);
        } while (t_end == 0);
    }
};

// P carries a factor 2^P_OFF where 16-bit floats run out of small numbers (fp16); the reference maximum may lag by 2^LAG.
template <int DTYPE> struct ExpRange { static constexpr float P_OFF = DTYPE == 0 ? 6.f : 0.f, LAG = 8.f; };

// GH: query rows of an item, 8 (up to 8 query heads per K/V head) or 16.
template <int D, int DTYPE, int GH>
__global__ void __launch_bounds__(DecodeCfg<D, GH>::THREADS, 1)
attn_paged_decode_kernel(const DecodeParams p) {
    using C = DecodeCfg<D, GH>;
    constexpr int NW = C::NW, NSTAGE = C::NSTAGE, NCH = C::NCH;
    constexpr int KI = D / 32, VI = D / 64;         // 16-byte pieces of a thread: per key row of K, per key row of V
    constexpr float P_OFF = ExpRange<DTYPE>::P_OFF, LAG = ExpRange<DTYPE>::LAG;
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    float* merge = reinterpret_cast<float*>(smem + NSTAGE * C::STAGE_BYTES);
    float2* merge_ml = reinterpret_cast<float2*>(merge + NW * GH * C::ROW);
    int64_t* scan = reinterpret_cast<int64_t*>(smem);        // before the ring is used: [0..31] warp sums, then the start
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- lay out the tile list: total tiles, and the pair and tile at which this CTA's part begins ----
    const int heads = p.Hkv * p.sub;
    const int per = (p.B + C::THREADS - 1) / C::THREADS;     // consecutive sequences of a thread
    const int b0 = tid * per, b1 = b0 + per < p.B ? b0 + per : p.B;
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) {
        mine += seq_tiles<NW>(seq_range(p, b));
        if (p.seq_lens[b] > p.max_len && blockIdx.x == 0) report_bad_index(p.status);
    }
    int64_t incl = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int64_t up = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += up;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    int64_t before = incl - mine, total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < warp) before += scan[w];
        total += scan[w];
    }
    total *= heads;
    const int ctas = cta_count(total, p.grid);
    if (static_cast<int>(blockIdx.x) >= ctas) return;
    const int64_t first = cta_begin(total, blockIdx.x, ctas), steps = cta_begin(total, blockIdx.x + 1, ctas) - first;
    // the thread whose sequences hold tile `first` finds it
    if (first >= before * heads && first < (before + mine) * heads) {
        int64_t rem = first - before * heads;
        for (int b = b0; b < b1; ++b) {
            const int n = seq_tiles<NW>(seq_range(p, b));
            if (rem < static_cast<int64_t>(n) * heads) {
                scan[32] = b;
                scan[33] = rem / n;
                scan[34] = rem % n;
                break;
            }
            rem -= static_cast<int64_t>(n) * heads;
        }
    }
    __syncthreads();
    TileWalk<NW> ld, cu;      // the copies run NSTAGE - 1 tiles ahead of the arithmetic
    ld.b = static_cast<int>(scan[32]);
    ld.h = static_cast<int>(scan[33]);
    ld.t = static_cast<int>(scan[34]);
    ld.r = seq_range(p, ld.b);
    ld.t_end = seq_tiles<NW>(ld.r);
    cu = ld;
    __syncthreads();          // the ring takes over the scan's shared memory

    const uint32_t ring = sm100::smem_u32(smem) + warp * NCH * 512 + lane * 16;
    // key 16 of this warp's chunk of tile t, first key index; negative: no chunk
    auto chunk_key = [&](const TileWalk<NW>& w) {
        const int ch = w.t * NW + warp;
        if (ch >= w.r.n_chunks) return -1;
        return (ch < w.r.n_sink ? ch : w.r.lo + ch - w.r.n_sink) << 4;
    };
    auto visible = [&](const SeqRange& r, int key) { return key < r.len && (key >= r.win_lo || key < p.sinks); };
    // page of key chunk + lane % 16 of the walk's tile (-1: hidden or not a page)
    auto fetch_page = [&](const TileWalk<NW>& w) {
        const int k0 = chunk_key(w);
        int page = -1;
        if (k0 >= 0) {
            const int key = k0 + (lane & 15);
            if (visible(w.r, key)) {
                page = __ldg(p.block_table + static_cast<int64_t>(w.b) * p.table_stride + (key >> p.page_shift));
                if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages)) page = -2;
            }
        }
        return page;
    };
    int64_t loaded = 0;
    int page_next = fetch_page(ld);
    // live keys of the chunks in flight, one bit per key, NSTAGE deep
    uint32_t live_q[NSTAGE];
#pragma unroll
    for (int s = 0; s < NSTAGE; ++s) live_q[s] = 0;
    const int slot_mask = (1 << p.page_shift) - 1;
    auto issue = [&](int stage, uint32_t& live_out) {
        live_out = 0;
        if (loaded < steps) {
            const int k0 = chunk_key(ld);
            int page = page_next;
            if (page == -2) report_bad_index(p.status);
            const uint32_t live = __ballot_sync(0xffffffffu, page >= 0) & 0xffffu;
            live_out = live;
            if (live) {
                const int kvh = ld.h / p.sub;
                const uint32_t dst = ring + stage * C::STAGE_BYTES;
                const uint8_t* kb = p.k_cache + kvh * p.k_head + c * 16;
                const uint8_t* vb = p.v_cache + kvh * p.v_head + g * 16;
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const int row = 8 * n + g;
                    const int pg = __shfl_sync(0xffffffffu, page, row);
                    const uint8_t* src = pg >= 0 ? kb + pg * p.k_page + ((k0 + row) & slot_mask) * p.k_slot : p.k_cache;
#pragma unroll
                    for (int i = 0; i < KI; ++i) cp_async16(dst + (n * KI + i) * 512, pg >= 0 ? src + i * 64 : src, pg >= 0);
                }
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const int row = 8 * (n >> 1) + 2 * c + (n & 1);
                    const int pg = __shfl_sync(0xffffffffu, page, row);
                    const uint8_t* src = pg >= 0 ? vb + pg * p.v_page + ((k0 + row) & slot_mask) * p.v_slot : p.v_cache;
#pragma unroll
                    for (int i = 0; i < VI; ++i) cp_async16(dst + (2 * KI + n * VI + i) * 512, pg >= 0 ? src + i * 128 : src, pg >= 0);
                }
            }
            ld.next(p, heads);
            if (++loaded < steps) page_next = fetch_page(ld);
        }
        cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < NSTAGE - 1; ++s) issue(s, live_q[s]);

    uint32_t qa[KI][4], qb[KI][4];        // Q fragments: rows g and (GH == 16) g + 8
    float acc[VI][8][4];
    float m[2], l[2];                     // reference maximum of the raw scores and this thread's part of the sum, rows g, g + 8
    auto start_pair = [&]() {
        const int kvh = cu.h / p.sub, r0 = (cu.h - kvh * p.sub) * 16;
#pragma unroll
        for (int i = 0; i < KI; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) { qa[i][e] = 0; qb[i][e] = 0; }
            const uint8_t* qp = static_cast<const uint8_t*>(p.q) +
                                ((static_cast<int64_t>(cu.b) * p.H + kvh * p.group + r0 + g) * D + 32 * i + 8 * c) * 2;
            if (r0 + g < p.group) {
                const uint4 w = __ldg(reinterpret_cast<const uint4*>(qp));
                qa[i][0] = w.x; qa[i][1] = w.y; qa[i][2] = w.z; qa[i][3] = w.w;
            }
            if (GH == 16 && r0 + g + 8 < p.group) {
                const uint4 w = __ldg(reinterpret_cast<const uint4*>(qp + 8 * D * 2));
                qb[i][0] = w.x; qb[i][1] = w.y; qb[i][2] = w.z; qb[i][3] = w.w;
            }
        }
#pragma unroll
        for (int i = 0; i < VI; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int x = 0; x < 4; ++x) acc[i][e][x] = 0.f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
    };
    const float sc = p.scale_log2;
    bool fresh = true;
    int pair_first_t = cu.t;    // first tile of the current pair in this CTA's part
    int n_pairs = 0;            // pairs finished so far by this CTA (0: a cut pair goes to slot 0)

    for (int64_t s0 = 0; s0 < steps; s0 += NSTAGE) {
#pragma unroll
        for (int st = 0; st < NSTAGE; ++st) {
            const int64_t s = s0 + st;
            if (s >= steps) break;
            if (fresh) {
                start_pair();
                fresh = false;
                pair_first_t = cu.t;
            }
            issue((st + NSTAGE - 1) % NSTAGE, live_q[(st + NSTAGE - 1) % NSTAGE]);
            cp_async_wait<NSTAGE - 1>();
            const uint32_t live = live_q[st];
            if (live) {      // uniform over the warp
                const uint32_t src = ring + st * C::STAGE_BYTES;
                float sf[2][4];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    float even[4] = {0.f, 0.f, 0.f, 0.f}, odd[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < KI; ++i) {
                        const uint4 w = lds128(src + (n * KI + i) * 512);
                        mma16816<DTYPE>(even, qa[i][0], qb[i][0], qa[i][1], qb[i][1], w.x, w.y);
                        mma16816<DTYPE>(odd, qa[i][2], qb[i][2], qa[i][3], qb[i][3], w.z, w.w);
                    }
#pragma unroll
                    for (int x = 0; x < 4; ++x) sf[n][x] = even[x] + odd[x];
                }
                if (live != 0xffffu) {
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            if (!((live >> (8 * n + 2 * c + (x & 1))) & 1)) sf[n][x] = -INFINITY;
                }
                // advance the reference maximum only when a score ran ahead of it by more than 2^LAG (or there is none yet)
                float mx[2];
                mx[0] = fmaxf(fmaxf(sf[0][0], sf[0][1]), fmaxf(sf[1][0], sf[1][1]));
                mx[1] = fmaxf(fmaxf(sf[0][2], sf[0][3]), fmaxf(sf[1][2], sf[1][3]));
                bool ahead = m[0] == -INFINITY || (mx[0] - m[0]) * sc > LAG;
                if (GH == 16) ahead |= m[1] == -INFINITY || (mx[1] - m[1]) * sc > LAG;
                if (__any_sync(0xffffffffu, ahead)) {
#pragma unroll
                    for (int r = 0; r < GH / 8; ++r) {
                        float x = mx[r];
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));   // finite: the chunk has a live key
                        const float mn = fmaxf(m[r], x);
                        const float alpha = m[r] == -INFINITY ? 0.f : sm100::ex2_approx((m[r] - mn) * sc);
                        m[r] = mn;
                        l[r] *= alpha;
#pragma unroll
                        for (int i = 0; i < VI; ++i)
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                if (GH == 8) {
#pragma unroll
                                    for (int x4 = 0; x4 < 4; ++x4) acc[i][e][x4] *= alpha;
                                } else {
                                    acc[i][e][2 * r] *= alpha;
                                    acc[i][e][2 * r + 1] *= alpha;
                                }
                            }
                    }
                }
                uint32_t hi[2][2], lo[2][2];   // [key half][row half]
#pragma unroll
                for (int r = 0; r < GH / 8; ++r) {
                    const float off = P_OFF - (m[r] == -INFINITY ? 0.f : m[r] * sc);   // every score so far -inf: P = 0
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        float p0 = sm100::ex2_approx(fmaf(sf[n][2 * r], sc, off)), p1 = sm100::ex2_approx(fmaf(sf[n][2 * r + 1], sc, off));
                        if (live != 0xffffu) {      // explicit zeros: with scale 0 the hidden scores' -inf * 0 is no number
                            const uint32_t bits = live >> (8 * n + 2 * c);
                            p0 = (bits & 1) ? p0 : 0.f;
                            p1 = (bits & 2) ? p1 : 0.f;
                        }
                        l[r] += p0 + p1;
                        split2<DTYPE>(p0, p1, hi[n][r], lo[n][r]);
                    }
                }
#pragma unroll
                for (int i = 0; i < VI; ++i) {
                    uint32_t v[4][4];
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const uint4 w = lds128(src + (2 * KI + n * VI + i) * 512);
                        v[n][0] = w.x; v[n][1] = w.y; v[n][2] = w.z; v[n][3] = w.w;
                    }
#pragma unroll
                    for (int w = 0; w < 4; ++w)
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const uint32_t vb0 = __byte_perm(v[0][w], v[1][w], x ? 0x7632 : 0x5410);
                            const uint32_t vb1 = __byte_perm(v[2][w], v[3][w], x ? 0x7632 : 0x5410);
                            float* a = acc[i][2 * w + x];
                            if (GH == 8) {
                                mma16816<DTYPE>(a, hi[0][0], lo[0][0], hi[1][0], lo[1][0], vb0, vb1);
                            } else {
                                mma16816<DTYPE>(a, hi[0][0], hi[0][1], hi[1][0], hi[1][1], vb0, vb1);
                                mma16816<DTYPE>(a, lo[0][0], lo[0][1], lo[1][0], lo[1][1], vb0, vb1);
                            }
                        }
                }
            }
            // ---- end of the pair, or of this CTA's part: merge the warps ----
            const bool end_pair = cu.t + 1 == cu.t_end;
            if (end_pair || s + 1 == steps) {
#pragma unroll
                for (int r = 0; r < GH / 8; ++r) {
                    float x = l[r];
                    x += __shfl_xor_sync(0xffffffffu, x, 1);
                    x += __shfl_xor_sync(0xffffffffu, x, 2);
                    if (c == 0) merge_ml[warp * GH + 8 * r + g] = make_float2(m[r] * sc, x);   // x = 0: no key, the first value is not used
                }
#pragma unroll
                for (int i = 0; i < VI; ++i)
#pragma unroll
                    for (int r = 0; r < GH / 8; ++r)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            // value dims 64 i + 16 c + 8 j + (0 .. 7) of row g + 8 r
                            float* dst = merge + (warp * GH + 8 * r + g) * C::ROW + 64 * i + 16 * c + 8 * j;
                            float v[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = GH == 8 ? acc[i][e][j] + acc[i][e][2 + j] : acc[i][e][2 * r + j];
                            *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
                            *reinterpret_cast<float4*>(dst + 4) = make_float4(v[4], v[5], v[6], v[7]);
                        }
                __syncthreads();
                const int kvh = cu.h / p.sub, r0 = (cu.h - kvh * p.sub) * 16;
                const int rows = p.group - r0 < GH ? p.group - r0 : GH;
                const bool whole = end_pair && pair_first_t == 0;
                float* part = p.parts + (2 * static_cast<int64_t>(blockIdx.x) + (n_pairs > 0 ? 1 : 0)) * C::PART_FLOATS;
                for (int e = tid; e < rows * (D / 4); e += C::THREADS) {
                    const int row = e / (D / 4), d4 = e % (D / 4);
                    float mm = -INFINITY;
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        const float2 ml = merge_ml[w * GH + row];
                        if (ml.y != 0.f) mm = fmaxf(mm, ml.x);
                    }
                    float sum = 0.f;
                    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
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
                    if (whole) {
                        const int64_t out_row = static_cast<int64_t>(cu.b) * p.H + kvh * p.group + r0 + row;
                        const float inv = sum != 0.f ? 1.f / sum : 0.f;
                        uint2 w;
                        w.x = sm100::pack2<DTYPE>(o.x * inv, o.y * inv);
                        w.y = sm100::pack2<DTYPE>(o.z * inv, o.w * inv);
                        reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.o) + out_row * D * 2)[d4] = w;
                        if (d4 == 0) p.lse[out_row] = sum != 0.f ? (mm - P_OFF) * 0.6931471805599453f + logf(sum) : -INFINITY;
                    } else {
                        *reinterpret_cast<float4*>(part + row * D + 4 * d4) = o;
                        if (d4 == 0) *reinterpret_cast<float2*>(part + GH * D + 2 * row) = make_float2(mm, sum);
                    }
                }
                __syncthreads();     // the merge buffer may be written again
                ++n_pairs;
                fresh = true;
            }
            cu.next(p, heads);
        }
    }
    cp_async_wait<0>();
}

// Joins the partial results of the pairs that more than one CTA of the first kernel worked on, and writes the rows of
// sequences without a visible key.  One CTA per (sequence, K/V head, head part); the list layout is worked out before
// the first kernel's results are waited for.
template <int D, int DTYPE, int GH>
__global__ void __launch_bounds__(256)
attn_paged_join_kernel(const DecodeParams p) {
    using C = DecodeCfg<D, GH>;
    constexpr int NW = C::NW;
    constexpr float P_OFF = ExpRange<DTYPE>::P_OFF;
    __shared__ int64_t red[16];
    __shared__ float wgt[GH][2 * kMaxCtas + 2];
    const int heads = p.Hkv * p.sub;
    const int b = blockIdx.x / heads, h = blockIdx.x - b * heads;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int64_t before = 0, total = 0;
    for (int x = tid; x < p.B; x += 256) {
        const int n = seq_tiles<NW>(seq_range(p, x));
        total += n;
        if (x < b) before += n;
    }
    before = warp_sum(before);
    total = warp_sum(total);
    if (lane == 0) {
        red[warp] = before;
        red[8 + warp] = total;
    }
    __syncthreads();
    before = total = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        before += red[w];
        total += red[8 + w];
    }
    total *= heads;
    const int n = seq_tiles<NW>(seq_range(p, b));
    // Every CTA waits for the first kernel, also one without work: in a graph this kernel's end stands for both.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int kvh = h / p.sub, r0 = (h - kvh * p.sub) * 16;
    const int rows = p.group - r0 < GH ? p.group - r0 : GH;
    const int64_t row0 = static_cast<int64_t>(b) * p.H + kvh * p.group + r0;
    if (n == 0) {
        for (int e = tid; e < rows * (D / 4); e += 256) {
            reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.o) + row0 * D * 2)[e] = make_uint2(0u, 0u);
            if (e < rows) p.lse[row0 + e] = -INFINITY;
        }
        return;
    }
    const int64_t t0 = before * heads + static_cast<int64_t>(h) * n, t1 = t0 + n;
    const int ctas = cta_count(total, p.grid);
    const int c0 = cta_of_tile(total, t0, ctas), c1 = cta_of_tile(total, t1 - 1, ctas);
    if (c0 == c1) return;                        // finished by the first kernel
    // the pair is the first of every CTA but, perhaps, of c0
    const int slot0 = 2 * c0 + (cta_begin(total, c0, ctas) < t0 ? 1 : 0);
    const int np = c1 - c0 + 1;
    auto slot = [&](int i) { return i == 0 ? slot0 : 2 * (c0 + i); };
    for (int e = tid; e < rows * np; e += 256) {
        const int row = e / np, i = e - row * np;
        const float2 ml = __ldcg(reinterpret_cast<const float2*>(p.parts + static_cast<int64_t>(slot(i)) * C::PART_FLOATS + GH * D + 2 * row));
        wgt[row][2 * i] = ml.x;
        wgt[row][2 * i + 1] = ml.y;
    }
    __syncthreads();
    for (int row = warp; row < rows; row += 8) {     // weights exp2(m_i - max), scaled by 1 / sum
        float mm = -INFINITY;
        for (int i = lane; i < np; i += 32)
            if (wgt[row][2 * i + 1] != 0.f) mm = fmaxf(mm, wgt[row][2 * i]);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, off));
        float sum = 0.f;
        for (int i = lane; i < np; i += 32) {
            const float l = wgt[row][2 * i + 1];
            const float f = l != 0.f ? sm100::ex2_approx(wgt[row][2 * i] - mm) : 0.f;
            sum = fmaf(f, l, sum);
            wgt[row][2 * i] = f;
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        const float inv = sum != 0.f ? 1.f / sum : 0.f;
        for (int i = lane; i < np; i += 32) wgt[row][2 * i] *= inv;
        if (lane == 0) p.lse[row0 + row] = sum != 0.f ? (mm - P_OFF) * 0.6931471805599453f + logf(sum) : -INFINITY;
    }
    __syncthreads();
    for (int e = tid; e < rows * (D / 4); e += 256) {
        const int row = e / (D / 4), d4 = e % (D / 4);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int i = 0; i < np; ++i) {
            const float f = wgt[row][2 * i];
            const float4 v = __ldcg(reinterpret_cast<const float4*>(p.parts + static_cast<int64_t>(slot(i)) * C::PART_FLOATS + row * D + 4 * d4));
            if (f != 0.f) {     // a part without a visible key adds nothing
                o.x = fmaf(f, v.x, o.x);
                o.y = fmaf(f, v.y, o.y);
                o.z = fmaf(f, v.z, o.z);
                o.w = fmaf(f, v.w, o.w);
            }
        }
        uint2 w;
        w.x = sm100::pack2<DTYPE>(o.x, o.y);
        w.y = sm100::pack2<DTYPE>(o.z, o.w);
        reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.o) + (row0 + row) * D * 2)[d4] = w;
    }
}

}  // namespace attn_paged
