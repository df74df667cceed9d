// The gradient of attn_rope.cuh's forward pass with all rows moved by TMA, for dense [B, S, heads, D] tensors.
//
// A tile is 8 tokens x 1024 / D heads of one of the three tensors (16 KB, and as much of the forward pass's input beside it),
// or, of a tensor with fewer heads, as many more tokens (8 tokens of 2 heads of 64 would fill an eighth of it: 24578 tokens of
// 2 + 2 x 2 such heads took 51 us, now 22), laid out [head][token][D] in shared memory whatever the strides of its source
// are (the tensor maps order the axes), so that the result is written over it and leaves through another map: the change of
// layout costs nothing.  One CTA per SM walks a contiguous run of tiles; a ring of 192 KB keeps loads and stores in flight
// while 16 warps work.  The register form in
// attn_rope.cuh (a load, arithmetic and a store per warp: 64 KB in flight at most, and only while nobody computes) takes
// 70 us for 4 x 2048 tokens x 48 heads of 128, this one 59 (4.8 TB/s; 50 with the arithmetic left out).  What bounds it now
// is the arithmetic: its shuffles' latency, which 16 warps of 96 registers do not hide, and half of all issue slots.  Two
// groups of warps on alternate tiles (61 us), two or four rows at a time (78 us and more: fewer warps for their registers)
// are slower.  For the forward pass, with half the arithmetic and no second operand, this form gains nothing over the
// registers (71 us either way for 16384 tokens x 48 heads of 128).
//
//   warps 0-15  arithmetic: warp w has token w % 8 and every other group of heads, and the rotation's factors stay in registers
//               while tiles of the same tokens pass; in a tile of more tokens each row brings its own
//   warp  16    loads (one lane)
//   warp  17    stores (one lane); frees a stage once its store has read it
//
// Every wait is bounded (see sm100_ptx.cuh).
#pragma once
#include <type_traits>

#include "attn_rope.cuh"
#include "attn_tc_common.cuh"

namespace attn_rope {
template <int D>
struct TmaCfg {
    static constexpr int ROWS = 8192 / D;                     // tokens x heads of a tile
    static constexpr int TILE = ROWS * D * 2;
    static constexpr int STAGE = 2 * TILE;                    // the output's gradient, and the forward pass's input
    static constexpr int NSTAGE = 196608 / STAGE;
    static constexpr int WARPS = 16, THREADS = (WARPS + 2) * 32;
    static constexpr int RPW = 256 / D;                       // rows of a warp at a time
    static constexpr int SMEM = 128 + NSTAGE * STAGE + 3 * NSTAGE * 8 + 16;
    static_assert(2 * WARPS * RPW * D * 4 <= NSTAGE * STAGE && SMEM <= 232448, "shared memory (the ring later holds the warps' sums)");
};

struct TmaParams {
    RopeParams r;             // heads, weights, table, positions, eps, S, status
    int units[3];             // groups of heads of q, k, v, 1 << hb_shift of them to a tile
    int hb_shift[3], tb_shift[3];   // log2 of a tile's heads and tokens
    int block_shift;          // log2 of the tokens of a block: the largest tile's
    int token_blocks;         // per sequence
    int per_block;            // tiles of a block: those of q, k, v
    int64_t tiles;
    float* partial;           // [CTA][2][D]: sums of q's and k's weight gradients
#ifdef ATTN_TEST_HOOKS
    int test_skip_tile;       // test build only: the tile of every CTA whose copies are left out (-1: none)
#endif
};

struct TmaMaps {
    CUtensorMap dy[3];        // dq, dk, dv (head-major)
    CUtensorMap x[2];         // q, k
    CUtensorMap out[3];
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
        : "memory");
}
__device__ __forceinline__ void tma_store_4d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(src), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
                 : "memory");
}

__device__ __forceinline__ uint4 lds_row(uint32_t row, const Place& at) {
    uint4 x;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(row + 2 * at.a) : "memory");
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.z), "=r"(x.w) : "r"(row + 2 * at.b) : "memory");
    return x;
}
__device__ __forceinline__ void sts_row(uint32_t row, const Place& at, const uint4& x) {
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(row + 2 * at.a), "r"(x.x), "r"(x.y) : "memory");
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(row + 2 * at.b), "r"(x.z), "r"(x.w) : "memory");
}

// A CTA's walk over its run of tiles: by sequence, token block, tensor, (PACKED) tokens inside the block, heads.
template <bool PACKED>
struct TileAt {
    int b, tb, kind, unit, sub;
    __device__ __forceinline__ int subs(const TmaParams& p) const { return PACKED ? 1 << (p.block_shift - p.tb_shift[kind]) : 1; }
    __device__ __forceinline__ void start(const TmaParams& p, int64_t tile) {
        const int64_t block = tile / p.per_block;
        int u = static_cast<int>(tile - block * p.per_block);
        b = static_cast<int>(block / p.token_blocks);
        tb = static_cast<int>(block - static_cast<int64_t>(b) * p.token_blocks);
        for (kind = 0; kind < 2; ++kind) {
            const int n = p.units[kind] * subs(p);
            if (u < n) break;
            u -= n;
        }
        sub = PACKED ? u / (p.units[kind] > 0 ? p.units[kind] : 1) : 0;
        unit = u - sub * p.units[kind];
    }
    // true: the next tile belongs to other tokens, or (PACKED) another tensor
    __device__ __forceinline__ bool next(const TmaParams& p) {
        if (++unit < p.units[kind]) return false;
        unit = 0;
        if (PACKED) {
            if (++sub < subs(p)) return true;
            sub = 0;
        }
        bool other = PACKED;
        do {
            if (++kind == 3) {
                kind = 0;
                other = true;
                if (++tb == p.token_blocks) {
                    tb = 0;
                    ++b;
                }
            }
        } while (p.units[kind] == 0);
        return other;
    }
    __device__ __forceinline__ int token0(const TmaParams& p) const {
        return PACKED ? (tb << p.block_shift) + (sub << p.tb_shift[kind]) : tb * 8;
    }
    __device__ __forceinline__ int head0(const TmaParams& p) const { return unit << p.hb_shift[kind]; }
};

// PACKED: q or k has tiles of more than 8 tokens (a form of its own: what their rows need costs the others registers).
template <int D, int DTYPE, bool PACKED, bool AXES>
__global__ void __launch_bounds__(TmaCfg<D>::THREADS, 1)
attn_rope_bwd_tma_kernel(const __grid_constant__ TmaMaps maps, const __grid_constant__ TmaParams p) {
    using C = TmaCfg<D>;
    constexpr int NST = C::NSTAGE, LPR = D / 8, RPW = C::RPW;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (sm100::smem_u32(smem_raw) + 127u) & ~127u;
    const uint32_t bars = base + NST * C::STAGE;              // full[NST], done[NST], empty[NST]
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_raw + (bars - sm100::smem_u32(smem_raw)) + 3 * NST * 8);
    auto full = [&](int s) { return bars + 8 * s; };
    auto done = [&](int s) { return bars + 8 * (NST + s); };
    auto empty = [&](int s) { return bars + 8 * (2 * NST + s); };
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int s = 0; s < NST; ++s) {
            sm100::mbar_init(full(s), 1);
            sm100::mbar_init(done(s), C::WARPS);
            sm100::mbar_init(empty(s), 1);
        }
        sm100::fence_barrier_init();
        sm100::fence_proxy_async_smem();
    }
    __syncthreads();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t first = p.tiles * blockIdx.x / gridDim.x;
    const int n = static_cast<int>(p.tiles * (blockIdx.x + 1) / gridDim.x - first);
    TileAt<PACKED> at_tile;
    if (n > 0) at_tile.start(p, first);
    F2 dw[2][4];                                              // this lane's part of the weights' gradients
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) dw[k][e] = F2(0.f, 0.f);

    if (warp == C::WARPS) {
        // =========================== loads ===========================
        if (lane == 0) {
            for (int i = 0; i < n; ++i) {
                const int s = i % NST;
                if (!sm100::mbar_wait(empty(s), ((i / NST) & 1) ^ 1, abort_flag)) break;
                const int kind = at_tile.kind, h0 = at_tile.head0(p), t0 = at_tile.token0(p);
                const bool with_x = kind < 2 && p.r.weight[kind] != nullptr;
                sm100::mbar_arrive_expect_tx(full(s), with_x ? 2 * C::TILE : C::TILE);
#ifdef ATTN_TEST_HOOKS
                if (i == p.test_skip_tile) {                  // this tile's copies are left out
                    at_tile.next(p);
                    continue;
                }
#endif
                tma_load_4d(base + s * C::STAGE, &maps.dy[kind], full(s), 0, t0, h0, at_tile.b);
                if (with_x) tma_load_4d(base + s * C::STAGE + C::TILE, &maps.x[kind & 1], full(s), 0, t0, h0, at_tile.b);
                at_tile.next(p);
            }
        }
    } else if (warp == C::WARPS + 1) {
        // =========================== stores ===========================
        if (lane == 0) {
            constexpr int PENDING = 2;                        // stores that may still be reading their stage
            bool ok = true;
            for (int i = 0; i < n; ++i) {
                const int s = i % NST;
                if (!(ok = sm100::mbar_wait(done(s), (i / NST) & 1, abort_flag))) break;
                // (the last block of a sequence may end before all of its tiles begin)
                if (at_tile.token0(p) < p.r.S)
                    tma_store_4d(&maps.out[at_tile.kind], base + s * C::STAGE, 0, at_tile.token0(p), at_tile.head0(p), at_tile.b);
                sm100::tma_store_commit();
                if (i >= PENDING) {
                    sm100::tma_store_wait_read<PENDING>();
                    sm100::mbar_arrive(empty((i - PENDING) % NST));
                }
                at_tile.next(p);
            }
            sm100::tma_store_wait_all<0>();                   // shared memory must outlive its readers
        }
    } else {
        // =========================== arithmetic ===========================
        const int sub = lane / LPR, l = lane % LPR;
        const Place at(p.r, l);
        const PairAxes axes = PairAxes::of_lane<AXES>(p.r, l);
        Turn turn;                                            // of the token whose rows this lane works on
        F2 w[4];
        int my_kind = -1;                                     // tensor that w belongs to
        bool new_tokens = true;
        auto load_turn = [&](int b, int token) {
            const bool bad = !turn.load_token<AXES>(p.r, static_cast<int64_t>(b) * p.r.S + token, token, axes, l, at);
            if (bad) {                                        // the token's gradients, and with them the weights', become NaN
#pragma unroll
                for (int e = 0; e < 4; ++e) turn.cs[e] = F2(__int_as_float(0x7fffffff), __int_as_float(0x7fffffff));
            }
        };
        for (int i = 0; i < n; ++i) {
            const int s = i % NST, kind = at_tile.kind, h0 = at_tile.head0(p), t0 = at_tile.token0(p);
            const bool norm = kind < 2 && p.r.weight[kind] != nullptr;
            const int hb = kind < 2 ? p.hb_shift[kind] : 0;
            const bool wide = kind < 2 && (!PACKED || p.tb_shift[kind] == 3);  // 8 tokens: a warp has one of them
            if (wide && new_tokens) {
                if (t0 + (warp & 7) < p.r.S) load_turn(at_tile.b, t0 + (warp & 7));
                new_tokens = false;
            }
            if (norm && kind != my_kind) load_weight<DTYPE>(p.r.weight[kind], p.r.weight_f32, at, w);
            my_kind = kind;
            // (the vote keeps a warp together where a wait runs out: its lanes shuffle)
            if (!__all_sync(0xffffffffu, sm100::mbar_wait(full(s), (i / NST) & 1, abort_flag))) break;
            if (kind < 2) {
                const int tb = p.tb_shift[kind], left = p.r.heads[kind] - h0;        // heads of this tile that exist
                by_form(p.r, D, [&](auto inter, auto whole_head) {
#pragma unroll
                    for (int k = 0; k < C::ROWS / (C::WARPS * RPW); ++k) {
                        int h, tok;                           // this lane's row
                        if (!PACKED || wide) {
                            h = (k * (C::WARPS / 8) + (warp >> 3)) * RPW;
                            tok = warp & 7;
                            if (h >= left || t0 + tok >= p.r.S) break;        // uniform over the warp
                            h += sub;
                        } else {
                            const int r = (k * C::WARPS + warp) * RPW + sub;
                            h = r & ((1 << hb) - 1);
                            tok = r >> hb;
                            if (t0 + tok < p.r.S) load_turn(at_tile.b, t0 + tok);
                        }
                        const bool live = h < left && t0 + tok < p.r.S;
                        const uint32_t row = base + s * C::STAGE + ((h << tb) + tok) * D * 2;
                        F2 g[4], y[4];
                        unpack_row<DTYPE>(lds_row(row, at), g);
                        turn_values<decltype(inter)::value, decltype(whole_head)::value>(y, g, turn.cs, turn.sn, at.turns);
                        if (norm) {
                            F2 x[4], hx[4], ss(0.f, 0.f), gx(0.f, 0.f);
                            unpack_row<DTYPE>(lds_row(row + C::TILE, at), x);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                ss = fma2(x[e], x[e], ss);
                                hx[e] = y[e] * x[e];
                                gx = fma2(hx[e], w[e], gx);
                            }
                            const float r = rsqrtf(row_sum<LPR>(ss.sum()) * (1.f / D) + p.r.eps);
                            const float k3 = -row_sum<LPR>(gx.sum()) * (1.f / D) * r * r * r;
                            const F2 rr(r, r), kk(k3, k3);
                            // (rows that do not exist are zero in x and g: at eps 0 their r is infinite)
                            if (live) {
                                if (kind == 0) {
#pragma unroll
                                    for (int e = 0; e < 4; ++e) dw[0][e] = fma2(hx[e], rr, dw[0][e]);
                                } else {
#pragma unroll
                                    for (int e = 0; e < 4; ++e) dw[1][e] = fma2(hx[e], rr, dw[1][e]);
                                }
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e) y[e] = fma2(y[e], w[e] * rr, kk * x[e]);
                        }
                        sts_row(row, at, pack_row<DTYPE>(y));
                    }
                });
                sm100::fence_proxy_async_smem();              // the store reads what was just written
            }
            __syncwarp();
            if (lane == 0) sm100::mbar_arrive(done(s));
            if (at_tile.next(p)) new_tokens = true;
        }
    }
    __syncthreads();                                          // loads and stores are over: the ring is free
    // this CTA's sums of the weight gradients: the warps' side by side, then column by column, always in the same order
    float* sums = reinterpret_cast<float*>(smem_raw + (base - sm100::smem_u32(smem_raw)));
    constexpr int ROWS = C::WARPS * RPW;
    if (warp < C::WARPS) {
        const int l = lane % LPR;
        const Place at(p.r, l);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float* mine = sums + (k * ROWS + warp * RPW + lane / LPR) * D;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                dw[k][e].get(mine[at.a + 2 * e], mine[at.a + 2 * e + 1]);
                dw[k][2 + e].get(mine[at.b + 2 * e], mine[at.b + 2 * e + 1]);
            }
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += C::THREADS) {
        float x = 0.f;
#pragma unroll 8
        for (int r = 0; r < ROWS; ++r) x += sums[((i / D) * ROWS + r) * D + i % D];
        p.partial[static_cast<int64_t>(blockIdx.x) * 2 * D + i] = x;
    }
    if (threadIdx.x == 0 && *abort_flag != 0) attn_tc::report_timeout(p.r.status);
}

}  // namespace attn_rope
